"""The operators around the int4 linears of a decoder layer, as a scoring service calls them,
case by case.  The kinds:

  norm      the residual stream's update by a block's output (normalised, gated, scaled) and the
            norm that the next block reads (w4a16.residual_norm);
  rotary    rotary positions on the queries and keys of fused projections, in place, for packed
            prompts (w4a16.rotary) and for the tokens that a cache has grown by (w4a16.kv_rotary);
  logprobs  log probabilities of given tokens, entropy and best alternatives from a head's
            logits (w4a16.log_probs);
  adapters  each sequence's own low-rank adapter added to a shared projection's output
            (w4a16.add_adapters).

Definitions, with bf16 inputs and outputs unless said:

  norm      h = scale * residual + gate * post(block), out = pre(h); pre and post are
            v / sqrt(mean(v^2) + eps) * (offset + weight) (rms), or the same of v - mean(v) (layer),
            plus a bias; out is of h before its rounding.
  rotary    pairs (a, b) -> (a cos t - b sin t, a sin t + b cos t), t = position * theta_i, i < rot / 2;
            pair i is elements (i, i + rot / 2) of a head (half) or (2i, 2i + 1) (pairs).
  logprobs  fp32: x[target] - lse(x) (0 where the target is -1), -sum p log p, and the k largest
            logits' indices and log probabilities, in descending order, equal ones by index.
  adapters  out = base + scale[a] * (x A[a]^T) B[a]^T with the adapter a of the row's sequence
            (-1: out = base).
"""
from __future__ import annotations

import itertools
import math

import torch

own = False

DEVICE = "cuda"
LARGEST = 4.0e9  # bytes that a drawn case reads and writes, at most
_W = None


def _lib():
    global _W
    if _W is None:
        from paper_2608_30877_gb300 import w4a16
        _W = w4a16
    return _W


def _norm(name, M, D, norm="rms", post=False, gate=0, bias=False, bits=16, scale=1.0):
    """gate: its rows (0: none, 1: one for all tokens, -1: each token's own)."""
    return {"name": name, "kind": "norm", "M": M, "D": D, "norm": norm, "post": post, "gate": gate, "bias": bias,
            "bits": bits, "scale": scale}


def _rotary(name, H, Hkv, rot, layout, nseq, shortest, longest, first=0, scaling="none", cached=False):
    return {"name": name, "kind": "rotary", "H": H, "Hkv": Hkv, "rot": rot, "layout": layout, "nseq": nseq,
            "shortest": shortest, "longest": longest, "first": first, "scaling": scaling, "cached": cached}


def _logprobs(name, M, V, bits, k, pad=0, masked=0):
    """pad: columns between rows; masked: of how many rows one is left to a grammar's tokens."""
    return {"name": name, "kind": "logprobs", "M": M, "V": V, "bits": bits, "k": k, "pad": pad, "masked": masked}


def _adapters(name, K, N, R, pool, nseq, shortest, longest):
    return {"name": name, "kind": "adapters", "K": K, "N": N, "R": R, "pool": pool, "nseq": nseq, "shortest": shortest,
            "longest": longest}


def listed():
    return [
        # one pair's next token between two blocks: all latency
        _norm("norm_step", 1, 12288),
        # the packed prefill of 64 ragged pairs, between attention and MLP
        _norm("norm_64_pairs", 39004, 12288),
        # a block with norms on both sides, gated, on a stream held in fp32
        _norm("norm_sandwich", 4097, 8200, "layer", post=True, gate=1, bias=True, bits=32, scale=0.5),
        # one decode step of 64 pairs over the cache
        _rotary("rotary_step", 96, 96, 128, "half", 64, 200, 1024, cached=True),
        # prefill of the 64 pairs
        _rotary("rotary_64_pairs", 96, 96, 128, "half", 64, 200, 1024),
        # chunks of a few very long contexts, half of each head rotated, scaled beyond the trained length
        _rotary("rotary_long_part", 64, 8, 64, "pairs", 3, 2001, 4096, first=100000, scaling="index"),
        # one token's distribution with its 20 best alternatives
        _logprobs("logprobs_step", 1, 131072, 16, 20),
        # scoring four thousand prompt tokens
        _logprobs("logprobs_prompt", 4099, 131072, 16, 0),
        # many alternatives of a few hundred tokens from fp32 logits of odd width, some rows under a grammar's mask
        _logprobs("logprobs_top", 513, 100003, 32, 64, masked=4),
        # one decode step of 64 requests with 48 adapters on the fused QKV projection
        _adapters("adapters_step", 12288, 36864, 16, 48, 64, 1, 1),
        # prefill of the 64 pairs, each for one of eight targets' adapters, on the output projection
        _adapters("adapters_64_pairs", 12288, 12288, 16, 8, 64, 200, 1024),
        # a few short prompts on the down projection with adapters of a larger rank
        _adapters("adapters_rank64", 49152, 12288, 64, 3, 5, 1, 300),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = [(96, 96), (32, 32), (16, 16), (96, 8), (64, 8), (32, 4), (20, 1), (8, 2)]


def draw(rng):
    kind = rng.choice(["norm", "rotary", "logprobs", "adapters"])
    if kind == "norm":
        D = rng.choice([12288, 4096, 49152, _log_int(rng, 64, 20000), 8 * _log_int(rng, 8, 2500)])
        M = _log_int(rng, 1, max(2, min(65536, int(LARGEST / (D * 14)))))
        post = rng.random() < 0.5
        return {"kind": kind, "M": M, "D": D, "norm": rng.choice(["rms", "rms", "layer"]), "post": post,
                "gate": rng.choice([0, 0, 1, -1]), "bias": rng.random() < 0.3, "bits": rng.choice([16, 16, 32]),
                "scale": rng.choice([1.0, 1.0, 0.7])}
    if kind == "rotary":
        H, Hkv = rng.choice(HEADS)
        nseq = _log_int(rng, 1, 256)
        most = max(2, min(8192, int(LARGEST / ((H + Hkv) * 512) / nseq)))
        longest = _log_int(rng, 1, most)
        return {"kind": kind, "H": H, "Hkv": Hkv, "rot": rng.choice([128, 128, 64, 32, 96]),
                "layout": rng.choice(["half", "pairs"]), "nseq": nseq,
                "shortest": rng.choice([longest, rng.randint(1, longest), 1]), "longest": longest,
                "first": rng.choice([0, 0, _log_int(rng, 1, 1000000)]),
                "scaling": rng.choice(["none", "linear", "index", "turns"]), "cached": rng.random() < 0.4}
    if kind == "logprobs":
        V = rng.choice([131072, 50001, 32000, _log_int(rng, 64, 262144)])
        bits = rng.choice([16, 16, 32])
        k = rng.choice([0, 1, 5, 20, 64])
        # (the plain form orders 64-bit keys)
        M = _log_int(rng, 1, max(2, min(8192, int((2.0e9 if k == 0 else 3.0e8) / (V * bits // 8)))))
        return {"kind": kind, "M": M, "V": V, "bits": bits, "k": k, "pad": rng.choice([0, 0, -V % 64, 3]),
                "masked": rng.choice([0, 0, 3])}
    K, N = rng.choice([(12288, 36864), (12288, 12288), (49152, 12288), (4096, 4096),
                       (64 * _log_int(rng, 2, 200), _log_int(rng, 16, 20000))])
    R = rng.choice([8, 16, 16, 32, 64, 40])
    nseq = _log_int(rng, 1, 128)
    pool = _log_int(rng, 1, 64)
    most = max(1, min(2048, int(2.0e9 / (2 * (K + 2 * N)) / nseq)))
    longest = rng.choice([1, _log_int(rng, 1, most)])
    return {"kind": kind, "K": K, "N": N, "R": R, "pool": pool, "nseq": nseq,
            "shortest": rng.choice([longest, rng.randint(1, longest), 1]), "longest": longest}


# ---------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _lengths(case):
    """Ragged over the range, the same for every seed, so that a case has one work."""
    span = case["longest"] - case["shortest"] + 1
    return [case["shortest"] + (i * 0x9E3779B1 >> 8) % span for i in range(1, case["nseq"] + 1)]


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEVICE)


def _normal(gen, shape, dtype=torch.bfloat16, scale=1.0):
    x = torch.empty(shape, dtype=dtype, device=DEVICE).normal_(generator=gen)
    return x.mul_(scale) if scale != 1.0 else x


EPS = 1e-5
OFFSET = 1.0
BASE = 500000.0
TRAINED = 8192  # tokens that the frequencies were trained for
# factor; turns within the trained length below which a frequency is divided by it, and above which it is kept
SCALING = {"none": (1.0, 0.0, 0.0), "linear": (4.0, 0.0, 0.0), "index": (32.0, 1.0, 32.0), "turns": (8.0, 1.0, 4.0)}


def _prepare_norm(case, gen, s):
    M, D = case["M"], case["D"]
    stream = torch.bfloat16 if case["bits"] == 16 else torch.float32
    # a residual stream has a few dimensions far larger than the others
    s["residual"] = _normal(gen, (M, D), stream, 2.0)
    s["residual"][:, ::max(1, D // 7)] *= 30.0
    s["block"] = _normal(gen, (M, D))
    s["weight"] = _normal(gen, (D,), scale=0.2)  # (an offset of one comes on top)
    s["bias"] = _normal(gen, (D,), scale=0.1) if case["bias"] else None
    s["post_weight"] = _normal(gen, (D,), scale=0.2) if case["post"] else None
    s["post_bias"] = _normal(gen, (D,), scale=0.1) if case["post"] and case["bias"] else None
    s["gate"] = _normal(gen, (1 if case["gate"] == 1 else M, D)) if case["gate"] else None


def _prepare_rotary(case, gen, s):
    lengths = _lengths(case)
    n, cached = case["nseq"], case["cached"]
    step = cached and case["longest"] > 1  # a step of sequences that long; else prompts
    rows = n if step else sum(lengths)
    s["qkv"] = _normal(gen, (rows, (case["H"] + 2 * case["Hkv"]) * 128))
    s["seq_start"] = None if step else _i32(list(itertools.accumulate(lengths, initial=0)))
    s["first"] = torch.randint(case["first"], case["first"] + 100, (n,), generator=gen, device=DEVICE, dtype=torch.int32)
    if cached:
        # slots in any order; the rows are the last tokens of their sequences
        s["slots"] = torch.randperm(n + 3, generator=gen, device=DEVICE)[:n].to(torch.int32)
        T = 64
        pages = -(-(case["first"] + 100 + case["longest"]) // T)
        s["seq_len"] = torch.zeros(n + 3, dtype=torch.int32, device=DEVICE)
        s["seq_len"][s["slots"].long()] = s["first"] + _i32(lengths)
        s["page_table"] = torch.zeros((n + 3, pages), dtype=torch.int32, device=DEVICE)
        s["page_refs"] = torch.ones(1, dtype=torch.int32, device=DEVICE)
        s["pages"] = torch.zeros((1, 2, 1, case["Hkv"], T, 128), dtype=torch.bfloat16, device=DEVICE)
    if own:  # what a program makes once
        W = _lib()
        factor, low, high = SCALING[case["scaling"]]
        scaling = {"none": W.ROTARY_SCALE_NONE, "linear": W.ROTARY_SCALE_LINEAR, "index": W.ROTARY_SCALE_BY_INDEX,
                   "turns": W.ROTARY_SCALE_BY_TURNS}[case["scaling"]]
        s["table"] = W.RotaryTable(case["rot"], BASE, scaling, factor, TRAINED, low, high,
                                   layout=W.ROTARY_HALF if case["layout"] == "half" else W.ROTARY_PAIRS)
        if cached:
            s["cache"] = W.KVCache.from_tensors(s["pages"], s["page_table"], s["seq_len"], s["page_refs"])


def _prepare_logprobs(case, gen, s):
    M, V = case["M"], case["V"]
    dtype = torch.bfloat16 if case["bits"] == 16 else torch.float32
    logits = _normal(gen, (M, V + case["pad"]), dtype, 2.5)[:, :V]
    s["targets"] = torch.randint(0, V, (M,), generator=gen, device=DEVICE, dtype=torch.int32)
    # a model is fairly sure of most tokens
    rows = torch.arange(M, device=DEVICE)
    logits[rows, s["targets"].long()] += torch.rand(M, generator=gen, device=DEVICE).mul_(20).to(dtype)
    if case["masked"]:
        few = torch.randint(0, V, (max(1, V // 1000),), generator=gen, device=DEVICE)
        off = torch.ones(V, dtype=torch.bool, device=DEVICE)
        off[few] = False
        logits[::case["masked"], off] = -math.inf
    s["targets"][3::5] = -1  # tokens that are not scored
    s["logits"] = logits


def _prepare_adapters(case, gen, s):
    lengths = _lengths(case)
    K, N, R, pool = case["K"], case["N"], case["R"], case["pool"]
    M = sum(lengths)
    s["x"] = _normal(gen, (M, K))
    s["base"] = _normal(gen, (M, N))
    s["A"] = _normal(gen, (pool, R, K), scale=K ** -0.5)
    s["B"] = _normal(gen, (pool, N, R), scale=R ** -0.5)
    s["scale"] = torch.rand(pool, generator=gen, device=DEVICE) + 0.5
    s["seq_start"] = None if case["longest"] == 1 else _i32(list(itertools.accumulate(lengths, initial=0)))
    # (which requests share an adapter, and every ninth has none: the same for each seed)
    s["ids"] = _i32([-1 if i % 9 == 8 else (i * 0x9E3779B1 >> 8) % pool for i in range(case["nseq"])])


def prepare(case, seed):
    s = {"case": case}
    {"norm": _prepare_norm, "rotary": _prepare_rotary, "logprobs": _prepare_logprobs,
     "adapters": _prepare_adapters}[case["kind"]](case, _gen(seed), s)
    return s


# ---------------------------------------------------------------- one pass

def run(s):
    kind = s["case"]["kind"]
    if kind == "norm":
        return _run_norm(s)
    if kind == "rotary":
        return _run_rotary(s)
    if kind == "logprobs":
        return _run_logprobs(s)
    return _run_adapters(s)


def _plain_norm(v, kind, weight, bias):
    if kind == "layer":
        v = v - v.mean(-1, keepdim=True)
    v = v * torch.rsqrt((v * v).mean(-1, keepdim=True) + EPS) * (OFFSET + weight.float())
    return v if bias is None else v + bias.float()


def _run_norm(s):
    case = s["case"]
    if own:
        W = _lib()
        out, h = W.residual_norm(
            s["residual"], s["weight"], s["block"], bias=s["bias"], gate=s["gate"], post_weight=s["post_weight"],
            post_bias=s["post_bias"], kind=W.NORM_LAYER if case["norm"] == "layer" else W.NORM_RMS, eps=EPS,
            weight_offset=OFFSET, residual_scale=case["scale"])
        return {"out": out, "h": h}
    b = s["block"].float()
    if case["post"]:
        b = _plain_norm(b, case["norm"], s["post_weight"], s["post_bias"])
    if s["gate"] is not None:
        b = b * s["gate"].float()
    h = case["scale"] * s["residual"].float() + b
    return {"out": _plain_norm(h, case["norm"], s["weight"], s["bias"]).to(torch.bfloat16), "h": h.to(s["residual"].dtype)}


def _frequencies(case):
    """theta_i in 64 bits, [rot / 2]."""
    i = torch.arange(case["rot"] // 2, dtype=torch.float64, device=DEVICE)
    theta = BASE ** (-2 * i / case["rot"])
    factor, low, high = SCALING[case["scaling"]]
    if case["scaling"] in ("none", "linear"):
        return theta / factor
    if case["scaling"] == "turns":  # in between: linear in the turns
        kept = (TRAINED * theta / (2 * math.pi) - low) / (high - low)
    else:  # linear in i, between the whole i next to those turns
        first, last = (case["rot"] * math.log(TRAINED / (2 * math.pi * turns)) / (2 * math.log(BASE)) for turns in (high, low))
        first, last = max(math.floor(first), 0), min(math.ceil(last), case["rot"] - 1)
        kept = 1 - (i - first) / max(last - first, 0.001)
    kept = kept.clamp(0, 1)
    return theta * kept + theta / factor * (1 - kept)


def _positions(s):
    first = s["first"].long()
    if s["seq_start"] is None:  # the last token of each sequence
        return s["seq_len"][s["slots"].long()].long() - 1 if s["case"]["cached"] else first
    token = torch.arange(s["qkv"].shape[0], device=DEVICE)
    start = s["seq_start"].long()
    seq = torch.searchsorted(start[1:], token, right=True)
    return first[seq] + token - start[seq]


def _run_rotary(s):
    case = s["case"]
    qkv, H, Hkv, rot = s["qkv"], case["H"], case["Hkv"], case["rot"]
    if own:
        if case["cached"]:
            _lib().kv_rotary(s["cache"], qkv, s["slots"], H, s["table"], seq_start=s["seq_start"])
        else:
            _lib().rotary(qkv, s["table"], H, Hkv, seq_start=s["seq_start"], first=s["first"])
        return qkv
    angle = _positions(s).double().unsqueeze(1) * _frequencies(case)
    cos, sin = angle.cos().float().unsqueeze(1), angle.sin().float().unsqueeze(1)
    heads = qkv.view(-1, H + 2 * Hkv, 128)[:, :H + Hkv, :rot]
    if case["layout"] == "half":
        a, b = heads[..., :rot // 2], heads[..., rot // 2:]
    else:
        a, b = heads[..., 0::2], heads[..., 1::2]
    x, y = a.float(), b.float()
    a.copy_(x * cos - y * sin)
    b.copy_(x * sin + y * cos)
    return qkv


def _run_logprobs(s):
    x, t, k = s["logits"], s["targets"], s["case"]["k"]
    if own:
        logp, entropy, index, score = _lib().log_probs(x, t, k)
        return {"logp": logp, "entropy": entropy, "index": index, "score": score}
    z = x.float()
    z = z - z.amax(-1, keepdim=True)
    e = torch.exp(z)
    total = e.sum(-1)
    lse = torch.log(total)
    logp = torch.where(t >= 0, z.gather(1, t.clamp(min=0).long().unsqueeze(1)).squeeze(1) - lse, 0.0)
    entropy = lse - (e * z.clamp(min=-1e4)).sum(-1) / total
    out = {"logp": logp, "entropy": entropy, "index": None, "score": None}
    if k:
        # order by value, then by index: the bits of a number as a whole one, above its place from the end
        bits = x.float().view(torch.int32)
        bits = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
        key = bits * 2 ** 32 + (2 ** 31 - torch.arange(x.shape[1], device=DEVICE))
        index = 2 ** 31 - (key.topk(k, dim=-1).values & 0xFFFFFFFF)
        out["index"] = index.to(torch.int32)
        out["score"] = z.gather(1, index) - lse.unsqueeze(1)
    return out


def _run_adapters(s):
    case = s["case"]
    if own:
        return _lib().add_adapters(s["base"], s["x"], s["A"], s["B"], s["scale"], s["ids"], seq_start=s["seq_start"])
    ids = s["ids"].long()
    x, base = s["x"], s["base"]
    A, B = s["A"][ids.clamp(min=0)].float(), s["B"][ids.clamp(min=0)].float()  # of each sequence
    factor = torch.where(ids >= 0, s["scale"][ids.clamp(min=0)], 0.0)
    n = case["nseq"]
    if s["seq_start"] is None:
        delta = torch.bmm(torch.bmm(x.float().unsqueeze(1), A.transpose(1, 2)), B.transpose(1, 2)).squeeze(1)
        return (base.float() + factor.unsqueeze(1) * delta).to(torch.bfloat16)
    # the sequences side by side, each filled up to the longest
    start = s["seq_start"].long()
    token = torch.arange(x.shape[0], device=DEVICE)
    seq = torch.searchsorted(start[1:], token, right=True)
    at = seq * case["longest"] + token - start[seq]
    row = torch.zeros(n * case["longest"], dtype=torch.long, device=DEVICE)
    row[at] = token
    t = torch.bmm(x[row].view(n, case["longest"], -1).float(), A.transpose(1, 2)) * factor.view(n, 1, 1)
    delta = torch.bmm(t, B.transpose(1, 2)).view(n * case["longest"], -1)
    return (base.float() + delta[at]).to(torch.bfloat16)


# ---------------------------------------------------------------- what a pass needs

def work(case):
    kind = case["kind"]
    if kind == "norm":
        M, D = case["M"], case["D"]
        vectors = 1 + case["post"] + (case["gate"] == 1) + case["bias"] * (1 + case["post"])
        each = 2 * case["bits"] // 8 + 4 + (2 if case["gate"] == -1 else 0)
        return {"bytes": M * D * each + 2 * D * vectors, "flops": 12.0 * M * D}
    if kind == "rotary":
        lengths = _lengths(case)
        rows = case["nseq"] if case["cached"] and case["longest"] > 1 else sum(lengths)
        values = rows * (case["H"] + case["Hkv"]) * case["rot"]
        return {"bytes": 4 * values + 4 * (2 * case["nseq"] + case["rot"]), "flops": 3.0 * values}
    if kind == "logprobs":
        M, V, k = case["M"], case["V"], case["k"]
        return {"bytes": M * V * case["bits"] // 8 + M * (12 + 8 * k), "flops": 6.0 * M * V}
    M, K, N, R = sum(_lengths(case)), case["K"], case["N"], case["R"]
    used = {(i * 0x9E3779B1 >> 8) % case["pool"] for i in range(case["nseq"]) if i % 9 != 8}
    with_one = sum(n for i, n in enumerate(_lengths(case)) if i % 9 != 8)
    return {"bytes": 2 * (with_one * K + 2 * M * N + len(used) * R * (K + N)), "flops": 2.0 * with_one * R * (K + N)}


# ---------------------------------------------------------------- 64-bit results

def _exact_norm(case, s):
    h = torch.empty((case["M"], case["D"]), dtype=torch.float64, device=DEVICE)
    out = torch.empty_like(h)
    norm = (lambda v, w, b: torch.addcmul(torch.zeros_like(v) if b is None else b.double().expand_as(v),
                                          (v - v.mean(1, True)) if case["norm"] == "layer" else v,
                                          (1.0 + w.double()) / ((v.var(1, correction=0, keepdim=True) if case["norm"] == "layer" else
                                                                 v.square().mean(1, True)) + EPS).sqrt()))
    step = max(1, 1 << 25 >> case["D"].bit_length())
    for i in range(0, case["M"], step):
        b = s["block"][i:i + step].double()
        if case["post"]:
            b = norm(b, s["post_weight"], s["post_bias"])
        if case["gate"]:
            b = b * (s["gate"] if case["gate"] == 1 else s["gate"][i:i + step]).double()
        h[i:i + step] = b + s["residual"][i:i + step].double() * case["scale"]
        out[i:i + step] = norm(h[i:i + step], s["weight"], s["bias"])
    return {"out": out, "h": h}


def _exact_frequency(case, i):
    rot, (factor, low, high) = case["rot"], SCALING[case["scaling"]]
    theta = math.exp(-2 * i / rot * math.log(BASE))
    kept = 0.0
    if case["scaling"] == "turns":
        kept = (TRAINED * theta / math.tau - low) / (high - low)
    elif case["scaling"] == "index":
        index = lambda turns: rot / 2 * math.log(TRAINED / (math.tau * turns), BASE)  # noqa: E731
        first, last = max(0, math.floor(index(high))), min(rot - 1, math.ceil(index(low)))
        kept = (last - i) / (last - first) if last > first else float(i <= first)
    kept = min(1.0, max(0.0, kept))
    return theta * (kept + (1 - kept) / factor)


def _exact_rotary(case, s):
    """Each sequence's heads as complex numbers, turned."""
    H, Hkv, rot = case["H"], case["Hkv"], case["rot"]
    theta = torch.tensor([_exact_frequency(case, i) for i in range(rot // 2)], dtype=torch.float64, device=DEVICE)
    lengths, first = _lengths(case), s["first"].tolist()
    step = s["seq_start"] is None
    out = s["qkv"].double()
    row = 0
    for n, f in zip(lengths, first):
        rows = 1 if step else n
        at = f + n - 1 if step and case["cached"] else f
        x = out[row:row + rows].view(rows, H + 2 * Hkv, 128)[:, :H + Hkv, :rot]
        turn = torch.polar(torch.ones(1, dtype=torch.float64, device=DEVICE),
                           torch.outer(torch.arange(at, at + rows, dtype=torch.float64, device=DEVICE), theta)).unsqueeze(1)
        if case["layout"] == "half":
            z = torch.complex(*x.split(rot // 2, dim=-1)) * turn
            x.copy_(torch.cat([z.real, z.imag], dim=-1))
        else:
            z = torch.view_as_complex(x.reshape(rows, H + Hkv, rot // 2, 2)) * turn
            x.copy_(torch.view_as_real(z).flatten(-2))
        row += rows
    return out


def _exact_logprobs(case, s):
    M, k = case["M"], case["k"]
    logp, entropy = (torch.zeros(M, dtype=torch.float64, device=DEVICE) for _ in range(2))
    score = torch.empty((M, k), dtype=torch.float64, device=DEVICE) if k else None
    step = max(1, 1 << 25 >> case["V"].bit_length())
    for i in range(0, M, step):
        lp = torch.log_softmax(s["logits"][i:i + step].double(), dim=1)
        entropy[i:i + step] = torch.special.entr(lp.exp()).sum(1)
        t = s["targets"][i:i + step].long()
        scored = t >= 0
        logp[i:i + step][scored] = lp[scored, t[scored]]
        if k:
            score[i:i + step] = lp.sort(dim=1, descending=True).values[:, :k]
    return {"logp": logp, "entropy": entropy, "index": None, "score": score}


def _exact_adapters(case, s):
    out = s["base"].double()
    row = 0
    for n, a in zip(_lengths(case), s["ids"].tolist()):
        if a >= 0:
            t = s["x"][row:row + n].double() @ s["A"][a].double().t()
            out[row:row + n] += float(s["scale"][a]) * (t @ s["B"][a].double().t())
        row += n
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "rotary": _exact_rotary, "logprobs": _exact_logprobs,
            "adapters": _exact_adapters}[case["kind"]](case, s)
