"""The paged key-value cache's operators as a screening service calls them, case by case.

The service prefills a protein's tokens once, shares their pages among the ligands that
it is screened against, and feeds each ligand's tokens one step at a time.  The kinds:

  decode   attention of one new token per sequence over the cache, the token's own key
           and value stored (w4a16.attention_decode);
  write    keys and values of a packed prompt into its pages (w4a16.kv_write);
  fork     a prefix shared by many sequences, each grown by its own tokens (which copies the
           half-full page they share) and freed again (kv_fork, kv_extend, kv_trim);
  step     every sequence of a batch grown by one token and rolled back (kv_extend, kv_trim);
  compact  the pages in use moved to the front of the pool (kv_compact).

A cache is pages [layers, 2, num_pages, kv_heads, page_tokens, 128] in bf16, or in e4m3
with a power-of-two exponent for each token's key and value ([layers, num_pages, kv_heads,
page_tokens, 2] bytes, biased by 127), a page table [slots, max_pages], lengths [slots] and
reference counts [num_pages], where 0 marks a free page.
"""
from __future__ import annotations

import itertools
import math

import torch

own = False

DEVICE = "cuda"
D = 128
E4M3 = torch.float8_e4m3fn
MIN_EXP = -120       # smallest exponent of an e4m3 row
LARGEST = 2.0e9      # bytes of a drawn case's cache, every sequence at its longest


def _decode(name, bits, H, Hkv, T, nseq, shortest, longest, window=32768):
    return {"name": name, "kind": "decode", "bits": bits, "H": H, "Hkv": Hkv, "T": T, "nseq": nseq,
            "shortest": shortest, "longest": longest, "window": window}


def _write(name, bits, H, Hkv, T, nseq, shortest, longest):
    return {"name": name, "kind": "write", "bits": bits, "H": H, "Hkv": Hkv, "T": T, "nseq": nseq,
            "shortest": shortest, "longest": longest}


def _fork(name, bits, layers, Hkv, T, prefix, children, grow):
    return {"name": name, "kind": "fork", "bits": bits, "layers": layers, "Hkv": Hkv, "T": T,
            "prefix": prefix, "children": children, "grow": grow}


def listed():
    return [
        # a single pair's next token on the 96-head decoder: all latency
        _decode("decode_1_short", 16, 96, 96, 16, 1, 333, 333),
        # one step of a scored batch of 64 pairs of ragged lengths
        _decode("decode_64_pairs", 16, 96, 96, 64, 64, 200, 1024),
        # one long context under the sliding window
        _decode("decode_long_window", 16, 96, 96, 64, 1, 10007, 10007, 4096),
        # shared heads (12 queries to a key), small pages, lengths from one token on
        _decode("decode_gqa_ragged", 16, 96, 8, 16, 37, 1, 8192),
        # the 64 pairs on an 8-bit cache
        _decode("decode_e4m3_64_pairs", 8, 96, 96, 64, 64, 200, 1024),
        # three very long contexts on an 8-bit cache of shared heads: few rows, the
        # length split over the whole GPU
        _decode("decode_e4m3_long", 8, 64, 8, 32, 3, 60000, 131072),
        # prefill of the 64 pairs: their keys and values into the pages
        _write("write_64_pairs", 16, 96, 96, 64, 64, 200, 1024),
        # short ragged prompts of a decoder with shared heads, stored in 8 bits
        _write("write_e4m3_ragged", 8, 96, 8, 16, 37, 1, 700),
        # a protein's 1000 tokens shared by 64 ligands of 60 tokens (a few of the layers)
        _fork("fork_64_ligands", 16, 4, 96, 16, 1000, 64, 60),
        # the same with large pages of an 8-bit cache of shared heads, every layer
        _fork("fork_e4m3", 8, 96, 8, 128, 500, 48, 33),
        # the page work of one decode step of 512 sequences
        {"name": "step_512", "kind": "step", "T": 16, "nseq": 512, "shortest": 100, "longest": 1700,
         "spare": 20000},
        # a pool half in use after many sequences have left it
        {"name": "compact_half", "kind": "compact", "bits": 16, "layers": 4, "Hkv": 8, "T": 64,
         "pages": 2000, "live": 1001, "moves": 480, "nseq": 40},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = [(96, 96), (32, 32), (16, 16), (96, 8), (64, 8), (32, 4), (24, 1), (8, 2)]


def draw(rng):
    kind = rng.choice(["decode"] * 6 + ["write"] * 2 + ["fork", "step", "compact"])
    bits = rng.choice([16, 16, 8])
    T = rng.choice([16, 32, 64, 128])
    H, Hkv = rng.choice(HEADS)
    row = Hkv * 2 * D * bits // 8  # bytes of a token
    if kind in ("decode", "write"):
        nseq = _log_int(rng, 1, 256)
        most = max(2, min(131072 if kind == "decode" else 8192, int(LARGEST / row / nseq)))
        if kind == "write":  # (a row of the fused projection has the queries too)
            most = max(2, min(most, int(3 * LARGEST / ((H + 2 * Hkv) * D * 2) / nseq)))
        longest = _log_int(rng, 1, most)
        shortest = rng.choice([longest, rng.randint(1, longest), 1])
        if kind == "write":
            return {"kind": kind, "bits": bits, "H": H, "Hkv": Hkv, "T": T, "nseq": nseq,
                    "shortest": shortest, "longest": longest}
        return {"kind": kind, "bits": bits, "H": H, "Hkv": Hkv, "T": T, "nseq": nseq,
                "shortest": shortest, "longest": longest,
                "window": rng.choice([32768, 32768, 4096, _log_int(rng, 1, 2 * longest)])}
    if kind == "fork":
        children = _log_int(rng, 1, 128)
        layers = max(1, min(_log_int(rng, 1, 96), int(LARGEST / (row * (T + 100) * (children + 4)))))
        return {"kind": kind, "bits": bits, "layers": layers, "Hkv": Hkv, "T": T,
                "prefix": rng.randint(1, 1000 if layers * row * 1000 < LARGEST else 2 * T),
                "children": children, "grow": rng.randint(1, 100)}
    if kind == "step":
        longest = _log_int(rng, 16, 4000)
        return {"kind": kind, "T": T, "nseq": _log_int(rng, 1, 600), "shortest": rng.randint(1, longest),
                "longest": longest, "spare": _log_int(rng, 700, 30000)}
    layers = _log_int(rng, 1, 32)
    pages = max(20, min(_log_int(rng, 20, 8000), int(LARGEST / (layers * row * T))))
    live = rng.randint(2, pages - 2)
    return {"kind": kind, "bits": bits, "layers": layers, "Hkv": Hkv, "T": T, "pages": pages, "live": live,
            "moves": rng.randint(0, min(live, pages - live)), "nseq": min(live, _log_int(rng, 1, 100))}


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


def _pool(gen, bits, layers, pages, Hkv, T):
    """A cache in use: keys and values of unit scale, in e4m3 each row with an exponent of
    its own (rows' largest values between 224 and 448 codes, scales over a few octaves)."""
    shape = (layers, 2, pages, Hkv, T, D)
    if bits == 16:
        pool = torch.empty(shape, dtype=torch.bfloat16, device=DEVICE)
        for layer in pool.view(layers * 2, pages, Hkv, T, D):
            layer.normal_(generator=gen)
        return pool, None
    pool = torch.empty(shape, dtype=E4M3, device=DEVICE)
    flat = pool.view(-1)
    step = 1 << 28
    for i in range(0, flat.numel(), step):
        part = flat[i:i + step]
        part.copy_(torch.randn(part.shape, generator=gen, device=DEVICE).mul_(112).clamp_(-448, 448))
    exponents = torch.randint(118, 123, (layers, pages, Hkv, T, 2), generator=gen, device=DEVICE,
                              dtype=torch.uint8)
    return pool, exponents


def _tables(gen, counts, num_pages, slots, num_slots, max_pages):
    """A page table whose sequences (of `counts` pages) have their pages all over the pool."""
    table = torch.zeros((num_slots, max_pages), dtype=torch.int32, device=DEVICE)
    pages = torch.randperm(num_pages, generator=gen, device=DEVICE).to(torch.int32)
    starts = list(itertools.accumulate(counts, initial=0))
    for slot, n, a in zip(slots, counts, starts):
        table[slot, :n] = pages[a:a + n]
    refs = torch.zeros(num_pages, dtype=torch.int32, device=DEVICE)
    refs[pages[:starts[-1]].long()] = 1
    return table, refs, pages[:starts[-1]]


def _sequences(case, gen, s, lengths, spare, layers=1, bits=16, Hkv=1):
    T = case["T"]
    nseq = len(lengths)
    counts = [-(-n // T) for n in lengths]
    num_slots = nseq + 3
    slots = torch.randperm(num_slots, generator=gen, device=DEVICE)[:nseq].tolist()
    pages = sum(counts) + spare
    s["max_pages"] = max(counts) + 1
    s["page_table"], s["page_refs"], _ = _tables(gen, counts, pages, slots, num_slots, s["max_pages"])
    s["seq_len"] = torch.zeros(num_slots, dtype=torch.int32, device=DEVICE)
    s["seq_len"][torch.tensor(slots, device=DEVICE)] = _i32(lengths)
    s["slots"] = _i32(slots)
    s["pages"], s["exponents"] = _pool(gen, bits, layers, pages, Hkv, T)


def _prepare_fork(case, gen, s):
    """One sequence with the prefix, and another whose pages lie all over the pool, so that
    the free ones do too."""
    T, c = case["T"], case["children"]
    n = -(-case["prefix"] // T)
    after = -(-(case["prefix"] + case["grow"]) // T)
    busy = max(1, (n + c) // 4)
    pages = n + busy + c * (after - n + 1) + 3
    s["max_pages"] = max(after, busy) + 1
    s["page_table"], s["page_refs"], _ = _tables(gen, [n, busy], pages, [0, 1], c + 2, s["max_pages"])
    s["seq_len"] = _i32([case["prefix"], busy * T] + [0] * c)
    s["parents"] = torch.zeros(c, dtype=torch.int32, device=DEVICE)
    s["children"] = _i32([2 + i for i in range(c)])
    s["grow"] = torch.full((c,), case["grow"], dtype=torch.int32, device=DEVICE)
    s["pages"], s["exponents"] = _pool(gen, case["bits"], case["layers"], pages, case["Hkv"], T)


def _prepare_compact(case, gen, s):
    """`live` pages, `moves` of them beyond the first `live` pages; the sequences share them
    out, and the second half of them share the first one's first page."""
    T, live, nseq = case["T"], case["live"], case["nseq"]
    low = torch.randperm(live, generator=gen, device=DEVICE)[:live - case["moves"]]
    high = live + torch.randperm(case["pages"] - live, generator=gen, device=DEVICE)[:case["moves"]]
    used = torch.cat([low, high])
    used = used[torch.randperm(live, generator=gen, device=DEVICE)].to(torch.int32)
    counts = [live // nseq + (i < live % nseq) for i in range(nseq)]
    table = torch.zeros((nseq, max(counts) + 2), dtype=torch.int32, device=DEVICE)
    a = 0
    lengths = []
    for i, n in enumerate(counts):
        shared = int(i >= nseq // 2 and i > 0)
        table[i, shared:shared + n] = used[a:a + n]
        if shared:
            table[i, 0] = used[0]
        lengths.append((n + shared) * T - (7 * i) % T)
        a += n
    refs = torch.zeros(case["pages"], dtype=torch.int32, device=DEVICE)
    refs[used.long()] = 1
    refs[used[0].long()] += sum(1 for i in range(nseq) if i >= nseq // 2 and i > 0)
    s["page_table"], s["page_refs"], s["seq_len"] = table, refs, _i32(lengths)
    s["max_pages"] = table.shape[1]
    s["pages"], s["exponents"] = _pool(gen, case["bits"], case["layers"], case["pages"], case["Hkv"], T)
    # the scheduler's record of the tables, from which every pass starts
    s["was"] = (table.clone(), refs.clone())


def prepare(case, seed):
    gen = _gen(seed)
    kind = case["kind"]
    s = {"case": case}
    if kind in ("decode", "write"):
        lengths = _lengths(case)
        _sequences(case, gen, s, lengths, 8, bits=case["bits"], Hkv=case["Hkv"])
        rows = case["nseq"] if kind == "decode" else sum(lengths)
        width = (case["H"] + 2 * case["Hkv"]) * D
        qkv = torch.empty((rows, width), dtype=torch.bfloat16, device=DEVICE).normal_(generator=gen)
        if kind == "decode":
            qkv[:, :case["H"] * D] *= 2  # scores that differ by a few units, as trained heads have them
        else:
            s["seq_start"] = _i32(list(itertools.accumulate(lengths, initial=0)))
        s["qkv"] = qkv
    elif kind == "fork":
        _prepare_fork(case, gen, s)
    elif kind == "step":
        lengths = _lengths(case)
        _sequences(case, gen, s, lengths, case["spare"])
        s["one"] = torch.ones(case["nseq"], dtype=torch.int32, device=DEVICE)
        s["keep"] = _i32(lengths)
    else:
        _prepare_compact(case, gen, s)
    if own:
        from paper_2608_30877_gb300 import w4a16 as W
        s["W"] = W
        s["cache"] = W.KVCache.from_tensors(s["pages"], s["page_table"], s["seq_len"], s["page_refs"],
                                            s["exponents"])
    return s


# ---------------------------------------------------------------- one pass

def run(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "decode":
        if own:
            out = s["W"].attention_decode(s["cache"], 0, s["qkv"], s["slots"], case["H"],
                                          window=case["window"])
        else:
            out = _plain_decode(s)
        return {"out": out, "pages": s["pages"], "exponents": s["exponents"]}
    if kind == "write":
        if own:
            s["W"].kv_write(s["cache"], 0, s["qkv"], s["seq_start"], s["slots"], case["H"])
        else:
            _plain_write(s)
        return {"pages": s["pages"], "exponents": s["exponents"]}
    if kind == "fork":
        if own:
            s["W"].kv_fork(s["cache"], s["parents"], s["children"])
            s["W"].kv_extend(s["cache"], s["children"], s["grow"])
            grown = (s["page_table"].clone(), s["page_refs"].clone())
            s["W"].kv_trim(s["cache"], s["children"])
        else:
            _plain_fork(s)
            _plain_extend(s, s["children"].long(), s["grow"].long())
            grown = (s["page_table"].clone(), s["page_refs"].clone())
            _plain_trim(s, s["children"].long(), torch.zeros_like(s["grow"]).long())
        return {"grown": grown, "pages": s["pages"], "exponents": s["exponents"],
                "page_table": s["page_table"], "page_refs": s["page_refs"], "seq_len": s["seq_len"]}
    if kind == "step":
        if own:
            s["W"].kv_extend(s["cache"], s["slots"], s["one"])
            grown = (s["page_table"].clone(), s["page_refs"].clone())
            s["W"].kv_trim(s["cache"], s["slots"], s["keep"])
        else:
            _plain_extend(s, s["slots"].long(), s["one"].long())
            grown = (s["page_table"].clone(), s["page_refs"].clone())
            _plain_trim(s, s["slots"].long(), s["keep"].long())
        return {"grown": grown, "page_table": s["page_table"], "page_refs": s["page_refs"],
                "seq_len": s["seq_len"]}
    s["page_table"].copy_(s["was"][0])
    s["page_refs"].copy_(s["was"][1])
    if own:
        s["W"].kv_compact(s["cache"])
    else:
        _plain_compact(s)
    return {"pages": s["pages"], "exponents": s["exponents"], "page_table": s["page_table"],
            "page_refs": s["page_refs"]}


# ---------------------------------------------------------------- the plain form

def _power(e):
    """2^e for whole e within fp32's normal range, from its bits."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _encode(x):
    """Rows of fp32 as e4m3 codes and exponents: the smallest that keeps the largest finite
    value within 448."""
    finite = torch.where(torch.isfinite(x), x.abs(), 0.0).amax(-1)
    m, e = torch.frexp(finite)  # finite = m 2^e, and 448 = 0.875 2^9
    e = torch.where(finite > 0, e - 9 + (m > 0.875), MIN_EXP).clamp(min=MIN_EXP)
    codes = (x * _power(-e).unsqueeze(-1)).clamp(-448, 448).to(E4M3)
    return codes, (e + 127).to(torch.uint8)


def _store(s, page, at, k, v):
    """Rows k, v [n, Hkv, D] into token `at` of pages `page`."""
    if s["exponents"] is None:
        s["pages"][0, 0][page, :, at] = k
        s["pages"][0, 1][page, :, at] = v
        return
    bytes_ = s["pages"].view(torch.uint8)
    (kc, ke), (vc, ve) = _encode(k.float()), _encode(v.float())
    bytes_[0, 0][page, :, at] = kc.view(torch.uint8)
    bytes_[0, 1][page, :, at] = vc.view(torch.uint8)
    s["exponents"][0][page, :, at] = torch.stack([ke, ve], dim=-1)


def _load(s, which, table):
    """Keys or values of whole page lists, fp32 [n, W, Hkv, T, D]."""
    if s["exponents"] is None:
        return s["pages"][0, which][table].float()
    codes = s["pages"].view(torch.uint8)[0, which][table].view(E4M3).float()
    return codes * _power(s["exponents"][0][table][..., which].int() - 127).unsqueeze(-1)


def _plain_decode(s):
    case = s["case"]
    n, H, Hkv, T, W = case["nseq"], case["H"], case["Hkv"], case["T"], s["max_pages"]
    slots = s["slots"].long()
    length = s["seq_len"][slots].long()
    table = s["page_table"][slots].long()
    q, k, v = s["qkv"].split([H * D, Hkv * D, Hkv * D], dim=1)
    last = length - 1
    page = table.gather(1, (last // T).unsqueeze(1)).squeeze(1)
    _store(s, page, last % T, k.reshape(n, Hkv, D), v.reshape(n, Hkv, D))
    pos = torch.arange(W * T, device=DEVICE)
    seen = (pos < length.unsqueeze(1)) & (pos >= (length - case["window"]).unsqueeze(1))
    keys = _load(s, 0, table).transpose(1, 2).reshape(n, Hkv, W * T, D)
    scores = (q.float().view(n, Hkv, H // Hkv, D) @ keys.transpose(2, 3)) / math.sqrt(D)
    scores = scores.masked_fill(~seen[:, None, None], -math.inf)
    p = torch.exp(scores - scores.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    values = _load(s, 1, table).transpose(1, 2).reshape(n, Hkv, W * T, D)
    values = values.masked_fill(~seen[:, None, :, None], 0.0)
    return (p @ values).reshape(n, H * D).to(torch.bfloat16)


def _plain_write(s):
    case = s["case"]
    H, Hkv, T = case["H"], case["Hkv"], case["T"]
    M = s["qkv"].shape[0]
    token = torch.arange(M, device=DEVICE)
    start = s["seq_start"].long()
    seq = torch.searchsorted(start[1:], token, right=True)
    slot = s["slots"].long()[seq]
    pos = s["seq_len"].long()[slot] - start[seq + 1] + token
    page = s["page_table"][slot, pos // T].long()
    _, k, v = s["qkv"].split([H * D, Hkv * D, Hkv * D], dim=1)
    _store(s, page, pos % T, k.reshape(M, Hkv, D), v.reshape(M, Hkv, D))


def _in_use(s, length):
    """Which entries of a page list of this length are its pages."""
    T = s["case"]["T"]
    return torch.arange(s["max_pages"], device=DEVICE) < ((length + T - 1) // T).unsqueeze(1)


def _count(s, table, which):
    """How often each page occurs among the entries `which` of page lists."""
    P = s["page_refs"].shape[0]
    at = torch.where(which, table, P).reshape(-1)
    count = torch.zeros(P + 1, dtype=torch.int32, device=DEVICE)
    return count.index_add_(0, at, torch.ones_like(at, dtype=torch.int32))[:P]


def _plain_fork(s):
    parents, children = s["parents"].long(), s["children"].long()
    table = s["page_table"].long()
    length = s["seq_len"][parents]
    mine = _in_use(s, length)
    s["page_table"][children] = torch.where(mine, table[parents], table[children]).to(torch.int32)
    s["page_refs"] += _count(s, table[parents], mine)
    s["seq_len"][children] = length


def _plain_extend(s, slots, add):
    T, W = s["case"]["T"], s["max_pages"]
    P = s["page_refs"].shape[0]
    table = s["page_table"][slots].long()
    old = s["seq_len"][slots].long()
    new = old + add
    had, has = (old + T - 1) // T, (new + T - 1) // T
    last = table.gather(1, (had - 1).clamp(min=0).unsqueeze(1)).squeeze(1)
    copies = (add > 0) & (old % T != 0) & (s["page_refs"][last] > 1)
    need = has - had + copies
    first = need.cumsum(0) - need
    free = torch.argsort((s["page_refs"] > 0).to(torch.int32), stable=True)
    entry = torch.arange(W, device=DEVICE)
    begin = had - copies.long()  # the first entry that changes
    rank = first.unsqueeze(1) + entry - begin.unsqueeze(1)
    fresh = (entry >= begin.unsqueeze(1)) & (entry < has.unsqueeze(1))
    table = torch.where(fresh, free[rank.clamp(0, P - 1)], table)
    s["page_refs"] += _count(s, table, fresh)
    s["page_refs"] -= _count(s, last.unsqueeze(1), copies.unsqueeze(1))
    s["page_table"][slots] = table.to(torch.int32)
    s["seq_len"][slots] = new.to(torch.int32)
    # a copy's tokens; where nothing is copied a page takes its own
    own_page = table.gather(1, (had - 1).clamp(min=0).unsqueeze(1)).squeeze(1)
    token = torch.arange(T, device=DEVICE) < (old % T).unsqueeze(1)
    moves = (copies.unsqueeze(1) & token)[None, None, :, None, :, None]
    pool = s["pages"].view(torch.uint8) if s["exponents"] is not None else s["pages"]
    pool[:, :, own_page] = torch.where(moves, pool[:, :, last], pool[:, :, own_page])
    if s["exponents"] is not None:
        e = s["exponents"]
        e[:, own_page] = torch.where(moves[0], e[:, last], e[:, own_page])


def _plain_trim(s, slots, keep):
    table = s["page_table"][slots].long()
    gone = _in_use(s, s["seq_len"][slots].long()) & ~_in_use(s, keep)
    s["page_refs"] -= _count(s, table, gone)
    s["seq_len"][slots] = keep.to(torch.int32)


def _plain_compact(s):
    refs = s["page_refs"]
    P = refs.shape[0]
    index = torch.arange(P, device=DEVICE)
    live = refs > 0
    n = live.sum()
    movers, holes = live & (index >= n), ~live & (index < n)
    moved = index < movers.sum()
    from_ = torch.argsort((~movers).to(torch.int32), stable=True)
    to = torch.where(moved, torch.argsort((~holes).to(torch.int32), stable=True), from_)
    place = index.clone().scatter_(0, from_, to)  # where each page goes
    # what each page takes (the last entry stands for no page)
    source = torch.arange(P + 1, device=DEVICE).scatter_(0, torch.where(moved, to, P), from_)[:P]
    table = s["page_table"].long()
    s["page_table"].copy_(torch.where(_in_use(s, s["seq_len"].long()), place[table], table))
    refs.copy_(torch.zeros_like(refs).index_add_(0, place, refs.clone()))
    if s["exponents"] is None:
        s["pages"].copy_(s["pages"][:, :, source])
    else:
        pool = s["pages"].view(torch.uint8)
        pool.copy_(pool[:, :, source])
        s["exponents"].copy_(s["exponents"][:, source])


# ---------------------------------------------------------------- what a pass needs

def work(case):
    kind = case["kind"]
    if kind == "step":
        lengths = _lengths(case)
        pages = sum(-(-n // case["T"]) for n in lengths) + case["spare"]
        # the counts read to find free pages; lengths read and written, table entries and
        # counts of the pages that come and go
        return {"bytes": 4 * pages + case["nseq"] * 4 * 8, "flops": 0}
    token = 2 * D * case["bits"] // 8 + (2 if case["bits"] == 8 else 0)  # a head's key and value
    if kind in ("decode", "write"):
        lengths = _lengths(case)
        n, Hkv, T = case["nseq"], case["Hkv"], case["T"]
        if kind == "write":
            m = sum(lengths)
            return {"bytes": m * Hkv * (2 * D * 2 + token) + 4 * (sum(-(-i // T) for i in lengths) + 3 * n),
                    "flops": 0}
        seen = [min(i, case["window"]) for i in lengths]
        pages = sum(-(-i // T) for i in seen)
        # (the new token comes from the projection's row and goes to the cache)
        return {"bytes": sum(seen) * Hkv * token + n * (2 * case["H"] + 2 * Hkv) * D * 2 + 4 * (pages + 2 * n),
                "flops": 4.0 * D * case["H"] * sum(seen)}
    if kind == "fork":
        T, c = case["T"], case["children"]
        n, after = -(-case["prefix"] // T), -(-(case["prefix"] + case["grow"]) // T)
        copied = c * (case["prefix"] % T) * case["layers"] * case["Hkv"] * token
        return {"bytes": 2 * copied + 4 * (n + c * (after + 4) + after * c), "flops": 0}
    page = case["layers"] * case["Hkv"] * case["T"] * token
    return {"bytes": 2 * case["moves"] * page + 4 * (2 * case["pages"] + 3 * case["live"]), "flops": 0}


# ---------------------------------------------------------------- 64-bit results

def _exact_row(x):
    """One row as an 8-bit cache holds it: values of e4m3 (3 bits after the first, exponents
    from -6, 448 the largest) times the smallest power of two that reaches the row's largest."""
    top = x.abs().max().item()
    e = MIN_EXP
    while e < 127 and top > 448 * 2.0 ** e:
        e += 1
    y = x / 2.0 ** e
    unit = 2.0 ** (torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -60))).clamp(min=-6.0) - 3)
    return torch.round(y / unit) * unit, e


def _exact_rows(k):
    return torch.stack([c * 2.0 ** e for c, e in map(_exact_row, k)])


def _exact_decode(case, s):
    H, Hkv, T = case["H"], case["Hkv"], case["T"]
    out = torch.zeros((case["nseq"], H, D), dtype=torch.float64, device=DEVICE)
    for i, (slot, n) in enumerate(zip(s["slots"].tolist(), _lengths(case))):
        low = max(0, n - case["window"])
        pos = torch.arange(low, n, device=DEVICE)
        page, at = s["page_table"][slot].long()[pos // T], pos % T
        row = s["qkv"][i].double()
        q = row[:H * D].view(Hkv, H // Hkv, D)
        new = row[H * D:].view(2, Hkv, D)
        held = []
        for which in (0, 1):
            if case["bits"] == 16:
                x = s["pages"][0, which][page, :, at].double()
                x[-1] = new[which]
            else:
                e = s["exponents"][0][page, :, at][..., which].double() - 127
                x = s["pages"].view(torch.uint8)[0, which][page, :, at].view(E4M3).double()
                x = x * torch.pow(2.0, e).unsqueeze(-1)
                x[-1] = _exact_rows(new[which])
            held.append(x)
        for h in range(Hkv):
            w = torch.softmax(q[h] @ held[0][:, h].t() / math.sqrt(D), dim=-1)
            out[i, h * (H // Hkv):(h + 1) * (H // Hkv)] = w @ held[1][:, h]
    return out.view(case["nseq"], H * D)


def exact(case, seed):
    """Attention in 64 bits; everything else is copied, counted or rounded to 8 bits."""
    if case["kind"] != "decode":
        return None
    return {"out": _exact_decode(case, prepare(case, seed)), "pages": None, "exponents": None}
