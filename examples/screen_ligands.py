"""Screens one protein against many ligands with a shared key-value cache.

A protein's tokens are the same in every pair that it is scored in, and most of the
pair's length.  Here they are prefilled once (w4a16.attention_prefill, kv_write); every
ligand's sequence starts as a fork of the protein's (kv_fork), which shares its pages, and
the ligands' tokens then go through the decoder together, one step per token: growth
(kv_extend, which copies the protein's half-filled last page for each ligand), the int4 linears, and
attention over the cache (attention_decode).  The step is captured once as a CUDA graph and
replayed; ligands that have ended are padding.  The affinity head reads each ligand's last
state, and topk_smallest sorts the predictions.  Freed pages are compacted at the end.

    python examples/screen_ligands.py [--ligands 64] [--protein 700] [--e4m3]

Weights and token states are random: the model's are not available.
"""
from __future__ import annotations

import argparse
import dataclasses
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2608_30877_gb300 import synthetic as S  # noqa: E402
from paper_2608_30877_gb300 import w4a16 as W  # noqa: E402

HEAD_DIM = 128


@dataclasses.dataclass
class Decoder:
    """int4 decoder layers (QKV, attention, output, SwiGLU MLP; no norms, as the library
    has none: the outputs that are added to the stream are scaled down instead)."""
    heads: int
    layers: list
    head: tuple  # affinity head: packed, scales, bias

    @property
    def width(self):
        return self.heads * HEAD_DIM

    @classmethod
    def random(cls, heads: int, n_layers: int, seed: int = 0):
        d = heads * HEAD_DIM

        def weights(n, k, seed, scale=1.0):
            return W.quantize(S.make_w_master(n, k, seed, "cuda").mul_(scale / (0.02 * k ** 0.5)))

        layers = [(weights(3 * d, d, seed + 10 * i), weights(d, d, seed + 10 * i + 1, 0.5),
                   weights(8 * d, d, seed + 10 * i + 2), weights(d, 4 * d, seed + 10 * i + 3, 0.5))
                  for i in range(n_layers)]
        return cls(heads, layers, (*weights(1, d, seed + 7), torch.zeros(1, dtype=torch.bfloat16, device="cuda")))

    def forward(self, x, attend):
        """x [tokens, width]; attend(layer, qkv) -> [tokens, width]."""
        for i, (qkv, o, up, down) in enumerate(self.layers):
            a = attend(i, W.linear(x, *qkv))
            x = W.linear_fused(a, *o, residual=x)
            x = W.linear_fused(W.linear_fused(x, *up, act=W.ACT_SWIGLU), *down, residual=x)
        return x

    def affinities(self, states):
        return W.linear_fused(states, self.head[0], self.head[1], bias=self.head[2])[:, 0].contiguous()


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def screen(model: Decoder, protein: torch.Tensor, ligands: list[torch.Tensor], page_tokens: int = 16,
           dtype=torch.bfloat16):
    """Affinities [len(ligands)] of the protein (token states [tokens, width]) with each
    ligand ([tokens, width]), and the cache that was used."""
    n, H = len(ligands), model.heads
    lengths = [x.shape[0] for x in ligands]
    steps = max(lengths)
    pages = -(-protein.shape[0] // page_tokens)
    after = -(-(protein.shape[0] + steps) // page_tokens)
    cache = W.KVCache(len(model.layers), pages + n * (after - pages + 1), H, n + 1, after, page_tokens, dtype)

    # the protein, in slot 0
    start, slot0 = _i32([0, protein.shape[0]]), _i32([0])
    W.kv_extend(cache, slot0, _i32([protein.shape[0]]))

    def prefill(layer, qkv):
        W.kv_write(cache, layer, qkv, start, slot0, H)
        return W.attention_prefill(qkv, start, H)

    model.forward(protein, prefill)

    # every ligand goes on from it
    slots = _i32(range(1, n + 1))
    W.kv_fork(cache, torch.zeros_like(slots), slots)

    # one step: a token of each ligand that has one left (a slot of -1 otherwise)
    token = torch.empty((n, model.width), dtype=torch.bfloat16, device="cuda")
    active, one = slots.clone(), torch.ones_like(slots)
    workspace = cache.new_workspace(H)

    def step():
        W.kv_extend(cache, active, one)
        return model.forward(token, lambda layer, qkv: W.attention_decode(cache, layer, qkv, active, H,
                                                                          workspace=workspace))

    inputs = torch.zeros((steps, n, model.width), dtype=torch.bfloat16, device="cuda")
    left = torch.full((steps, n), -1, dtype=torch.int32)
    for i, x in enumerate(ligands):
        inputs[:x.shape[0], i] = x
        left[:x.shape[0], i] = i + 1
    left = left.cuda()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    last = torch.empty_like(token)
    ends = _i32(lengths) - 1
    for t in range(steps):
        token.copy_(inputs[t])
        active.copy_(left[t])
        graph.replay()
        last = torch.where((ends == t).unsqueeze(1), out, last)
    affinities = model.affinities(last)

    # the ligands leave; the protein stays for the next ones
    W.kv_trim(cache, slots)
    W.kv_compact(cache)
    return affinities, cache


def screen_without_cache(model: Decoder, protein: torch.Tensor, ligands: list[torch.Tensor]):
    """The same by prefilling every pair."""
    pairs = [torch.cat([protein, x]) for x in ligands]
    ends = torch.tensor([p.shape[0] for p in pairs]).cumsum(0)
    start = _i32([0, *ends.tolist()])
    states = model.forward(torch.cat(pairs), lambda layer, qkv: W.attention_prefill(qkv, start, model.heads))
    return model.affinities(W.gather_rows(states, (start[1:] - 1).contiguous()))


def random_states(tokens: int, width: int, seed: int):
    return S.make_x(tokens, width, seed, "cuda")


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--ligands", type=int, default=64)
    ap.add_argument("--protein", type=int, default=700)
    ap.add_argument("--heads", type=int, default=16)
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--best", type=int, default=5)
    ap.add_argument("--e4m3", action="store_true", help="an 8-bit cache")
    a = ap.parse_args()
    model = Decoder.random(a.heads, a.layers)
    protein = random_states(a.protein, model.width, 1)
    ligands = [random_states(20 + 7 * i % 41, model.width, 100 + i) for i in range(a.ligands)]
    dtype = torch.float8_e4m3fn if a.e4m3 else torch.bfloat16
    times = {}
    for name, run in (("shared cache", lambda: screen(model, protein, ligands, dtype=dtype)[0]),
                      ("every pair prefilled", lambda: screen_without_cache(model, protein, ligands))):
        result = run()  # (the first call loads the kernels)
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        begin.record()
        result = run()
        end.record()
        torch.cuda.synchronize()
        times[name] = begin.elapsed_time(end)
        index, score = W.topk_smallest(result.float(), min(a.best, a.ligands))
        print(f"{name}: {times[name]:.1f} ms, best {[(i, round(s, 3)) for i, s in zip(index.tolist(), score.tolist())]}")
    if W.get_device_error() != W.OK:
        raise SystemExit("device status word set")


if __name__ == "__main__":
    main()
