"""The operators around the linears as a decoder runs them: norms, int4 linears with adapters, rotary positions,
the cache and its attention, then a head's log probabilities.  Every call of a run is held to the bounds
of its own tests, from what it was given; a captured step gives the bits of the launched one; and the
example's two ways to an affinity agree."""
import os
import sys

import numpy as np
import pytest
import torch

from tests import kv_reference as KV
from tests import layer_reference as R
from tests import test_gpu_log_probs as LP
from tests import test_gpu_residual_norm as RN
from tests import test_gpu_rotary as RO

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

f64 = RN.f64


class Checked:
    """w4a16 whose operators around the linears are checked on every call."""

    def __init__(self, W, positions):
        self._W, self._positions, self.calls = W, positions, {}

    def __getattr__(self, name):
        return getattr(self._W, name)

    def _count(self, name):
        self.calls[name] = self.calls.get(name, 0) + 1

    def residual_norm(self, residual, weight, block):
        self._count("norm")
        given = dict(residual=residual, block=block, weight=weight, bias=None, gate=None, post_weight=None, post_bias=None)
        refs, errs = RN.reference(**given, layer=False, eps=1e-5, offset=0.0, scale=1.0)
        got = self._W.residual_norm(residual, weight, block)
        for g, ref, err in zip(got, refs, errs):
            assert (np.abs(f64(g) - ref) <= 2.0 ** -8 * np.abs(ref) + 1.01 * err).all()
        return got

    def add_adapters(self, base, x, A, B, scale, ids, seq_start=None, out=None):
        self._count("adapters")
        rows = ids.tolist()
        if seq_start is not None:
            starts = seq_start.tolist()
            rows = [a for a, s, e in zip(rows, starts, starts[1:]) for _ in range(e - s)]
        args = [f64(t) for t in (x, base, A, B, scale)]
        ref, size = R.adapters(*args, rows)
        t = [np.abs(args[3][a]) @ np.abs(args[4][a] * (args[2][a] @ args[0][m])) for m, a in enumerate(rows)]
        bound = 2.0 ** -8 * np.abs(ref) + 1.01 * 2.0 ** -8 * np.array(t) + \
            2.0 ** -22 * ((x.shape[1] / 64 + 40) * size + 8 * np.abs(args[1]))
        got = self._W.add_adapters(base, x, A, B, scale, ids, seq_start=seq_start, out=out)
        assert (np.abs(f64(got) - ref) <= bound).all()
        return got

    def _turned(self, name, qkv, table, H, call):
        self._count(name)
        before = qkv.clone()
        call()
        RO.check(before, qkv, H, H, 128, self._positions(), RO.theta_of(128), False)
        return qkv

    def rotary(self, qkv, table, H, seq_start=None):
        return self._turned("rotary", qkv, table, H, lambda: self._W.rotary(qkv, table, H, seq_start=seq_start))

    def kv_rotary(self, cache, qkv, slots, H, table, seq_start=None):
        return self._turned("kv_rotary", qkv, table, H,
                            lambda: self._W.kv_rotary(cache, qkv, slots, H, table, seq_start=seq_start))


def test_every_call_of_a_run(monkeypatch):
    import screen_ligands as E
    W = E.W
    H, protein, lengths = 4, 37, [3, 1, 2]
    model = E.Decoder.random(H, 2, whole=True)
    table = model.around.table
    cache = W.KVCache(2, 40, H, 4, 8, 16)
    at = []
    checked = Checked(W, lambda: at)
    monkeypatch.setattr(E, "W", checked)
    # the protein's prompt
    start, slot0 = KV.i32([0, protein]), KV.i32([0])
    W.kv_extend(cache, slot0, KV.i32([protein]))
    at[:] = range(protein)

    def prefill(layer, qkv):
        W.kv_write(cache, layer, qkv, start, slot0, H)
        return W.attention_prefill(qkv, start, H)

    states = model.forward(E.random_states(protein, model.width, 1), prefill,
                           lambda q: checked.kv_rotary(cache, q, slot0, H, table, seq_start=start), KV.i32([2]), start)
    # its ligands, a token each at a time, one of them ended after the first
    slots = KV.i32([1, 2, 3])
    W.kv_fork(cache, KV.i32([0, 0, 0]), slots)
    outs = []
    for step in range(max(lengths)):
        active = KV.i32([s + 1 if step < n else -1 for s, n in enumerate(lengths)])
        W.kv_extend(cache, active, KV.i32([1, 1, 1]))
        at[:] = [protein + step if step < n else None for n in lengths]
        token = E.random_states(3, model.width, 20 + step)
        outs.append(model.forward(token, lambda layer, q: W.attention_decode(cache, layer, q, active, H),
                                  lambda q: checked.kv_rotary(cache, q, active, H, table), KV.i32([2, 0, 3])))
    assert W.get_device_error() == W.OK
    # the head's distribution at every prompt token
    head = W.quantize(torch.randn(1000, model.width, device="cuda", generator=torch.Generator(device="cuda").manual_seed(5)) / 8)
    LP.check(W.linear(states, *head), [(7 * i) % 1000 for i in range(protein)], 20)
    LP.check(W.linear(outs[-1], *head), None, 64)
    # and the same sequences without a cache
    at[:] = [*range(protein), *range(5)]
    both = KV.i32([0, protein, protein + 5])
    model.forward(E.random_states(protein + 5, model.width, 1), lambda layer, q: W.attention_prefill(q, both, H),
                  lambda q: checked.rotary(q, table, H, seq_start=both), KV.i32([1, 3]), both)
    assert checked.calls == {"norm": 25, "adapters": 10, "kv_rotary": 8, "rotary": 2}


def test_a_captured_step_is_the_launched_one():
    """Several steps of ragged sequences, twice: launched, and by replaying one captured step, with the batch
    padded; every state has the same bits."""
    import screen_ligands as E
    W = E.W
    H, lengths = 4, [33, 1, 16, 64, 7]
    model = E.Decoder.random(H, 2, whole=True)
    table, n = model.around.table, len(lengths)

    def make():
        cache = W.KVCache(2, 60, H, n, 8, 16)
        cache.pages.zero_()
        W.kv_extend(cache, KV.i32(range(n)), KV.i32(lengths))
        start = KV.i32(np.concatenate([[0], np.cumsum(lengths)]))

        def prefill(layer, qkv):
            W.kv_write(cache, layer, qkv, start, KV.i32(range(n)), H)
            return W.attention_prefill(qkv, start, H)

        model.forward(E.random_states(sum(lengths), model.width, 3), prefill,
                      lambda q: W.kv_rotary(cache, q, KV.i32(range(n)), H, table, seq_start=start), KV.i32([0, 1, -1, 3, 1]), start)
        return cache

    token = torch.empty((n, model.width), dtype=torch.bfloat16, device="cuda")
    active, one, target = KV.i32(range(n)), KV.i32([1] * n), KV.i32([0, 1, -1, 3, 1])

    def step(cache, workspace):
        W.kv_extend(cache, active, one)
        return model.forward(token, lambda layer, q: W.attention_decode(cache, layer, q, active, H, workspace=workspace),
                             lambda q: W.kv_rotary(cache, q, active, H, table), target)

    launched, replayed = make(), make()
    w0, w1 = launched.new_workspace(H), replayed.new_workspace(H)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(replayed, w1)
    for t in range(6):
        token.copy_(E.random_states(n, model.width, 50 + t))
        active.copy_(KV.i32([-1 if t > 2 and i % 2 else i for i in range(n)]))
        want = step(launched, w0)
        graph.replay()
        assert W.get_device_error() == W.OK
        # (a padding row's queries and keys are not turned, and its attention is zero: the same both ways)
        assert torch.equal(out, want)
    assert torch.equal(launched.seq_len, replayed.seq_len) and torch.equal(launched.page_table, replayed.page_table)


@pytest.mark.parametrize("e4m3,protein,page_tokens", [(False, 200, 16), (True, 201, 64)])
def test_shared_cache_matches_prefilled_pairs(e4m3, protein, page_tokens):
    """As the example without norms is tested: both ways round to bf16 at the same places.  A layer's four
    linears, attention and adapters are within 5e-3 of their outputs' norms, its two norms and the
    rotation within 2^-8 each; a norm keeps relative errors.  Two layers and the last norm: 2 (6 * 5e-3 + 3 *
    2^-8) + 2^-8 < 0.09; an 8-bit cache adds 2^-5 of keys and values a layer."""
    import screen_ligands as E
    from paper_2608_30877_gb300 import w4a16 as W
    model = E.Decoder.random(heads=4, n_layers=2, whole=True)
    x = E.random_states(protein, model.width, 1)
    ligands = [E.random_states(k, model.width, 10 + i) for i, k in enumerate([1, 17, 30, 5, 16, 40])]
    dtype = torch.float8_e4m3fn if e4m3 else torch.bfloat16
    got, _ = E.screen(model, x, ligands, page_tokens, dtype, target=3)
    want = E.screen_without_cache(model, x, ligands, target=3)
    assert W.get_device_error() == W.OK
    scale = model.affinities(E.random_states(64, model.width, 3)).float().std().item()
    err = (got.float() - want.float()).abs().max().item()
    assert err <= (0.09 + (2 * 2.0 ** -5 if e4m3 else 0.0)) * max(scale, want.float().abs().max().item()), err
    # it tells: the positions and the adapter matter
    other = E.screen_without_cache(model, x, ligands, target=1)
    assert (other.float() - want.float()).abs().max().item() > 3 * err
