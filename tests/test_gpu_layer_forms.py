"""Forms of the layer operators that their own files leave out: rotation by the lengths of an 8-bit cache, scaled frequencies of
neighbouring pairs, log probabilities past 2^31 elements within their elementwise bounds."""
import types

import pytest
import torch

from tests import kv_reference as KV
from tests import test_gpu_log_probs as LP
from tests import test_gpu_rotary as RO
from tests.test_gpu_layer_limits import _bf16, _rows

pytestmark = pytest.mark.gpu


def _W():
    from paper_2608_30877_gb300 import w4a16 as W
    return W


@pytest.mark.parametrize("pairs", [False, True])
def test_rotary_of_an_8_bit_cache(pairs):
    W = _W()
    lengths = [40, 1, 17, 300, 16]
    c = RO._cache(lengths, e4m3=True)
    table = W.RotaryTable(128, layout=W.ROTARY_PAIRS if pairs else W.ROTARY_HALF)
    slots = [3, -1, 0, 4, 6, 1, 3]
    qkv = RO.make(len(slots), 4, 2)
    before = qkv.clone()
    W.kv_rotary(c, qkv, KV.i32(slots), 4, table)
    assert W.get_device_error() == W.OK
    RO.check(before, qkv, 4, 2, 128, [None if s in (-1, 6) else lengths[s] - 1 for s in slots], RO.theta_of(128), pairs)
    slots, starts = [4, 2, 3], [0, 16, 21, 320]
    qkv = RO.make(325, 4, 2)
    before = qkv.clone()
    W.kv_rotary(c, qkv, KV.i32(slots), 4, table, seq_start=KV.i32(starts))
    assert W.get_device_error() == W.OK
    want = [lengths[s] - (e - a) + i for s, a, e in zip(slots, starts, starts[1:]) for i in range(e - a)] + [None] * 5
    RO.check(before, qkv, 4, 2, 128, want, RO.theta_of(128), pairs)


@pytest.mark.parametrize("scaling", [("LINEAR", 4.0, 0, 1.0, 32.0), ("BY_TURNS", 8.0, 8192, 1.0, 4.0), ("BY_INDEX", 32.0, 4096, 1.0, 32.0)])
def test_scaling_of_neighbouring_pairs(scaling):
    W = _W()
    name, factor, trained, low, high = scaling
    kind = getattr(W, "ROTARY_SCALE_" + name)
    table = W.RotaryTable(96, 500000.0, kind, factor, trained, low, high, W.ROTARY_PAIRS, attention_factor=1.25)
    qkv = RO.make(50, 8, 2)
    before = qkv.clone()
    W.rotary(qkv, table, 8, 2, first=KV.i32([2000 * i for i in range(50)]))
    RO.check(before, qkv, 8, 2, 128, [2000 * i for i in range(50)], RO.theta_of(96, 500000.0, kind, factor, trained, low, high),
             True, 1.25)


def test_log_probs_past_2_31_elements(monkeypatch):
    """The sampled rows, compared as test_gpu_log_probs compares whole calls."""
    W = _W()
    M, V, k = 17001, 131072, 20
    x = _bf16(M, V, scale=2.0, seed=15)
    targets = torch.arange(M, device="cuda", dtype=torch.int32) * 7
    results = W.log_probs(x, targets, k)
    at = _rows(M, V)
    index = torch.tensor(at, device="cuda")
    sampled = types.SimpleNamespace(log_probs=lambda *_: tuple(t[index] for t in results))
    monkeypatch.setattr(LP, "_W", lambda: sampled)
    LP.check(x[index], [7 * r for r in at], k)
    assert W.get_device_error() == W.OK
