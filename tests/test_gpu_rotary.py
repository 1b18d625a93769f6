"""Rotary positions against 64 bits.

Bound: one rounding to bf16 (2^-8 of the value), and cosine and sine: the angle's fraction of a turn is cut at
2^-32 and rounded to 2^-25 of a turn at most (2^-22 radians), the function is within 2 steps (2^-22), the products
add 2^-23; a frequency is off by a few 2^-53 of itself, which position times angle multiplies (also in the
reference)."""
import numpy as np
import pytest
import torch

from tests import layer_reference as R
from tests import kv_reference as KV

pytestmark = pytest.mark.gpu


def _W():
    from paper_2608_30877_gb300 import w4a16 as W
    return W


def f64(t):
    return t.detach().double().cpu().numpy()


def make(M, H, Hkv, d=128, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + M)
    return torch.randn((M, (H + 2 * Hkv) * d), generator=g, device="cuda").bfloat16()


def check(before, after, H, Hkv, d, positions, theta, pairs, factor=1.0):
    """positions: a number for each row, None for one that is left as it is."""
    M = len(positions)
    x, y = f64(before).reshape(M, H + 2 * Hkv, d), f64(after).reshape(M, H + 2 * Hkv, d)
    rot = 2 * len(theta)
    left = np.array([p is None for p in positions])
    assert np.array_equal(x[left], y[left])
    assert np.array_equal(x[:, H + Hkv:], y[:, H + Hkv:]) and np.array_equal(x[..., rot:], y[..., rot:])
    at = np.array([0 if p is None else p for p in positions], dtype=np.float64)
    ref = R.rotate(x[:, :H + Hkv], at, theta, pairs, factor)[~left]
    got = y[:, :H + Hkv][~left]
    slip = 2.0 ** -20 + 2.0 ** -49 * at[~left, None] * np.asarray(theta)
    both = np.abs(x[:, :H + Hkv])[~left]
    if pairs:
        size, slip = both[..., 0:rot:2] + both[..., 1:rot:2], np.repeat(slip, 2, axis=1)
        size = np.repeat(size, 2, axis=-1)
    else:
        size = both[..., :rot // 2] + both[..., rot // 2:rot]
        size, slip = np.concatenate([size, size], axis=-1), np.concatenate([slip, slip], axis=1)
    bound = 2.0 ** -8 * np.abs(ref[..., :rot]) + 1.01 * slip[:, None, :] * size * abs(factor)
    worst = (np.abs(got[..., :rot] - ref[..., :rot]) - bound).max() if len(ref) else 0.0
    assert worst <= 0, worst


def theta_of(rot, base=10000.0, *scaling):
    return [R.frequency(rot, i, base, *scaling) for i in range(rot // 2)]


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("d,rot", [(128, 128), (128, 64), (128, 16), (128, 96), (64, 64), (64, 48), (256, 256), (80, 80), (72, 16), (512, 32)])
def test_heads(d, rot, pairs):
    W = _W()
    table = W.RotaryTable(rot, layout=W.ROTARY_PAIRS if pairs else W.ROTARY_HALF)
    for M, H, Hkv in ((1, 1, 1), (5, 3, 3), (33, 12, 2), (300, 8, 1), (2, 96, 96), (4, 0, 5), (4, 7, 0)):
        qkv = make(M, H, Hkv, d)
        before = qkv.clone()
        W.rotary(qkv, table, H, Hkv, first=torch.arange(M, dtype=torch.int32, device="cuda") * 37, head_dim=d)
        check(before, qkv, H, Hkv, d, [37 * i for i in range(M)], theta_of(rot), pairs)


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("starts", [[0, 7], [0, 0, 1, 1, 40, 41], [3, 10, 10, 64, 200], [0, 5000], [2, 3, 4, 5, 6, 1000, 3001]])
def test_packed(starts, pairs):
    """Sequences of none, one and many tokens, rows outside them, first positions, skipped sequences."""
    W = _W()
    H, Hkv, M = 4, 2, starts[-1] + 3
    table = W.RotaryTable(64, 500000.0, layout=W.ROTARY_PAIRS if pairs else W.ROTARY_HALF)
    seq = KV.i32(starts)
    for first in (None, [0 if i % 3 else 1000 * i for i in range(len(starts) - 1)], [-1 if i % 2 else 5 for i in range(len(starts) - 1)]):
        qkv = make(M, H, Hkv)
        before = qkv.clone()
        W.rotary(qkv, table, H, Hkv, seq_start=seq, first=None if first is None else KV.i32(first))
        assert W.get_device_error() == W.OK
        want = [None] * M
        for s, (a, b) in enumerate(zip(starts, starts[1:])):
            f = 0 if first is None else first[s]
            for m in range(a, b):
                want[m] = None if f < 0 else f + m - a
        check(before, qkv, H, Hkv, 128, want, theta_of(64, 500000.0), pairs)


@pytest.mark.parametrize("pairs", [False, True])
def test_far_positions(pairs):
    """Angles are taken modulo a turn exactly: up to 2^31 tokens from the start, and past it within a
    sequence."""
    W = _W()
    at = [0, 1, 100003, 1 << 24, (1 << 24) + 1, 123456789, (1 << 31) - 1]
    table = W.RotaryTable(128, 10000.0, layout=W.ROTARY_PAIRS if pairs else W.ROTARY_HALF)
    qkv = make(len(at), 4, 4)
    before = qkv.clone()
    W.rotary(qkv, table, 4, first=KV.i32(at))
    check(before, qkv, 4, 4, 128, at, theta_of(128), pairs)
    qkv = make(6, 4, 4)
    before = qkv.clone()
    W.rotary(qkv, table, 4, seq_start=KV.i32([0, 6]), first=KV.i32([(1 << 31) - 3]))
    check(before, qkv, 4, 4, 128, [(1 << 31) - 3 + i for i in range(6)], theta_of(128), pairs)


@pytest.mark.parametrize("scaling", [("LINEAR", 4.0, 0, 1.0, 32.0), ("BY_TURNS", 8.0, 8192, 1.0, 4.0), ("BY_INDEX", 32.0, 4096, 1.0, 32.0)])
def test_scaling_and_factor(scaling):
    W = _W()
    name, factor, trained, low, high = scaling
    kind = getattr(W, "ROTARY_SCALE_" + name)
    table = W.RotaryTable(128, 500000.0, kind, factor, trained, low, high, attention_factor=1.3465)
    qkv = make(50, 8, 2)
    before = qkv.clone()
    W.rotary(qkv, table, 8, 2, first=KV.i32([2000 * i for i in range(50)]))
    check(before, qkv, 8, 2, 128, [2000 * i for i in range(50)], theta_of(128, 500000.0, kind, factor, trained, low, high), False,
          float(np.float32(1.3465)))


def test_bad_tables():
    W = _W()
    table = W.RotaryTable(64)
    for starts in ([0, 5, 3, 10], [-1, 5], [0, 11], [4, 2, 2, 2]):
        qkv = make(10, 2, 2)
        W.rotary(qkv, table, 2, seq_start=KV.i32(starts))
        assert W.get_device_error() == W.ERR_INVALID_ARG
    qkv = make(10, 2, 2)
    W.rotary(qkv, table, 2, seq_start=KV.i32([0, 10]))
    assert W.get_device_error() == W.OK


def _cache(lengths, T=16, spare=3, e4m3=False):
    W = _W()
    n = len(lengths)
    pages = sum(-(-k // T) for k in lengths) + 20
    c = W.KVCache(1, pages, 2, n + spare, max(-(-k // T) for k in lengths) + 4, T,
                  torch.float8_e4m3fn if e4m3 else torch.bfloat16)
    W.kv_extend(c, KV.i32(range(n)), KV.i32(lengths))
    assert W.get_device_error() == W.OK
    return c


@pytest.mark.parametrize("pairs", [False, True])
def test_of_a_cache(pairs):
    W = _W()
    lengths = [40, 1, 17, 300, 16]
    c = _cache(lengths)
    table = W.RotaryTable(128, layout=W.ROTARY_PAIRS if pairs else W.ROTARY_HALF)
    # one row each: in any order, skipped ones, an empty slot's, a slot twice
    slots = [3, -1, 0, 4, 6, 1, 3]
    qkv = make(len(slots), 4, 2)
    before = qkv.clone()
    W.kv_rotary(c, qkv, KV.i32(slots), 4, table)
    assert W.get_device_error() == W.OK
    want = [None if s == -1 or s == 6 else lengths[s] - 1 for s in slots]
    check(before, qkv, 4, 2, 128, want, theta_of(128), pairs)
    # prompts: the last tokens of their sequences
    slots, rows = [4, 2, -1, 0, 3], [16, 5, 4, 0, 299]
    starts = np.concatenate([[0], np.cumsum(rows)]).tolist()
    qkv = make(starts[-1] + 2, 4, 2)
    before = qkv.clone()
    W.kv_rotary(c, qkv, KV.i32(slots), 4, table, seq_start=KV.i32(starts))
    assert W.get_device_error() == W.OK
    want = [None] * (starts[-1] + 2)
    for s, a, n in zip(slots, starts, rows):
        for i in range(n):
            want[a + i] = None if s < 0 else lengths[s] - n + i
    check(before, qkv, 4, 2, 128, want, theta_of(128), pairs)


def test_of_a_cache_refusals():
    W = _W()
    c = _cache([40, 5])
    table = W.RotaryTable(128)
    for slots, starts in (([9], None), ([-2], None), ([1], [0, 6]), ([0, 1], [0, 8, 14])):
        qkv = make(1 if starts is None else starts[-1], 4, 2)
        before = qkv.clone()
        W.kv_rotary(c, qkv, KV.i32(slots), 4, table, seq_start=None if starts is None else KV.i32(starts))
        assert W.get_device_error() == W.ERR_INVALID_ARG
        bad = len(before) if starts is None or len(slots) == 1 else 6
        assert torch.equal(qkv[-bad:], before[-bad:])
    # a refused growth: the step's rows are left alone
    W.kv_extend(c, KV.i32([0]), KV.i32([100000]))
    assert W.get_device_error() != W.OK
    qkv = make(2, 4, 2)
    before = qkv.clone()
    W.kv_rotary(c, qkv, KV.i32([0, 1]), 4, table)
    assert W.get_device_error() == W.ERR_INVALID_ARG
    assert torch.equal(qkv[0], before[0])
    check(before[1:], qkv[1:], 4, 2, 128, [4], theta_of(128), False)


def test_graph_follows_the_cache():
    """A captured step turns by the lengths of its replay."""
    W = _W()
    lengths = [40, 1, 17]
    c = _cache(lengths)
    table = W.RotaryTable(64)
    slots, one = KV.i32([0, 1, 2]), KV.i32([1, 1, 1])
    x = make(3, 4, 2)
    qkv = torch.empty_like(x)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        W.kv_extend(c, slots, one)
        qkv.copy_(x)
        W.kv_rotary(c, qkv, slots, 4, table)
    for step in range(20):
        graph.replay()
        assert W.get_device_error() == W.OK
        check(x, qkv, 4, 2, 128, [n + step for n in lengths], theta_of(64), False)


def test_another_stream():
    W = _W()
    table = W.RotaryTable(64)
    x = make(700, 4, 2)
    want = W.rotary(x.clone(), table, 4, 2, seq_start=KV.i32([0, 300, 700]))
    seq = KV.i32([0, 300, 700])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    W.rotary(x, table, 4, 2, seq_start=seq, stream=side)
    side.synchronize()
    assert torch.equal(x, want)
