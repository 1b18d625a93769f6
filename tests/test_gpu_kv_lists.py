"""A slot twice in the list of a call that stores to the cache: an error, whatever its places."""
import numpy as np
import pytest
import torch

from tests import kv_reference as R
from tests.test_gpu_attention_decode import Case

pytestmark = pytest.mark.gpu
D = 128


def _W():
    from paper_2608_30877_gb300 import w4a16 as W
    return W


@pytest.mark.parametrize("bits,H,Hkv", [(16, 4, 2), (8, 4, 4), (8, 24, 2)])
@pytest.mark.parametrize("n,pairs", [(2, [(0, 1)]), (6, [(1, 4), (4, 5)]), (31, [(2, 30)]), (192, [(0, 191)]),
                                     (193, [(5, 192)]), (700, [(10, 650)]), (700, [(300, 301), (300, 699)])])
def test_attention_refuses_a_slot_twice(bits, H, Hkv, n, pairs):
    """All rows are zero, the cache is as it was and the status says so; entries of -1 repeat as they
    like, and the same list without the repetition gives what it gave."""
    W = _W()
    lengths = [1 + 29 * i % 120 for i in range(n)]
    case = Case(bits, H, Hkv, 16, lengths, n + bits, layers=1, layer=0)
    c = case.cache
    want = W.attention_decode(c, 0, case.qkv, case.slots, H)
    assert W.get_device_error() == W.OK
    before = [t.clone() for t in case.before() if t is not None]
    wrong = case.slots.clone()
    for a, b in pairs:
        wrong[b] = wrong[a]
    out = torch.full_like(want, 7.0)
    W.attention_decode(c, 0, case.qkv.neg(), wrong, H, out=out)
    assert W.get_device_error() == W.ERR_INVALID_ARG
    assert (out == 0).all()
    assert all(torch.equal(x, y) for x, y in zip(before, [t for t in case.before() if t is not None]))
    padded = case.slots.clone()
    gone = sorted({i for p in pairs for i in p})
    padded[gone] = -1
    out = W.attention_decode(c, 0, case.qkv, padded, H)
    assert (out[gone] == 0).all()
    for i in [i for i in range(n) if i not in gone][:8]:
        case.check_row(out, i, 32768)
    assert torch.equal(W.attention_decode(c, 0, case.qkv, case.slots, H), want)
    assert W.get_device_error() == W.OK


def test_attention_over_the_most_slots():
    """65536 slots of a cache, most of them empty, a row for each; then one of them twice."""
    W = _W()
    n = 1 << 16
    c = W.KVCache(1, 300, 1, n, 2, 16)
    c.pages.zero_()
    live = np.random.default_rng(3).permutation(n)[:200]
    W.kv_extend(c, R.i32(live), R.i32([1] * 200))
    slots = torch.randperm(n, device="cuda").to(torch.int32)
    qkv = torch.randn((n, 3 * D), device="cuda").bfloat16()
    out = W.attention_decode(c, 0, qkv, slots, 1)
    assert W.get_device_error() == W.OK
    rows = torch.isin(slots, R.i32(live))  # one token: the row's own value
    assert torch.equal(out[rows], qkv[rows, 2 * D:]) and (out[~rows] == 0).all()
    for a, b in ((0, n - 1), (40000, 40001), (5, 60000)):
        wrong = slots.clone()
        wrong[b] = wrong[a]
        before = c.pages.clone()
        out = W.attention_decode(c, 0, qkv.neg(), wrong, 1)
        assert W.get_device_error() == W.ERR_INVALID_ARG
        assert (out == 0).all() and torch.equal(before, c.pages)
