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


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("Hkv,lengths,pairs", [
    (2, [5, 9], [(0, 1)]), (1, [40, 1, 33, 64, 2], [(1, 3), (3, 4)]), (96, [3, 2, 4], [(0, 2)]),
    (1, [1 + i % 3 for i in range(300)], [(0, 299), (40, 41)]), (4, [1 + i % 20 for i in range(226)], [(3, 225), (100, 101)]),
    (1, [1 + i % 2 for i in range(1500)], [(7, 8), (2, 1499), (700, 1300)]),
    (1, [1 + i % 2 for i in range(40000)], [(20000, 39999)]), (1, [1] * 40000, [(33000, 33001), (2, 5)])])
def test_writes_report_a_slot_twice(bits, Hkv, lengths, pairs):
    """The status says so, the other sequences' rows are written and what no sequence of the list has
    is as it was.  A slot that is in the list again for a sequence without rows is no error."""
    W = _W()
    n, H, T = len(lengths), 1, 16
    g = torch.Generator(device="cuda").manual_seed(n + bits)

    def cache():
        c = W.KVCache(1, sum(-(-x // T) for x in lengths) + 1, Hkv, n + 1, max(-(-x // T) for x in lengths), T,
                      torch.bfloat16 if bits == 16 else torch.float8_e4m3fn)
        c.pages.view(torch.uint8).fill_(0x5A)
        if bits == 8:
            c.exponents.fill_(0x5A)
        W.kv_extend(c, R.i32(range(n)), R.i32(lengths))
        return c

    def rows(c):  # the sequences' rows as the cache has them, one list entry for each
        raw = c.pages.view(torch.uint8)[0]
        table = c.page_table.cpu()
        seq = np.repeat(np.arange(n), lengths)
        pos = np.concatenate([np.arange(x) for x in lengths])
        page, at = table[torch.from_numpy(seq), torch.from_numpy(pos // T)].long().cuda(), torch.from_numpy(pos % T).cuda()
        # [tokens, 2, heads, bytes], [tokens, heads, 2]
        held = [raw.transpose(0, 1)[page, :, :, at].cpu()] + ([c.exponents[0][page, :, at].cpu()] if bits == 8 else [])
        return seq, held

    start = np.concatenate([[0], np.cumsum(lengths)])
    qkv = torch.randn((int(start[-1]) + 3, (H + 2 * Hkv) * D), generator=g, device="cuda").bfloat16()
    good = cache()
    slots = R.i32(range(n))
    W.kv_write(good, 0, qkv, R.i32(start), slots, H)
    assert W.get_device_error() == W.OK
    wrong, bad = slots.clone(), set()
    for a, b in pairs:
        if lengths[b] > lengths[a]:  # (no more rows than the slot has tokens, which would be an error by itself)
            a, b = b, a
        wrong[b] = wrong[a]
        bad |= {a, b}
    c = cache()
    W.kv_write(c, 0, qkv, R.i32(start), wrong, H)
    assert W.get_device_error() == W.ERR_INVALID_ARG
    (seq, want), (_, got) = rows(good), rows(c)
    out = torch.from_numpy(np.isin(seq, sorted(bad)))
    left = torch.from_numpy(np.isin(seq, sorted(set(range(n)) - set(wrong.tolist()))))  # slots that went out of the list
    for w, x in zip(want, got):
        assert torch.equal(x[~out], w[~out])
        assert bool((x[left] == 0x5A).all())
    # a sequence of no rows with another's slot, before and after it
    c = cache()
    W.kv_write(c, 0, qkv, R.i32([0, 0, *start[1:], start[-1]]), R.i32([n - 1, *range(n), 0]), H)
    assert W.get_device_error() == W.OK
    assert all(torch.equal(w, x) for w, x in zip(want, rows(c)[1]))
