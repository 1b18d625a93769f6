"""Decode attention where its number formats end: 8-bit values with the smallest exponents,
weights that only matter where the large ones meet zeros, NaN codes, and the last tile of the
longest sequence that a table can have."""
import math

import numpy as np
import pytest
import torch

from tests import kv_reference as R
from tests.test_gpu_attention_decode import Case, _values

pytestmark = pytest.mark.gpu
D = 128


def _W():
    from paper_2608_30877_gb300 import w4a16 as W
    return W


def _reference(case, i, low=0):
    """Row i's inputs and 64-bit output: kv [2, n, Hkv, D], ref and size [H, D]."""
    n, H = case.lengths[i], case.H
    row = case.qkv[i].double().cpu().numpy()
    kv = _values(case.cache, case.layer, case.slot_pages[i], n, case.T)
    return kv, *R.attention(row[:H * D].reshape(H, D), kv[0, low:], kv[1, low:])


@pytest.mark.parametrize("H,Hkv", [(4, 4), (6, 2), (20, 1)])
def test_values_of_the_smallest_exponents(H, Hkv):
    """Values of up to 2^-111, whose exponents are at the format's end, with equal weights (sums of
    up to the length) and of one sign, so that their mean is not lost in what the bound
    allows: the other cases' bound without its absolute part."""
    W = _W()
    case = Case(8, H, Hkv, 32, [1, 20, 400, 5000, 20000], 31, layers=1, layer=0, q_scale=0.0)
    case.cache.exponents[..., 1] = 7  # 2^-120
    values = case.cache.pages.view(torch.uint8)[:, 1]
    values.copy_(values & 0x7F)
    case.qkv[:, (H + Hkv) * D:] = case.qkv[:, (H + Hkv) * D:].abs() * 2.0 ** -112
    out = W.attention_decode(case.cache, 0, case.qkv, case.slots, H)
    assert W.get_device_error() == W.OK
    for i in range(len(case.lengths)):
        _, ref, size = _reference(case, i)
        err = np.abs(out[i].double().cpu().numpy().reshape(H, D) - ref)
        bound = 1.01 * 2.0 ** -9 * np.abs(ref) + (2.0 ** -8 + 2.0 ** -10) * size
        assert (err <= bound).all(), f"row {i}: worst {np.max(err / bound):.3f} of the bound"


# bits below the largest key's weight of the keys that have values in dimensions 16 k on
LEVELS = [0, 6, 14, 20, 30, 38, 45, 58]


@pytest.mark.parametrize("by", ["scores", "value exponents"])
@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("H,Hkv", [(2, 2), (6, 2), (20, 1)])
@pytest.mark.parametrize("n", [60, 6000])
def test_small_weights_where_large_ones_meet_zeros(by, bits, H, Hkv, n):
    """Keys of eight weights; those of level k have zeros as values from dimension 16 (k + 1) on, so
    that the dimensions 16 k .. 16 k + 15 are the sum of the keys of level k and below.

    The bound is the other cases' elementwise one, in which `size` is then that small sum itself.
    On the 8-bit cache a weight (times its value's power of two) of less than 2^-51 of the largest
    is an fp16 subnormal of a unit of 2^-24, with 2^24 before and 2^12.9 at least for the largest: each
    is off by at most 2^-25-24-12.9 = 2^-61.9 of it, times the value's code."""
    W = _W()
    case = Case(bits, H, Hkv, 32, [n, n], 32, layers=1, layer=0)
    c, g = case.cache, torch.Generator(device="cuda").manual_seed(n + H + bits)
    # scores: 8.16 bits per unit of the key's first dimension for a query of 64 there
    case.qkv[:, :H * D] = 0
    case.qkv[:, 0:H * D:D] = 64.0
    unit = 64.0 * math.log2(math.e) / math.sqrt(D)
    level = torch.randint(0, len(LEVELS), (n,), generator=g, device="cuda")
    level[n // 3], level[-1] = 0, len(LEVELS) - 1
    if n > 100:  # one key has the most weight, the other 5999 are far below
        level = torch.where(level == 0, 3, level)
        level[n // 3] = 0
    drop = torch.tensor(LEVELS, device="cuda", dtype=torch.float32)[level]
    key0 = (-drop / unit if by == "scores" else torch.zeros_like(drop)).bfloat16().float()
    ve = (-drop if by == "value exponents" else torch.zeros_like(drop)).int()  # of the values' powers of two
    dims = torch.arange(D, device="cuda")
    for i in range(2):
        values = torch.randn((n, Hkv, D), generator=g, device="cuda").mul_(112).clamp_(-448, 448)
        values = values.to(torch.float8_e4m3fn).float()
        values[dims[None, None].expand(n, Hkv, D) >= 16 * (level[:, None, None] + 1)] = 0
        pos = torch.arange(n, device="cuda")
        page, at = case.slot_pages[i][pos // 32], pos % 32
        keys = torch.zeros((n, Hkv, D), device="cuda")
        keys[:, :, 0] = key0[:, None]
        if bits == 16:
            c.pages[0, 0][page, :, at] = keys.bfloat16()
            c.pages[0, 1][page, :, at] = (values * torch.exp2(ve.float())[:, None, None]).bfloat16()
        else:
            raw = c.pages.view(torch.uint8)
            raw[0, 0][page, :, at] = keys.to(torch.float8_e4m3fn).view(torch.uint8)
            raw[0, 1][page, :, at] = values.to(torch.float8_e4m3fn).view(torch.uint8)
            c.exponents[0][page, :, at] = torch.stack([torch.full_like(ve, 127), 127 + ve], -1) \
                .to(torch.uint8)[:, None].expand(n, Hkv, 2)
        # the new token: of the lowest level, the same by either way
        new = torch.cat([keys[-1], values[-1] * torch.exp2(ve[-1].float())]).bfloat16()
        case.qkv[i, H * D:] = new.reshape(-1)
    out = W.attention_decode(c, 0, case.qkv, case.slots, H)
    assert W.get_device_error() == W.OK
    two = np.ldexp(1.0, ve.cpu().numpy())[:, None]
    for i in range(2):
        kv, ref, size = _reference(case, i)
        s = kv[0, :, :, 0] * 64.0 / math.sqrt(D)  # [n, Hkv]
        p = np.exp(s - s.max(0))
        weight = p * two / (p * two).max(0)
        bound = 1.01 * 2.0 ** -9 * np.abs(ref) + (2.0 ** -8 + 2.0 ** -10) * size
        if bits == 8:
            codes = np.abs(kv[1] / two[:, :, None]).sum(0)  # (the new token's have their power in `kv` too)
            top = (p * two).max(0) / p.sum(0)
            bound = bound + np.repeat(2.0 ** -61.9 * top[:, None] * codes, H // Hkv, 0)
        err = np.abs(out[i].double().cpu().numpy().reshape(H, D) - ref)
        assert (err <= bound).all(), f"row {i}: worst {np.max(err / bound):.3f} at {np.argwhere(err > bound)[0]}"
        # the bound tells: without the keys below 2^-29, 2^-40, 2^-50 or 2^-57 of the largest the
        # reference itself is outside it
        for bits_down in (29, 40, 50, 57):
            part = np.einsum("nh,nhd->hd", np.where(weight < 2.0 ** -bits_down, 0.0, p), kv[1]) / p.sum(0)[:, None]
            assert (np.abs(np.repeat(part, H // Hkv, 0) - ref) > bound).any(), bits_down


@pytest.mark.parametrize("H,Hkv", [(2, 2), (6, 2), (24, 2)])
def test_nan_codes_are_felt(H, Hkv):
    """A NaN code as a key's makes its head's rows NaN, as a value's one dimension of them; other
    heads and sequences do not see it, and outside the window nobody does."""
    W = _W()
    case = Case(8, H, Hkv, 16, [50, 50, 50, 300], 33)
    raw = case.cache.pages.view(torch.uint8)
    raw[1, 0, case.slot_pages[0][1], 1, 3, 5] = 0x7F
    raw[1, 1, case.slot_pages[1][2], 0, 0, 77] = 0xFF
    raw[1, :, case.slot_pages[3][0], :, 7] = 0x7F
    out = W.attention_decode(case.cache, 1, case.qkv, case.slots, H, window=60)
    group = H // Hkv
    rows = out.float().view(4, Hkv, group, D)
    assert torch.isnan(rows[0, 1]).all() and torch.isfinite(rows[0, 0]).all()
    assert torch.isnan(rows[1, 0, :, 77]).all()
    rows[1, 0, :, 77] = 0
    assert torch.isfinite(rows[1]).all()
    case.check_row(out, 2, 60)
    case.check_row(out, 3, 60)
    assert W.get_device_error() == W.OK


@pytest.mark.parametrize("bits", [16, 8])
def test_infinities_of_the_new_token(bits):
    """The new token's infinities are the format's largest values on the 8-bit cache, and felt on
    the other."""
    W = _W()
    case = Case(bits, 6, 2, 16, [1, 40, 200], 34)
    case.qkv[:, 8 * D + 5] = float("inf")       # a value of head 0
    case.qkv[:, 9 * D + 9] = float("-inf")      # and of head 1
    out = W.attention_decode(case.cache, 1, case.qkv, case.slots, 6)
    if bits == 8:
        for i in range(3):
            case.check_row(out, i, 32768)
        return
    rows = out.float().view(3, 2, 3, D)
    assert torch.isposinf(rows[:, 0, :, 5]).all() and torch.isneginf(rows[:, 1, :, 9]).all()
    rows[:, 0, :, 5] = rows[:, 1, :, 9] = 0
    assert torch.isfinite(rows).all()


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("before", [0, 1, 17, 40, 120])
def test_the_last_tokens_below_two_to_the_31(bits, before):
    """The longest sequence of a table, 2^31 - 16 tokens in pages of 16, seen through a window: its
    last tile ends where 31 bits do."""
    W = _W()
    H, Hkv, T, window, pages = 6, 2, 16, 300, 24
    entries = (2 ** 31 - 1) // T
    n = entries * T - before
    table = torch.zeros((1, entries), dtype=torch.int32, device="cuda")
    last = (n - 1) // T
    table[0, last - pages + 1:last + 1] = torch.randperm(pages, device="cuda").to(torch.int32)
    g = torch.Generator(device="cuda").manual_seed(before + bits)
    shape = (1, 2, pages, Hkv, T, D)
    if bits == 16:
        pool, exps = torch.randn(shape, generator=g, device="cuda").bfloat16(), None
    else:
        pool = (torch.randn(shape, generator=g, device="cuda") * 112).clamp(-448, 448).to(torch.float8_e4m3fn)
        exps = torch.randint(116, 124, (1, pages, Hkv, T, 2), generator=g, device="cuda", dtype=torch.uint8)
    refs = torch.ones(pages, dtype=torch.int32, device="cuda")
    c = W.KVCache.from_tensors(pool, table, torch.tensor([n], dtype=torch.int32, device="cuda"), refs, exps)
    qkv = torch.randn((1, (H + 2 * Hkv) * D), generator=g, device="cuda").bfloat16()
    out = W.attention_decode(c, 0, qkv, R.i32([0]), H, window=window)
    assert W.get_device_error() == W.OK
    pos = torch.arange(n - window, n, device="cuda")
    page, at = table[0, pos // T].long(), pos % T
    if bits == 16:
        kv = torch.stack([pool[0, w][page, :, at] for w in (0, 1)]).double().cpu().numpy()
    else:
        codes = np.stack([pool.view(torch.uint8)[0, w][page, :, at].view(torch.float8_e4m3fn).double().cpu().numpy()
                          for w in (0, 1)])
        e = exps[0][page, :, at].int().cpu().numpy() - 127
        kv = np.stack([np.ldexp(codes[w], e[..., w, None]) for w in (0, 1)])
    row = qkv[0].double().cpu().numpy()
    assert np.array_equal(kv[:, -1], R.held(row[H * D:].reshape(2, Hkv, D), bits))
    ref, size = R.attention(row[:H * D].reshape(H, D), kv[0], kv[1])
    err = np.abs(out[0].double().cpu().numpy().reshape(H, D) - ref)
    assert (err <= 1.01 * 2.0 ** -9 * np.abs(ref) + (2.0 ** -8 + 2.0 ** -10) * size).all()
