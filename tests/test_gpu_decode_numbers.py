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
