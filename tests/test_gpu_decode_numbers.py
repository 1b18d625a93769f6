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
