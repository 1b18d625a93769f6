"""Residual norms of rows up to the type's largest finite value, whose squares overflow: the formula's finite numbers.

Bounds as in test_gpu_residual_norm: the row is taken again times a power of two, which rounds nothing that counts."""
import numpy as np
import pytest
import torch

from tests import test_gpu_residual_norm as RN

pytestmark = pytest.mark.gpu
TYPES = {16: torch.bfloat16, 32: torch.float32}


def _rows(M, D, bits, size, seed=0):
    """Magnitudes of size / 2 to size and of a hundredth and less of that, the largest among them."""
    g = torch.Generator(device="cuda").manual_seed(seed + M + D)
    size = torch.finfo(TYPES[bits]).max if size is None else size
    x = (torch.rand(M, D, generator=g, device="cuda") * 0.5 + 0.5) * size
    x *= torch.randint(0, 2, (M, D), generator=g, device="cuda") * 2 - 1
    x[:, 1::3] *= 1e-2
    x[:, 2::5] *= 1e-20
    x[:, 0] = size
    x = x.clamp(-size, size).to(TYPES[bits])
    assert x.isfinite().all()
    return x


def _given(residual, block=None, post=False):
    given = RN.inputs(*residual.shape, 16 if residual.dtype is torch.bfloat16 else 32, block is not None, 0, post, True)
    return dict(given, residual=residual, block=block)


# 2^126 = 8.507e37: the exponents at which a scale made from the largest one's own would leave the range
SIZES = [3e37, 8.4e37, 8.6e37, 1e38, 1.6e38, 1.8e38, 3.3e38, None]


@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("bits", [16, 32])
@pytest.mark.parametrize("size", SIZES)
def test_largest_values(size, bits, layer):
    """A warp to a row, a CTA to one, rows in shared memory, of whole and of odd units; the ring has thousands of rows."""
    for M, D in ((9, 64), (9, 515), (3, 12288), (3, 4099), (2, 49152)):
        out, _ = RN.check(_given(_rows(M, D, bits, size)), layer)
        assert out.isfinite().all()
    out, _ = RN.check(_given(_rows(1300, 2048, bits, size)), layer)
    assert out.isfinite().all()


@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("size", [3e37, 1e38, 1.8e38, None])
@pytest.mark.parametrize("M,D", [(9, 64), (9, 515), (3, 12288), (2, 20000), (1300, 2048)])
def test_post_norms_of_the_largest_values(M, D, size, layer):
    """The block's output overflows when squared, the stream does not."""
    for bits in (16, 32):
        stream = torch.randn(M, D, generator=torch.Generator(device="cuda").manual_seed(D), device="cuda").to(TYPES[bits])
        out, h = RN.check(_given(stream, _rows(M, D, 16, size), True), layer)
        assert out.isfinite().all() and h.isfinite().all()


@pytest.mark.parametrize("bits", [16, 32])
@pytest.mark.parametrize("M,D", [(5, 8), (9, 515), (3, 12288), (2, 20000), (1300, 2048)])
def test_differences_from_the_mean_past_the_largest_value(M, D, bits):
    """One value at the upper end among others at the lower one: twice the largest finite value apart."""
    W, most = RN._W(), torch.finfo(TYPES[bits]).max
    x = torch.full((M, D), -most, device="cuda", dtype=TYPES[bits])
    x[:, D // 2] = most
    out, _ = W.residual_norm(x, kind=W.NORM_LAYER)
    # (x - mean) / std of one value among D: sqrt(D - 1) there, -1 / sqrt(D - 1) elsewhere; a rounding, and a mean and
    # a mean square within 2^-17 each of magnitudes of which the others' distance from the mean is 2 / D
    want = np.full((M, D), -1 / np.sqrt(D - 1))
    want[:, D // 2] = np.sqrt(D - 1)
    got = RN.f64(out)
    moved = RN.ROOT * np.sqrt(D) / 2 + 2.0 ** -20  # the mean's error over the standard deviation, 2 most / sqrt(D)
    assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 1.01 * (moved + RN.ROOT * 2 * np.abs(want))).all()


@pytest.mark.parametrize("bits", [16, 32])
@pytest.mark.parametrize("D", [64, 515, 4096, 20000])
def test_rows_of_equal_largest_values(bits, D):
    """A layer norm is finite (what it is depends on the mean's last bit), an RMS norm one."""
    W = RN._W()
    x = torch.full((3, D), torch.finfo(TYPES[bits]).max, device="cuda", dtype=TYPES[bits])
    assert W.residual_norm(x, kind=W.NORM_LAYER)[0].isfinite().all()
    assert (W.residual_norm(x)[0] == 1).all() and (W.residual_norm(-x)[0] == -1).all()


@pytest.mark.parametrize("layer", [False, True])
def test_infinities_and_nan_beside_the_largest_values(layer):
    W = RN._W()
    for M, D in ((6, 64), (6, 515), (6, 4096), (6, 20000), (1300, 2048)):
        x = _rows(M, D, 16, None)
        x[1, 5], x[3, 7] = float("inf"), float("nan")
        out, _ = W.residual_norm(x, kind=W.NORM_LAYER if layer else W.NORM_RMS)
        assert out[3].isnan().all()
        rest = torch.arange(D, device="cuda") != 5
        assert out[1, 5].isnan() and (out[1].isnan().all() if layer else (out[1, rest] == 0).all())
        assert out[[0, 2, 4, 5]].isfinite().all()
