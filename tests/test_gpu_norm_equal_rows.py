"""Layer norms of rows whose values are equal, or nearly so: the formula's 0 times the weight, plus the bias."""
import numpy as np
import pytest
import torch

from tests import test_gpu_residual_norm as RN

pytestmark = pytest.mark.gpu
SHAPES = [(9, 64), (9, 100), (9, 515), (5, 1000), (3, 4099), (3, 12288), (2, 20000), (2, 49151), (1300, 2056), (1300, 8200)]


def _equal(M, D):
    """A value of 24 bits for each row, of 10^-2 to 10^10."""
    x = torch.rand(M, 1, generator=torch.Generator(device="cuda").manual_seed(D), device="cuda") + 0.5
    return (x * 10.0 ** (torch.arange(M, device="cuda") % 13 - 2)[:, None]).expand(M, D)


@pytest.mark.parametrize("bits", [16, 32])
@pytest.mark.parametrize("M,D", SHAPES)
def test_equal_values(M, D, bits):
    """(x - mean) is 0 where the mean's sum is exact: values of 8 bits, of which at most 2^16 are added."""
    W = RN._W()
    given = RN.inputs(M, D, bits, False, 0, False, True)
    x = _equal(M, D).bfloat16().to(given["residual"].dtype).contiguous()
    for eps in (1e-5, 1e-12):
        out, _ = W.residual_norm(x, given["weight"], bias=given["bias"], kind=W.NORM_LAYER, eps=eps)
        assert torch.equal(out, given["bias"].expand(M, D))


@pytest.mark.parametrize("M,D", SHAPES)
def test_equal_values_of_24_bits(M, D):
    """The mean is off by what a sum's rounding leaves, within the bounds of test_gpu_residual_norm."""
    RN.check(dict(RN.inputs(M, D, 32, False, 0, False, True), residual=_equal(M, D).contiguous()), layer=True)


@pytest.mark.parametrize("M,D", SHAPES)
def test_one_value_apart(M, D):
    """All equal but one, a step of bf16 from them: most differences from the mean are of the size of an fp32 mean's
    error.  The mean is within a step of fp32's (2^-24 of it), which moves the differences and, through their mean square,
    all results; the mean square's root is within 2^-17, and the store rounds."""
    W = RN._W()
    x = torch.full((M, D), 100.0, device="cuda", dtype=torch.bfloat16)
    x[:, D // 2] = 100.5
    out = RN.f64(W.residual_norm(x, kind=W.NORM_LAYER)[0])
    v = RN.f64(x)
    c = v - v.mean(-1, keepdims=True)
    rstd = 1 / np.sqrt((c * c).mean(-1, keepdims=True) + 1e-5)
    mean_err = 2.0 ** -24 * 100.5
    bound = 2.0 ** -8 * np.abs(c * rstd) + 1.01 * (mean_err * rstd + np.abs(c * rstd) * (RN.ROOT + mean_err * rstd))
    assert (np.abs(out - c * rstd) <= bound).all()
