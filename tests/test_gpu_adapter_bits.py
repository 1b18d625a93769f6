"""What low-rank adapters keep of t = scale (x A^T) between their two products, against 64 bits.

The base is the update's own negative, rounded, so that the sum's rounding (2^-8 of what is left) hides nothing.
t is held in 16 bits, by blocks of eight ranks with a common exponent: 12 significant bits (2^-12 of each |t|), and
for those far below the block's largest 2^-18 of that; sums as in test_gpu_adapters (2^-22 of the magnitudes for each
addition in a row), with two products of at most four steps on base."""
import numpy as np
import pytest
import torch

from tests import layer_reference as R
from tests.kv_reference import i32
from tests.test_gpu_adapters import f64, make

pytestmark = pytest.mark.gpu


def _W():
    from paper_2608_30877_gb300 import w4a16 as W
    return W


def check(given, ids, starts=None):
    W = _W()
    M, K = given["x"].shape
    rows = list(ids) if starts is None else [-1] * M
    if starts is not None:
        for a, s, e in zip(ids, starts, starts[1:]):
            rows[s:e] = [a] * (e - s)
    x, A, B, scale = (f64(given[n]) for n in ("x", "A", "B", "scale"))
    update, size = R.adapters(x, np.zeros(given["base"].shape), A, B, scale, rows)
    given["base"] = -torch.from_numpy(update).to("cuda").float().bfloat16()
    base = f64(given["base"])
    out = f64(W.add_adapters(**given, adapters=i32(ids), seq_start=None if starts is None else i32(starts)))
    assert W.get_device_error() == W.OK
    bound = 2.0 ** -8 * np.abs(base + update) + 2.0 ** -22 * ((K / 64 + 40) * size + 16 * np.abs(base))
    for m, a in enumerate(rows):
        if a >= 0:
            t = np.abs(scale[a] * (A[a] @ x[m]))
            held = 2.0 ** -12 * t + 2.0 ** -18 * np.repeat(t.reshape(-1, 8).max(1), 8)
            bound[m] += 1.01 * np.abs(B[a]) @ held
    worst = (np.abs(out - base - update) / np.maximum(bound, 1e-300)).max()
    assert worst <= 1, worst


@pytest.mark.parametrize("rank", [8, 16, 24, 32, 40, 48, 64])
@pytest.mark.parametrize("M", [1, 7, 8, 40, 130])
def test_a_row_each(M, rank):
    for N, K, pool in ((100, 128, 5), (257, 320, 3), (4096, 512, 40)):
        check(make(M, N, K, rank, pool), [-1 if i % 5 == 1 else (7 * i) % pool for i in range(M)])


@pytest.mark.parametrize("rank", [8, 16, 24, 32, 40, 48, 64])
@pytest.mark.parametrize("starts", [[0, 64], [0, 100, 100, 333], [0, 7, 8, 9, 63, 64, 65, 200], [0, 1000]])
def test_packed(starts, rank):
    M = starts[-1] + 5
    for N, K in ((72, 192), (1031, 640), (2048, 256)):
        check(make(M, N, K, rank, 4), [i % 4 for i in range(len(starts) - 1)], starts)


@pytest.mark.parametrize("starts", [None, [0, 40, 150, 300]])
@pytest.mark.parametrize("size", [1e-30, 1e-5, 1e5, 1e30])
def test_sizes_of_t(size, starts):
    """The blocks' exponents, for scales of any size: what the update is is the scale's, so that B can undo it."""
    M = 20 if starts is None else 300
    for rank in (8, 40):
        given = make(M, 200, 256, rank, 3)
        given["scale"] = given["scale"] * size
        given["B"] = (given["B"].float() / size).bfloat16()
        check(given, [i % 3 for i in range(M if starts is None else 3)], starts)


@pytest.mark.parametrize("starts", [None, [0, 40, 150, 300]])
def test_ranks_of_different_sizes(starts):
    """Ranks of a block that are 2^0 .. 2^-14 of the largest, each with features of its own."""
    M = 20 if starts is None else 300
    given = make(M, 128, 256, 16, 3)
    k = torch.arange(16, device="cuda") % 8
    given["A"] *= 2.0 ** (-2.0 * k)[None, :, None]
    given["B"] *= 2.0 ** (2.0 * k)[None, None, :]
    given["B"][:, torch.arange(128, device="cuda")[:, None] % 8 != k[None, :]] = 0
    check(given, [i % 3 for i in range(M if starts is None else 3)], starts)


@pytest.mark.parametrize("starts", [None, [0, 40, 150, 300]])
def test_infinities_of_t(starts):
    """An infinite t gives what the formula gives: infinities where the products agree, NaN where they do not."""
    W = _W()
    M = 20 if starts is None else 300
    given = make(M, 96, 128, 24, 3)
    given["scale"] = given["scale"].abs() + 0.1
    given["A"] = given["A"].abs() + 0.01
    given["B"][:, :32] = given["B"][:, :32].abs() + 0.01
    given["B"][:, 32:64] = -given["B"][:, 32:64].abs() - 0.01
    given["B"][:, 64:, 3] = 0
    given["x"][5, 9], given["x"][6, 9], given["x"][7, 9] = float("inf"), -float("inf"), float("nan")
    out = W.add_adapters(**given, adapters=i32([i % 3 for i in range(M if starts is None else 3)]),
                         seq_start=None if starts is None else i32(starts)).float()
    inf = float("inf")
    assert (out[5, :32] == inf).all() and (out[5, 32:64] == -inf).all()
    assert (out[6, :32] == -inf).all() and (out[6, 32:64] == inf).all()
    assert out[5:7, 64:].isnan().all() and out[7].isnan().all()
    assert out[:5].isfinite().all() and out[8:].isfinite().all()
