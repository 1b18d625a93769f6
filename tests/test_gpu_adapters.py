"""Low-rank adapters against 64 bits.

Bound: one rounding of the sum with base (2^-8), and of t = scale (x A^T) to bf16 (2^-8 of each |t|, times |B|); sums of
fp32, with at most K / 64 + 40 additions in a row, whose terms are cut at 2^-23 of the largest of a tensor
core's sixteen: 2^-22 of the sum of magnitudes for each."""
import numpy as np
import pytest
import torch

from tests import layer_reference as R
from tests.kv_reference import i32

pytestmark = pytest.mark.gpu


def _W():
    from paper_2608_30877_gb300 import w4a16 as W
    return W


def f64(t):
    return t.detach().double().cpu().numpy()


def make(M, N, K, rank, pool, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + M + N + K + rank)
    rnd = lambda *s, k=1.0: (torch.randn(s, generator=g, device="cuda") * k).bfloat16()  # noqa: E731
    return dict(base=rnd(M, N), x=rnd(M, K), A=rnd(pool, rank, K, k=K ** -0.5), B=rnd(pool, N, rank, k=2 * rank ** -0.5),
                scale=torch.rand(pool, generator=g, device="cuda") * 2 - 0.5)


def check(given, ids, starts=None, **more):
    """ids: of each sequence."""
    W = _W()
    M, K = given["x"].shape
    rows = list(ids) if starts is None else [-1] * M
    if starts is not None:
        for a, s, e in zip(ids, starts, starts[1:]):
            rows[s:e] = [a] * (e - s)
    out = W.add_adapters(**given, adapters=i32(ids), seq_start=None if starts is None else i32(starts), **more)
    assert W.get_device_error() == W.OK
    x, base, A, B, scale = (f64(given[n]) for n in ("x", "base", "A", "B", "scale"))
    ref, size = R.adapters(x, base, A, B, scale, rows)
    rounded = np.zeros_like(ref)
    for m, a in enumerate(rows):
        if a >= 0:
            rounded[m] = np.abs(B[a]) @ np.abs(scale[a] * (A[a] @ x[m]))
    bound = 2.0 ** -8 * np.abs(ref) + 1.01 * 2.0 ** -8 * rounded + 2.0 ** -22 * ((K / 64 + 40) * size + 8 * np.abs(base))
    worst = (np.abs(f64(out) - ref) - bound).max()
    assert worst <= 0, (worst, np.abs(f64(out) - ref).max())
    none = torch.tensor([a < 0 for a in rows], device="cuda")
    assert torch.equal(out[none], given["base"][none])
    return out


@pytest.mark.parametrize("rank", [8, 16, 24, 32, 40, 64])
@pytest.mark.parametrize("M", [1, 2, 7, 8, 9, 16, 40, 130])
def test_a_row_each(M, rank):
    """Single tokens: an adapter each, shared ones, none."""
    for N, K, pool in ((1, 64, 1), (100, 128, 5), (1000, 1024, 40), (257, 320, 3), (4096, 512, 7)):
        given = make(M, N, K, rank, pool)
        check(given, [(7 * i) % pool for i in range(M)])
        check(given, [-1 if i % 3 == 1 else (5 * i + i // 9) % pool for i in range(M)])


@pytest.mark.parametrize("rank", [8, 16, 32, 48, 64])
@pytest.mark.parametrize("starts", [[0, 1], [0, 64], [0, 100, 100, 333], [0, 7, 8, 9, 63, 64, 65, 200], [5, 6, 130], [0, 1000],
                                    [0, *range(3, 200, 11)], list(range(301)), [0] * 120 + [50] * 120 + [51, 200]])
def test_packed(starts, rank):
    """Sequences that begin and end inside tiles, empty ones, more than a tile's list of starts, rows before and
    after them."""
    n, M = len(starts) - 1, starts[-1] + 5
    for N, K in ((72, 192), (1031, 640), (2048, 256)):
        given = make(M, N, K, rank, 4)
        check(given, [(3 * i) % 4 for i in range(n)], starts)
        check(given, [-1 if i % 2 else i % 4 for i in range(n)], starts)


def test_long_products():
    given = make(70, 512, 12288, 16, 2)
    check(given, [0, 1, -1], [0, 33, 60, 70])
    check(make(3, 640, 49152, 64, 2), [1, 0, 1])


def test_in_place_and_workspaces():
    W = _W()
    for M, starts in ((40, None), (300, [0, 100, 250, 300])):
        given = make(M, 520, 256, 16, 4)
        ids = [i % 4 for i in range(M if starts is None else 3)]
        want = check(given, ids, starts)
        seq = None if starts is None else i32(starts)
        w = torch.full((W.adapters_workspace_bytes(M, 16) // 4,), float("nan"), device="cuda")
        out = torch.full_like(want, 7)
        got = W.add_adapters(**given, adapters=i32(ids), seq_start=seq, workspace=w, out=out)
        assert got is out and torch.equal(out, want)
        base = given["base"].clone()
        got = W.add_adapters(**dict(given, base=base), adapters=i32(ids), seq_start=seq, out=base)
        assert got is base and torch.equal(base, want)


def test_nan_stays_in_its_rows_and_adapters():
    W = _W()
    given = make(64, 130, 256, 16, 4)
    ids = [i % 4 for i in range(64)]
    want = check(given, ids)
    given["x"][9, 100] = float("nan")
    given["A"][2, 3, 5] = float("inf")
    got = W.add_adapters(**given, adapters=i32(ids))
    touched = torch.tensor([i == 9 or i % 4 == 2 for i in range(64)], device="cuda")
    assert torch.equal(got[~touched], want[~touched])
    assert got[9].isnan().all()
    given = make(200, 130, 256, 16, 4)
    want = check(given, [0, 1, 2], [0, 50, 90, 200])
    given["x"][60] = float("inf")
    given["B"][3] = float("nan")
    got = W.add_adapters(**given, adapters=i32([0, 1, 2]), seq_start=i32([0, 50, 90, 200]))
    keep = torch.arange(200, device="cuda") != 60
    assert torch.equal(got[keep], want[keep])


def test_bad_lists():
    W = _W()
    given = make(20, 64, 128, 16, 4)
    for ids, starts in (([4] * 20, None), ([-2] * 20, None), ([0], [0, 21]), ([0], [-1, 20]), ([0, 1], [0, 10, 5])):
        got = W.add_adapters(**given, adapters=i32(ids), seq_start=None if starts is None else i32(starts))
        assert W.get_device_error() == W.ERR_INVALID_ARG
        if starts is None:
            assert torch.equal(got, given["base"])
    with pytest.raises(ValueError):
        W.add_adapters(**given, adapters=i32([0] * 19))
    with pytest.raises(W.W4A16Error):
        W.add_adapters(**make(20, 64, 128, 16, 4) | {"A": torch.zeros(4, 12, 128, device="cuda", dtype=torch.bfloat16),
                                                     "B": torch.zeros(4, 64, 12, device="cuda", dtype=torch.bfloat16)},
                       adapters=i32([0] * 20))


def test_streams_and_graphs():
    W = _W()
    for M, starts in ((40, None), (300, [0, 100, 250, 300])):
        given = make(M, 1024, 512, 32, 4)
        ids = i32([i % 4 for i in range(M if starts is None else 3)])
        seq = None if starts is None else i32(starts)
        want = W.add_adapters(**given, adapters=ids, seq_start=seq)
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        got = W.add_adapters(**given, adapters=ids, seq_start=seq, stream=side)
        side.synchronize()
        assert torch.equal(got, want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = W.add_adapters(**given, adapters=ids, seq_start=seq)
        for _ in range(3):
            got.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(got, want)
