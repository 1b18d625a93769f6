"""Log probabilities, entropy and best alternatives against 64 bits.

Bounds: with m the largest logit, x - m is rounded once (2^-24 of it), e^(x - m) is within 2^-22 and twice 2^-24
|x - m| of its value, and a sum's relative error is at most its longest chain of additions times 2^-24:
V / 256 + 4 units in a thread and a dozen joins.  The order of the alternatives is exact."""
import numpy as np
import pytest
import torch

from tests import layer_reference as R

pytestmark = pytest.mark.gpu


def _W():
    from paper_2608_30877_gb300 import w4a16 as W
    return W


def f64(t):
    return t.detach().double().cpu().numpy()


def check(x, targets=None, k=0, **more):
    W = _W()
    t = None if targets is None else torch.tensor(targets, dtype=torch.int32, device="cuda")
    logp, entropy, index, score = W.log_probs(x, t, k, **more)
    a = x.float().cpu().numpy()
    lp, h = R.log_probs(a)
    M, V = a.shape
    with np.errstate(invalid="ignore", over="ignore"):
        z = a.astype(np.float64) - a.max(-1, keepdims=True).astype(np.float64)
        p = np.exp(lp)
        spread = np.where(p > 0, p * np.abs(z), 0.0).sum(-1)
    rel = 2.0 ** -24 * (V / 256 + 50 + 4 * spread)

    def close(got, ref, bound, name):
        got = f64(got)
        # (the lowest logit under the largest one is at twice fp32's range: -infinity in the result's type)
        ref = np.where(np.abs(ref) > np.finfo(np.float32).max, np.sign(ref) * np.inf, ref)
        finite = np.isfinite(ref)
        assert np.array_equal(finite, np.isfinite(got)), (name, got[~finite], ref[~finite])
        assert np.array_equal(got[~finite], ref[~finite], equal_nan=True), (name, got, ref)
        worst = (np.abs(got - ref) - bound)[finite]
        assert worst.size == 0 or worst.max() <= 0, (name, worst.max())

    with np.errstate(invalid="ignore"):
        if targets is not None:
            ts = np.array(targets)
            ref = np.where(ts >= 0, lp[np.arange(M), np.maximum(ts, 0)], 0.0)
            close(logp, ref, rel + 2.0 ** -22 * (1 + np.abs(ref)), "logp")
        else:
            assert logp is None
        if entropy is not None:
            close(entropy, h, (rel + 2.0 ** -22) * (2 + 2 * np.abs(h) + 2 * spread), "entropy")
        if k:
            want = R.top(a, k)
            assert np.array_equal(index.cpu().numpy(), want)
            ref = np.take_along_axis(lp, want, 1)
            close(score, ref, rel[:, None] + 2.0 ** -22 * (1 + np.abs(ref)), "score")
        else:
            assert index is None and score is None
    return logp, entropy, index, score


def logits(M, V, dtype, pad=0, seed=0, spread=3.0):
    g = torch.Generator(device="cuda").manual_seed(seed + M + V)
    return (torch.randn((M, V + pad), generator=g, device="cuda") * spread).to(dtype)[:, :V]


TYPES = [torch.bfloat16, torch.float32]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [1, 2, 7, 8, 64, 65, 511, 1000, 4096, 4097, 8191, 16384, 32000, 50001, 131072, 262143])
def test_vocabularies(V, dtype):
    """Every size of the groups, rows that begin anywhere."""
    for pad in (0, 3):
        for k in {0, 1, min(V, 5), min(V, 20), min(V, 64)}:
            check(logits(7, V, dtype, pad), [0, V - 1, -1, V // 2, V // 3, -1, 0], k)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M", [1, 2, 3, 19, 76, 153, 305, 700])
def test_rows(M, dtype):
    """Rows split over clusters of every size, and whole."""
    check(logits(M, 40000, dtype), [(37 * i) % 40000 for i in range(M)], 20)


def test_largest():
    x = logits(2, 1 << 20, torch.float32)
    check(x, [5, (1 << 20) - 1], 64)
    check(x.bfloat16(), [5, (1 << 20) - 1], 64)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V,k", [(300, 64), (5000, 20), (40000, 64), (100003, 64)])
def test_ties_and_order(V, k, dtype):
    """Equal logits by column: all of them, subnormal ones, few values, sorted both ways, one value more than k times."""
    i = torch.arange(V, device="cuda")
    rows = [torch.zeros(V, device="cuda"), (i % 3).float(), (i % 7 == 6).float() * 5, -(i.float()) / V * 8, i.float() / V * 8,
            torch.where(i >= V - 10, 3.0, 1.0), torch.where(i < k - 1, 9.0, 2.0), torch.where(i % 1000 == 999, 4.0, -4.0),
            i * 1e-40, -(i * 1e-40),  # (less than the smallest normal numbers)
            torch.where(i == V - 1, 0.0, -0.0), torch.where(i % 2 == 0, -0.0, 0.0), (i // 300).float().remainder(11)]
    check(torch.stack(rows).to(dtype), [0] * len(rows), k)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V,k", [(90, 20), (5000, 64), (50001, 20)])
def test_masks(V, k, dtype):
    """Logits of -infinity, of the type's lowest value, and rows that these leave empty or almost."""
    x = logits(12, V, dtype)
    inf, low = float("inf"), torch.finfo(dtype).min
    keep = torch.rand(V, device="cuda", generator=torch.Generator(device="cuda").manual_seed(V)) < 0.01
    x[0, ~keep] = -inf
    x[1] = -inf
    x[2] = -inf
    x[2, V - 1] = 3.0
    x[3, ~keep] = low
    x[4] = low
    x[5] = low
    x[5, 0] = 0.0
    x[6] = -inf
    x[6, 5:9] = low
    x[7, 1:] = -inf
    x[8, :V // 2] = -inf
    x[9] = torch.finfo(dtype).max
    x[10] = low
    x[10, 3] = torch.finfo(dtype).max
    check(x, [0, 0, V - 1, 5, 3, 0, 0, 0, 0, 1, 3, -1], k)
    check(x, [V - 1, 7, 0, V - 2, V - 1, 1, 5, V - 1, 1, 1, 0, 2], 1)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M", [1, 40, 700])
@pytest.mark.parametrize("size", [1e4, 1.2e5, 1.4e5, 3e5, 1e6, 1e9, 1e10, 1e20, 1e30, 3e38])
def test_magnitudes(size, M, dtype):
    """Masks of finite values: where whole runs of logits, as a thread sees them, hold nothing else; whole rows at
    such a value; and logits as large."""
    V = 20000
    x = logits(M, V, dtype)
    kinds = [lambda r: r[2000:].fill_(-size), lambda r: r[:-3].fill_(-size), lambda r: r.fill_(-size),
             lambda r: r[5:].sub_(size), lambda r: r.sub_(size), lambda r: r.add_(size), lambda r: r[777:900].add_(size),
             lambda r: r[3:4].fill_(size), lambda r: r.mul_(size / 8), lambda r: r[::2].fill_(-size)]
    for i in range(M):
        kinds[i % len(kinds)](x[i])
    x.clamp_(torch.finfo(dtype).min, torch.finfo(dtype).max)
    check(x, [(7 * i) % V for i in range(M)], 5)
    check(x[:1].clone(), [3], 64)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V,k", [(90, 20), (5000, 64), (50001, 20)])
def test_nan_and_infinity(V, k, dtype):
    """They stay in their rows; a NaN comes after every number."""
    x = logits(8, V, dtype)
    nan, inf = float("nan"), float("inf")
    x[1, V // 2] = nan
    x[2] = nan
    x[3, 7] = inf
    x[4, :] = inf
    x[5, :-3] = nan
    x[6, ::2] = nan
    x[6, 1] = -inf
    check(x, [0, V // 2, 1, 7, 3, V - 1, 1, 2], k)


@pytest.mark.parametrize("dtype", TYPES)
def test_sure_and_even(dtype):
    """Distributions of almost no and of the largest entropy, and logits that would overflow."""
    x = torch.zeros(6, 30000, device="cuda")
    x[0, 17] = 100.0
    x[1, 17] = 10.0
    x[2] += 80.0
    x[3] = -3000.0
    x[4] = 3000.0
    x[4, 3] = 3001.0
    x[5, :10] = 88.0
    check(x.to(dtype), [17, 17, 4, 5, 3, 29999], 20)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M", [1, 7, 400])
@pytest.mark.parametrize("V,at", [(300, 299), (32000, 17), (50001, 50000), (131072, 70001)])
def test_almost_certain(V, at, M, dtype):
    """One logit far above the others: its log probability is minus the others' sum S, and the entropy about S times
    their distance, each to S's relative error: 2^-22 + 2^-23 |y| of a term (|y| < 64 bits here) and the chain of
    additions of `check`, twice for the function's and the products'."""
    W = _W()
    gaps = [4.0, 6.0, 9.0, 14.0, 20.0, 30.0, 43.0][:M]
    x = logits(M, V, dtype, spread=1.0)
    for i in range(M):
        x[i, at] = x[i].float().logsumexp(0) + gaps[i % len(gaps)]
    x[:, at] = x[:, at].float() + (300.0 if dtype is torch.float32 else 0.0)
    if dtype is torch.float32:
        x[:, :at] += 300.0
        x[:, at + 1:] += 300.0
    t = torch.full((M,), at, dtype=torch.int32, device="cuda")
    logp, entropy, index, score = W.log_probs(x, t, 2)
    a = x.double().cpu().numpy()
    others = np.delete(a - a[:, at:at + 1], at, axis=1)
    S = np.exp(others).sum(1)
    H = np.log1p(S) - (np.exp(others) * others).sum(1) / (1 + S)
    rel = 2 * (2.0 ** -22 + 64 * 2.0 ** -23 + (V / 256 + 50) * 2.0 ** -24)
    assert (np.abs(f64(logp) + np.log1p(S)) <= rel * S).all()
    assert (np.abs(f64(entropy) - H) <= 2 * rel * H).all()
    assert (index[:, 0] == at).all() and torch.equal(score[:, 0], logp)


def test_bad_targets():
    W = _W()
    x = logits(4, 1000, torch.bfloat16)
    for bad in (1000, -2, 2 ** 31 - 1):
        t = torch.tensor([5, bad, -1, 7], dtype=torch.int32, device="cuda")
        logp, entropy, _, _ = W.log_probs(x, t)
        assert W.get_device_error() == W.ERR_INVALID_ARG
        assert logp[1] == 0 and logp[2] == 0
    check(x, [5, 0, -1, 7])
    assert W.get_device_error() == W.OK


def test_what_is_not_asked_for():
    W = _W()
    x = logits(5, 777, torch.float32)
    assert W.log_probs(x, k=3, entropy=False)[:2] == (None, None)
    check(x, None, 3)
    check(x, [1, 2, 3, 4, 5], 0, entropy=False)


def test_one_row_of_many_and_strides():
    """Rows of a wider tensor, and one row alone."""
    wide = logits(9, 4099, torch.bfloat16, pad=61)
    check(wide[3:4], [4], 5)
    W = _W()
    with pytest.raises((ValueError, W.W4A16Error)):
        W.log_probs(wide.t())


def test_same_bits_and_graphs():
    W = _W()
    x = logits(5, 50001, torch.bfloat16, pad=3)
    t = torch.tensor([1, 2, -1, 4, 50000], dtype=torch.int32, device="cuda")
    want = check(x, t.tolist(), 20)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = W.log_probs(x, t, 20, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = W.log_probs(x, t, 20)
    for _ in range(3):
        for a in got:
            a.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
