"""Residual norms against 64 bits.

Bounds: h is rounded once (half a step: 2^-8 of it in bf16, 2^-24 in fp32) from sums of two products in
fp32; out is rounded once.  A mean of squares is a sum of at most 128 terms in a row in a thread and 9 joins
over threads, so 1 / sqrt(..) is within 2^-17 of its value, with the 2 steps of the function; an error of
h moves out by its own size, by its mean and, through the mean square, by its root mean square."""
import itertools

import numpy as np
import pytest
import torch

from tests import layer_reference as R

pytestmark = pytest.mark.gpu
EPS = 1e-5
ROOT = 2.0 ** -17


def _W():
    from paper_2608_30877_gb300 import w4a16 as W
    return W


def f64(t):
    return t.detach().double().cpu().numpy()


def reference(residual, block, weight, bias, gate, post_weight, post_bias, layer, eps, offset, scale):
    """(out, h) and their bounds before the stores' rounding."""
    r = f64(residual)
    stream = 2.0 ** -23 * np.abs(scale * r)
    h = scale * r
    err = stream
    if block is not None:
        b = f64(block)
        berr = np.zeros_like(b)
        if post_weight is not None:
            w, wb = offset + f64(post_weight), 0.0 if post_bias is None else f64(post_bias)
            b = R.norm(b, layer, eps, w, 0.0)
            berr = ROOT * np.abs(b) + 2.0 ** -22 * (np.abs(b) + np.abs(wb))
            if layer:  # the mean's own error, a sum's of magnitudes
                v = f64(block)
                berr += ROOT * np.abs(v).mean(-1, keepdims=True) / np.sqrt(v.var(-1, keepdims=True) + eps) * np.abs(w)
            b = b + wb
        g = 1.0 if gate is None else f64(gate)
        h = h + g * b
        err = stream + np.abs(g) * berr + 2.0 ** -22 * np.abs(g * b)
    f = (1.0 if weight is None else offset + f64(weight))
    c = h - h.mean(-1, keepdims=True) if layer else h
    rstd = 1.0 / np.sqrt((c * c).mean(-1, keepdims=True) + eps)
    mean_err = (err + ROOT * np.abs(h)).mean(-1, keepdims=True) if layer else 0.0
    out = c * rstd * f
    moved = np.sqrt(((err + mean_err) ** 2).mean(-1, keepdims=True)) * rstd + ROOT + 2.0 ** -21
    out_err = rstd * np.abs(f) * (err + mean_err) + np.abs(out) * moved
    if bias is not None:
        out = out + f64(bias)
        out_err = out_err + 2.0 ** -22 * np.abs(f64(bias))
    return (out, h), (out_err, err)


def inputs(M, D, bits, block, gate, post, bias, weight=True, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + M * 7 + D)
    rnd = lambda *s, k=1.0: (torch.randn(s, generator=g, device="cuda") * k).bfloat16()  # noqa: E731
    residual = rnd(M, D, k=3.0) if bits == 16 else torch.randn((M, D), generator=g, device="cuda") * 3
    residual[:, ::max(1, D // 3)] *= 40
    return dict(residual=residual, block=rnd(M, D) if block else None, weight=rnd(D, k=0.3) if weight else None,
                bias=rnd(D, k=0.3) if bias else None, gate=rnd(1 if gate == 1 else M, D) if gate else None,
                post_weight=rnd(D, k=0.3) if post else None, post_bias=rnd(D, k=0.3) if post and bias else None)


def check(given, layer=False, eps=EPS, offset=1.0, scale=1.0, **more):
    W = _W()
    refs, errs = reference(**given, layer=layer, eps=eps, offset=offset, scale=scale)
    out, h = W.residual_norm(given["residual"], given["weight"], given["block"], bias=given["bias"], gate=given["gate"],
                             post_weight=given["post_weight"], post_bias=given["post_bias"],
                             kind=W.NORM_LAYER if layer else W.NORM_RMS, eps=eps, weight_offset=offset,
                             residual_scale=scale, **more)
    for name, got, ref, err in zip(("out", "h"), (out, h), refs, errs):
        if got is None:
            continue
        half = 2.0 ** -8 if got.dtype == torch.bfloat16 else 2.0 ** -24
        worst = (np.abs(f64(got) - ref) - half * np.abs(ref) - (1 + half) * err - 1e-38).max()
        assert worst <= 0, (name, worst, np.abs(f64(got) - ref).max())
    return out, h


WIDTHS = [1, 7, 8, 64, 100, 255, 256, 1000, 1016, 1024, 1025, 1032, 2047, 4096, 8193, 12288, 16392, 24560, 32768, 32775, 49151, 49152]


@pytest.mark.parametrize("D", WIDTHS)
@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("bits", [16, 32])
def test_widths(D, layer, bits):
    """Every number of pieces of a row, rows that begin anywhere in a 16-byte unit."""
    for M in (1, 9):
        check(inputs(M, D, bits, True, 0, False, False), layer)
        check(inputs(M, D, bits, True, 1, True, True), layer, scale=0.5)
        check(inputs(M, D, bits, False, 0, False, True), layer)


@pytest.mark.parametrize("M,D", [(1, 4096), (2, 40), (17, 515), (300, 1024), (1000, 130), (2000, 2560), (40, 12288)])
def test_every_part(M, D):
    for block, gate, post, bias, bits, layer in itertools.product((True, False), (0, 1, -1), (False, True), (False, True), (16, 32),
                                                                  (False, True)):
        if not block and (gate or post):
            continue
        check(inputs(M, D, bits, block, gate, post, bias), layer, offset=0.0 if gate == 1 else 1.0, scale=1.0 if bias else -0.7)


@pytest.mark.parametrize("bits", [16, 32])
@pytest.mark.parametrize("D", [96, 515, 12288])
def test_in_place_and_given_outputs(bits, D):
    W = _W()
    given = inputs(33, D, bits, True, 1, True, False)
    want_out, want_h = check(given)
    args = dict(gate=given["gate"], post_weight=given["post_weight"], weight_offset=1.0)
    x = given["residual"].clone()
    out = torch.full_like(want_out, 7)
    got_out, got_h = W.residual_norm(x, given["weight"], given["block"], residual_out=x, out=out, **args)
    assert got_h is x and got_out is out
    assert torch.equal(x, want_h) and torch.equal(out, want_out)
    # only the stream
    rc = W.lib().w4a16_residual_norm(given["residual"].data_ptr(), bits, given["block"].data_ptr(), given["gate"].data_ptr(), 1,
                                     given["post_weight"].data_ptr(), None, None, None, 33, D, 0, 1.0, EPS, 1.0, x.zero_().data_ptr(),
                                     None, W._stream(None))
    assert rc == W.OK and torch.equal(x, want_h)


def test_no_weight_and_plain_norm():
    W = _W()
    check(inputs(5, 200, 16, False, 0, False, False, weight=False))
    x = inputs(5, 200, 16, False, 0, False, False)["residual"]
    out, h = W.residual_norm(x)
    assert h is x
    out, h = W.residual_norm(x, residual_scale=0.5)
    assert h is None


def test_rows_do_not_touch_each_other():
    """NaN and infinities stay in their rows; columns at an odd row's ends stay with their rows."""
    W = _W()
    for D in (37, 1029, 4096, 12289):
        given = inputs(12, D, 16, True, 0, False, False)
        want = W.residual_norm(given["residual"], given["weight"], given["block"])
        given["block"][3, D // 2] = float("nan")
        given["residual"][7, 0] = float("inf")
        got = W.residual_norm(given["residual"], given["weight"], given["block"])
        for w, g in zip(want, got):
            keep = [i for i in range(12) if i not in (3, 7)]
            assert torch.equal(w[keep], g[keep])
        assert got[0][3].isnan().all()
        assert got[0][7, 0].isnan() and (got[0][7, 1:] == 0).all()
        assert got[1][7, 0] == float("inf") and got[1][3, D // 2].isnan()


@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("size", [1e-30, 1e-12, 1e15, 1e19, 1e25, 3e37])
def test_sizes(layer, size):
    """Squares that overflow or vanish."""
    for D in (64, 515, 12288):
        given = inputs(4, D, 32, False, 0, False, False)
        given["residual"] = torch.randn(4, D, generator=torch.Generator(device="cuda").manual_seed(D), device="cuda") * size / 4
        check(given, layer)


def test_zero_rows_and_single_columns():
    W = _W()
    x = torch.zeros(3, 512, device="cuda", dtype=torch.bfloat16)
    out, _ = W.residual_norm(x)
    assert (out == 0).all()
    x = torch.full((3, 1), 5.0, device="cuda", dtype=torch.bfloat16)
    assert (W.residual_norm(x, kind=W.NORM_LAYER)[0] == 0).all()
    assert (W.residual_norm(x)[0] == 1).all()


def test_offset_rows():
    """A layer norm of values far from zero: the variance is not a difference of large sums."""
    given = inputs(6, 4096, 32, False, 0, False, True)
    given["residual"] = 1000.0 + torch.randn(6, 4096, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    check(given, layer=True)


def test_other_streams_and_graphs():
    W = _W()
    given = inputs(64, 4096, 16, True, 1, True, True)
    want = check(given)
    args = dict(bias=given["bias"], gate=given["gate"], post_weight=given["post_weight"], post_bias=given["post_bias"],
                weight_offset=1.0)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = W.residual_norm(given["residual"], given["weight"], given["block"], stream=side, **args)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = W.residual_norm(given["residual"], given["weight"], given["block"], **args)
    for _ in range(3):
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
