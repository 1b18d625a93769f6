"""The operators around the linears at their limits: offsets past 2^31, waits that run out, calls on two streams
at once, two captured graphs, and the debug build's index checks."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from tests import layer_reference as R
from tests import test_gpu_residual_norm as RN
from tests import test_gpu_rotary as RO
from tests.kv_reference import i32

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
f64 = RN.f64


def _W():
    from paper_2608_30877_gb300 import w4a16 as W
    return W


def _rows(M, width):
    """The first, those around 2^31 elements and bytes, and the last."""
    return sorted({0, *(r + d for r in (2 ** 30 // width, 2 ** 31 // width) for d in (-1, 0, 1) if r + d < M), M - 1})


def _bf16(*shape, scale=1.0, seed=0):
    t = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    t.normal_(generator=torch.Generator(device="cuda").manual_seed(seed))
    return t.mul_(scale) if scale != 1.0 else t


@pytest.mark.parametrize("layer", [False, True])
def test_norm_past_2_31_elements(layer):
    W = _W()
    M, D = 180001, 12288
    residual, block, weight = _bf16(M, D, scale=3.0, seed=1), _bf16(M, D, seed=2), _bf16(D, scale=0.3, seed=3)
    out, h = W.residual_norm(residual, weight, block, kind=W.NORM_LAYER if layer else W.NORM_RMS, weight_offset=1.0)
    at = torch.tensor(_rows(M, D), device="cuda")
    refs, errs = RN.reference(residual[at], block[at], weight, None, None, None, None, layer, 1e-5, 1.0, 1.0)
    for got, ref, err in zip((out[at], h[at]), refs, errs):
        assert (np.abs(f64(got) - ref) <= 2.0 ** -8 * np.abs(ref) + 1.01 * err).all()


def test_rotary_past_2_31_elements():
    W = _W()
    M, H = 60001, 96
    qkv = _bf16(M, 3 * H * 128, seed=4)
    at = torch.tensor(_rows(M, 3 * H * 128), device="cuda")
    before = qkv[at].clone()
    W.rotary(qkv, W.RotaryTable(128), H, seq_start=i32([0, 1000, M]))
    RO.check(before, qkv[at], H, H, 128, [r if r < 1000 else r - 1000 for r in at.tolist()], RO.theta_of(128), False)


def test_log_probs_past_2_31_elements():
    W = _W()
    M, V = 17001, 131072
    x = _bf16(M, V, scale=2.0, seed=5)
    targets = torch.arange(M, device="cuda", dtype=torch.int32) * 7
    logp, entropy, index, score = W.log_probs(x, targets, 5)
    for r in _rows(M, V):
        a = x[r:r + 1].float().cpu().numpy()
        lp, h = R.log_probs(a)
        top = R.top(a, 5)[0]
        assert index[r].tolist() == top.tolist()
        bound = 2.0 ** -24 * (V / 256 + 250)
        assert abs(logp[r].item() - lp[0, 7 * r]) <= bound * 16 and abs(entropy[r].item() - h[0]) <= bound * 16
        assert np.abs(f64(score[r]) - lp[0, top]).max() <= bound * 16


def _adapters_close(got, x, base, A, B, scale, ids, K):
    ref, size = R.adapters(*(f64(t) for t in (x, base)), A, B, scale, ids)
    t = np.array([np.abs(B[a]) @ np.abs(scale[a] * (A[a] @ f64(x)[m])) for m, a in enumerate(ids)])
    bound = 2.0 ** -8 * np.abs(ref) + 1.01 * 2.0 ** -8 * t + 2.0 ** -22 * ((K / 64 + 40) * size + 8 * np.abs(f64(base)))
    assert (np.abs(f64(got) - ref) <= bound).all()


@pytest.mark.parametrize("packed", [False, True])
def test_adapters_past_2_31_elements(packed):
    """Of base and out, and of the pool."""
    W = _W()
    M, N, K, rank = 60001, 36864, 64, 16
    x, base = _bf16(M, K, seed=6), _bf16(M, N, seed=7)
    A, B, scale = _bf16(3, rank, K, scale=0.1, seed=8), _bf16(3, N, rank, scale=0.3, seed=9), torch.ones(3, device="cuda")
    ids = [0, 2, 1] if packed else [i % 3 for i in range(M)]
    starts = [0, 100, 58250, M] if packed else None
    out = W.add_adapters(base, x, A, B, scale, i32(ids), seq_start=i32(starts) if packed else None)
    rows = _rows(M, N)
    of = [next(a for a, e in zip(ids, starts[1:]) if r < e) for r in rows] if packed else [ids[r] for r in rows]
    at = torch.tensor(rows, device="cuda")
    _adapters_close(out[at], x[at], base[at], f64(A), f64(B), f64(scale), of, K)
    del x, base, out
    torch.cuda.empty_cache()
    pool, N, K, rank, M = 1500, 100, 24576, 64, 70
    A, B, scale = _bf16(pool, rank, K, scale=K ** -0.5, seed=10), _bf16(pool, N, rank, seed=11), torch.ones(pool, device="cuda")
    x, base = _bf16(M, K, seed=12), _bf16(M, N, seed=13)
    ids = [pool - 1, 0, 1365] if packed else [pool - 1 - 5 * i for i in range(M)]
    starts = [0, 30, 50, M] if packed else None
    out = W.add_adapters(base, x, A, B, scale, i32(ids), seq_start=i32(starts) if packed else None)
    rows = [0, 40, 69] if packed else [0, 1, 69]
    at = torch.tensor(rows, device="cuda")
    of = ids if packed else [ids[r] for r in rows]
    used = torch.tensor(of, device="cuda")
    _adapters_close(out[at], x[at], base[at], f64(A[used]), f64(B[used]), f64(scale[used]), [0, 1, 2], K)
    assert W.get_device_error() == W.OK


def test_waits_that_run_out():
    """With a lowered limit the kernels that wait for their copies give up, say so, and the next call is right."""
    W = _W()
    residual, block = torch.randn(3000, 4096, device="cuda"), _bf16(3000, 4096)
    x, base = _bf16(2000, 512), _bf16(2000, 640)
    A, B, scale = _bf16(2, 32, 512, scale=0.1), _bf16(2, 640, 32, scale=0.1), torch.ones(2, device="cuda")
    norm = lambda: W.residual_norm(residual, None, block)  # noqa: E731
    adapters = lambda: (W.add_adapters(base, x, A, B, scale, i32([0, 1]), seq_start=i32([0, 900, 2000])),)  # noqa: E731
    for call in (norm, adapters):
        want = call()
        W.set_wait_limit(1)
        try:
            call()
            assert W.get_device_error() == W.ERR_TIMEOUT
        finally:
            W.set_wait_limit(0)
        got = call()
        assert W.get_device_error() == W.OK
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_two_streams_and_two_graphs():
    """Calls at the same time, each with its own outputs and workspace, from the host and as graphs."""
    W = _W()
    x, base = _bf16(300, 2048), _bf16(300, 4096)
    A, B, scale = _bf16(4, 16, 2048, scale=0.1), _bf16(4, 4096, 16, scale=0.1), torch.ones(4, device="cuda")
    lists = [i32([i % 4 for i in range(300)]), i32([(i // 7) % 4 for i in range(300)])]
    logits = _bf16(300, 20000, scale=2.0)
    calls = [lambda k=k: (W.add_adapters(base, x, A, B, scale, lists[k]), *W.log_probs(logits[k:], None, 10)[1:],
                          *W.residual_norm(base[k:], None, base[:300 - k])) for k in (0, 1)]
    want = [f() for f in calls]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        got = []
        for f, s in zip(calls, streams):
            with torch.cuda.stream(s):
                got.append(f())
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for g, w in zip(got, want) for a, b in zip(g, w))
    graphs, outs = [torch.cuda.CUDAGraph() for _ in range(2)], []
    for g, f in zip(graphs, calls):
        with torch.cuda.graph(g):
            outs.append(f())
    for _ in range(5):
        for o in outs:
            for t in o:
                t.zero_()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for g, w in zip(outs, want) for a, b in zip(g, w))


_CHILD = r"""
import sys
sys.path.insert(0, {root!r})
import torch
from paper_2608_30877_gb300 import w4a16 as W
assert W.LIB_PATH.endswith("libw4a16_debug.so"), W.LIB_PATH
from tests import test_gpu_adapters as A, test_gpu_log_probs as L, test_gpu_residual_norm as N, test_gpu_rotary as Y
N.test_every_part(300, 1024)
N.test_every_part(17, 515)
N.test_widths(49151, True, 32)
N.test_widths(8193, False, 16)
given = N.inputs(2000, 4096, 32, True, -1, True, True)
N.check(given, True)
for pairs in (False, True):
    Y.test_heads(128, 96, pairs)
    Y.test_packed([0, 0, 1, 1, 40, 41], pairs)
    Y.test_of_a_cache(pairs)
for dtype in L.TYPES:
    L.test_ties_and_order(40000, 64, dtype)
    L.test_vocabularies(50001, dtype)
    L.test_masks(5000, 64, dtype)
for rank in (8, 40, 64):
    A.test_a_row_each(40, rank)
    A.test_packed([0, 7, 8, 9, 63, 64, 65, 200], rank)
assert W.get_device_error() == W.OK
print("ok")
"""


def test_debug_build():
    from paper_2608_30877_gb300 import build as B
    B.build(debug=True)
    r = subprocess.run([sys.executable, "-c", _CHILD.format(root=ROOT)], env=dict(os.environ, W4A16_DEBUG="1"),
                       capture_output=True, text=True, timeout=600)
    assert r.returncode == 0 and "ok" in r.stdout, r.stdout[-3000:] + r.stderr[-3000:]
