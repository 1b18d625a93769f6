"""Refusals of the operators around the linears before anything is launched, and the rotary frequencies,
which are host work (no GPU needed)."""
import ctypes
import math

import pytest
import torch

from paper_2608_30877_gb300 import w4a16 as W
from tests import layer_reference as R
from tests.test_kv_abi import BAD_CACHES, cache

A = 1 << 40  # fake, 16-byte aligned "device" addresses, far apart (never dereferenced)
BAD, UNSUPPORTED, ALIGNMENT = W.ERR_INVALID_ARG, W.ERR_UNSUPPORTED, W.ERR_ALIGNMENT


@pytest.fixture(scope="module")
def L():
    from paper_2608_30877_gb300 import build as B
    B.build()
    return W.lib()


def call(f, given, change):
    args = dict(given)
    assert set(change) <= set(args)
    args.update(change)
    return f(*args.values(), None)


NORM = dict(residual=A, bits=16, block=2 * A, gate=3 * A, gate_rows=1, post_weight=4 * A, post_bias=5 * A, weight=6 * A,
            bias=7 * A, M=4, D=256, norm=0, scale=1.0, eps=1e-5, offset=0.0, residual_out=8 * A, out=9 * A)


@pytest.mark.parametrize("change,want", [
    (dict(residual=None), BAD), (dict(bits=8), BAD), (dict(bits=64), BAD), (dict(norm=2), BAD), (dict(norm=-1), BAD),
    (dict(M=0), BAD), (dict(M=-1), BAD), (dict(D=0), BAD), (dict(gate_rows=2), BAD), (dict(gate_rows=0), BAD),
    (dict(eps=0.0), BAD), (dict(eps=-1e-5), BAD), (dict(eps=1e-13), BAD), (dict(eps=2.0), BAD), (dict(eps=math.nan), BAD),
    (dict(scale=math.inf), BAD), (dict(scale=math.nan), BAD), (dict(offset=math.nan), BAD),
    (dict(residual_out=None, out=None), BAD), (dict(block=None), BAD), (dict(block=None, gate=None), BAD),
    (dict(post_weight=None), BAD), (dict(out=None), BAD),
    (dict(M=1 << 31), UNSUPPORTED), (dict(D=49153), UNSUPPORTED),
    *((dict([(n, NORM[n] + 8)]), ALIGNMENT) for n in ("residual", "block", "gate", "post_weight", "post_bias", "weight",
                                                     "bias", "residual_out", "out")),
    (dict(residual_out=A + 16), BAD), (dict(out=A + 16), BAD), (dict(out=A), BAD), (dict(out=8 * A + 16), BAD),
    (dict(out=2 * A), BAD), (dict(residual_out=2 * A + 2032), BAD), (dict(out=6 * A), BAD), (dict(out=3 * A + 496), BAD),
    (dict(bits=32, residual_out=A + 4080), BAD),
])
def test_norm_arguments(L, change, want):
    assert call(L.w4a16_residual_norm, NORM, change) == want


ROTARY = dict(qkv=A, seq_start=2 * A, first=3 * A, nseq=3, M=10, H=8, kv_heads=2, d=128, turns=4 * A, rot=64, layout=0,
              factor=1.0)


@pytest.mark.parametrize("change,want", [
    (dict(qkv=None), BAD), (dict(turns=None), BAD), (dict(nseq=0), BAD), (dict(M=0), BAD), (dict(H=-1), BAD),
    (dict(kv_heads=-1), BAD), (dict(H=0, kv_heads=0), BAD), (dict(rot=0), BAD), (dict(rot=144), BAD), (dict(layout=2), BAD),
    (dict(factor=math.inf), BAD), (dict(seq_start=None), BAD),
    (dict(rot=24), UNSUPPORTED), (dict(d=100), UNSUPPORTED), (dict(d=512, rot=272), UNSUPPORTED), (dict(M=1 << 31), UNSUPPORTED),
    (dict(H=65536), UNSUPPORTED), (dict(H=60000, d=65536), UNSUPPORTED), (dict(nseq=1 << 30), UNSUPPORTED),
    (dict(qkv=A + 8), ALIGNMENT), (dict(seq_start=2 * A + 4), ALIGNMENT), (dict(first=3 * A + 4), ALIGNMENT),
    (dict(turns=4 * A + 8), ALIGNMENT), (dict(first=A + 16), BAD), (dict(turns=A + 25600 * 1 - 16), BAD),
])
def test_rotary_arguments(L, change, want):
    assert call(L.w4a16_rotary, ROTARY, change) == want


KV_ROTARY = dict(qkv=11 * A, seq_start=12 * A, slots=13 * A, nseq=3, M=10, H=8, turns=14 * A, rot=64, layout=1, factor=1.0)


@pytest.mark.parametrize("change,want", [
    (dict(qkv=None), BAD), (dict(turns=None), BAD), (dict(slots=None), BAD), (dict(nseq=0), BAD), (dict(M=0), BAD),
    (dict(H=-1), BAD), (dict(rot=0), BAD), (dict(rot=144), BAD), (dict(layout=-1), BAD), (dict(factor=math.nan), BAD),
    (dict(seq_start=None), BAD), (dict(rot=40), UNSUPPORTED), (dict(M=(1 << 31) - 1), UNSUPPORTED),
    (dict(H=65536), UNSUPPORTED), (dict(qkv=11 * A + 2), ALIGNMENT), (dict(turns=14 * A + 4), ALIGNMENT),
    (dict(slots=13 * A + 4), ALIGNMENT), (dict(qkv=A), BAD), (dict(slots=3 * A), BAD), (dict(turns=11 * A + 16), BAD),
])
def test_kv_rotary_arguments(L, change, want):
    assert call(lambda *a: L.w4a16_kv_rotary(ctypes.byref(cache()), *a), KV_ROTARY, change) == want


@pytest.mark.parametrize("change,want", BAD_CACHES)
def test_kv_rotary_refuses_bad_caches(L, change, want):
    assert call(lambda *a: L.w4a16_kv_rotary(ctypes.byref(cache(**change)), *a), KV_ROTARY, {}) == want


LOGPROBS = dict(logits=A, bits=16, M=4, V=1000, stride=1000, targets=2 * A, k=5, logp=3 * A, entropy=4 * A, index=5 * A,
                score=6 * A)


@pytest.mark.parametrize("change,want", [
    (dict(logits=None), BAD), (dict(bits=8), BAD), (dict(M=0), BAD), (dict(V=0), BAD), (dict(stride=999), BAD),
    (dict(k=-1), BAD), (dict(V=4, k=5), BAD), (dict(targets=None), BAD), (dict(logp=None), BAD), (dict(index=None), BAD),
    (dict(score=None), BAD), (dict(k=0), BAD),
    (dict(targets=None, logp=None, entropy=None, k=0, index=None, score=None), BAD),
    (dict(k=65), UNSUPPORTED), (dict(V=(1 << 20) + 1, stride=1 << 21), UNSUPPORTED), (dict(M=1 << 28), UNSUPPORTED),
    (dict(stride=1 << 31), UNSUPPORTED),
    *((dict([(n, LOGPROBS[n] + 4)]), ALIGNMENT) for n in ("logits", "targets", "logp", "entropy", "index", "score")),
    (dict(logp=A + 16), BAD), (dict(score=5 * A + 64), BAD), (dict(entropy=3 * A), BAD), (dict(index=2 * A), BAD),
    (dict(entropy=A + 7984), BAD),
])
def test_log_probs_arguments(L, change, want):
    assert call(L.w4a16_log_probs, LOGPROBS, change) == want


ADAPTERS = dict(x=A, a=2 * A, b=3 * A, scale=4 * A, pool=3, seq_start=5 * A, ids=6 * A, nseq=2, M=10, N=100, K=128, R=16,
                base=7 * A, out=8 * A, workspace=9 * A)


@pytest.mark.parametrize("change,want", [
    *((dict([(n, None)]), BAD) for n in ("x", "a", "b", "scale", "ids", "base", "out", "workspace")),
    (dict(seq_start=None), BAD), (dict(pool=0), BAD), (dict(nseq=0), BAD), (dict(M=0), BAD), (dict(N=0), BAD),
    (dict(K=0), BAD), (dict(R=0), BAD), (dict(K=100), UNSUPPORTED), (dict(K=32), UNSUPPORTED), (dict(R=12), UNSUPPORTED),
    *((dict([(n, ADAPTERS[n] + 8)]), ALIGNMENT) for n in ("x", "a", "b", "scale", "seq_start", "ids", "base", "out", "workspace")),
    (dict(out=A + 16), BAD), (dict(out=7 * A + 16), BAD), (dict(workspace=8 * A + 1984), BAD), (dict(out=3 * A), BAD),
    (dict(workspace=6 * A), BAD), (dict(R=72), UNSUPPORTED), (dict(M=1 << 26), UNSUPPORTED), (dict(N=1 << 26), UNSUPPORTED), (dict(pool=1 << 26), UNSUPPORTED),
])
def test_adapters_arguments(L, change, want):
    assert call(L.w4a16_add_adapters, ADAPTERS, change) == want


def test_adapters_workspace(L):
    assert L.w4a16_add_adapters_workspace(4, 16) == 128
    for M, R in ((0, 16), (4, 0), (4, 12), (4, 72), (1 << 26, 16)):
        assert L.w4a16_add_adapters_workspace(M, R) == 0


@pytest.mark.parametrize("change,want", [
    (dict(rot=0), BAD), (dict(rot=-16), BAD), (dict(base=0.5), BAD), (dict(base=math.inf), BAD), (dict(base=math.nan), BAD),
    (dict(scaling=4), BAD), (dict(scaling=-1), BAD), (dict(factor=0.5), BAD), (dict(factor=math.nan), BAD),
    (dict(trained=0), BAD), (dict(low=0.0), BAD), (dict(low=40.0), BAD), (dict(high=math.inf), BAD),
    (dict(base=1.0), BAD), (dict(turns=None), BAD), (dict(rot=24), UNSUPPORTED), (dict(rot=272), UNSUPPORTED),
])
def test_rotary_table_arguments(L, change, want):
    host = (ctypes.c_uint64 * 200)()
    given = dict(rot=64, base=10000.0, scaling=W.ROTARY_SCALE_BY_INDEX, factor=4.0, trained=4096, low=1.0, high=32.0, turns=host)
    given.update(change)
    assert L.w4a16_rotary_table(*given.values()) == want


@pytest.mark.parametrize("rot", [16, 64, 96, 128, 256])
@pytest.mark.parametrize("scaling,factor,low,high", [
    (W.ROTARY_SCALE_NONE, 1.0, 1.0, 32.0), (W.ROTARY_SCALE_LINEAR, 4.0, 1.0, 32.0), (W.ROTARY_SCALE_BY_TURNS, 8.0, 1.0, 4.0),
    (W.ROTARY_SCALE_BY_TURNS, 8.0, 0.5, 1000.0), (W.ROTARY_SCALE_BY_INDEX, 32.0, 1.0, 32.0), (W.ROTARY_SCALE_BY_INDEX, 2.0, 3.0, 3.5)])
@pytest.mark.parametrize("base,trained", [(10000.0, 4096), (500000.0, 8192), (1.5, 100)])
def test_rotary_frequencies(L, rot, scaling, factor, low, high, base, trained):
    """Turns per token within a few 2^-52 of the formula's, which 64-bit floating point gives: a power, a
    logarithm, and a handful of products."""
    host = (ctypes.c_uint64 * (rot // 2))()
    assert L.w4a16_rotary_table(rot, base, scaling, factor, trained, low, high, host) == W.OK
    for i in range(rot // 2):
        want = R.frequency(rot, i, base, scaling, factor, trained, low, high) / math.tau
        assert abs(host[i] / 2.0 ** 64 - want) <= 64 * 2.0 ** -53 * want + 2.0 ** -64, (i, host[i])


def test_binding_refuses_what_it_can_see():
    """CPU tensors, wrong types and shapes: an error before the library is asked."""
    t = torch.zeros(4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        W.residual_norm(t)
    with pytest.raises(ValueError):
        W.log_probs(t)
    with pytest.raises(ValueError):
        W.add_adapters(t, t, t.view(1, 4, 64), t.view(1, 64, 4), torch.ones(1), torch.zeros(4, dtype=torch.int32))
    with pytest.raises(ValueError):
        W.RotaryTable(64, layout=7)
    with pytest.raises(W.W4A16Error):
        W.RotaryTable(20, device="cpu")
    table = W.RotaryTable(64, device="cpu")
    with pytest.raises(ValueError):
        W.rotary(torch.zeros(4, 3 * 128, dtype=torch.bfloat16), table, 1)
