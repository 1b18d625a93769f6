"""Refusals of the key-value cache's entry points before anything is launched (no GPU
needed): bad sizes, types, alignment and overlaps."""
import ctypes

import pytest

from paper_2608_30877_gb300 import w4a16 as W

A = 1 << 40  # fake, 16-byte aligned "device" addresses, far apart (never dereferenced)


@pytest.fixture(scope="module")
def L():
    from paper_2608_30877_gb300 import build as B
    B.build()
    return W.lib()


def cache(**change):
    f = dict(pages=A, exponents=None, page_table=2 * A, seq_len=3 * A, page_refs=4 * A, scratch=5 * A,
             layers=2, num_pages=100, kv_heads=4, page_tokens=16, head_dim=128, num_slots=8, max_pages=10,
             kv_bits=16)
    f.update(change)
    return W.KVCacheStruct(*(f[n] for n, _ in W.KVCacheStruct._fields_))


BAD_CACHES = [
    (dict(pages=None), W.ERR_INVALID_ARG), (dict(page_table=None), W.ERR_INVALID_ARG),
    (dict(seq_len=None), W.ERR_INVALID_ARG), (dict(page_refs=None), W.ERR_INVALID_ARG),
    (dict(scratch=None), W.ERR_INVALID_ARG), (dict(layers=0), W.ERR_INVALID_ARG),
    (dict(num_pages=-1), W.ERR_INVALID_ARG), (dict(kv_heads=0), W.ERR_INVALID_ARG),
    (dict(num_slots=0), W.ERR_INVALID_ARG), (dict(max_pages=0), W.ERR_INVALID_ARG),
    (dict(kv_bits=4), W.ERR_INVALID_ARG), (dict(kv_bits=8), W.ERR_INVALID_ARG),
    (dict(exponents=6 * A), W.ERR_INVALID_ARG), (dict(head_dim=64), W.ERR_UNSUPPORTED),
    (dict(page_tokens=8), W.ERR_UNSUPPORTED), (dict(page_tokens=48), W.ERR_UNSUPPORTED),
    (dict(page_tokens=256), W.ERR_UNSUPPORTED), (dict(num_slots=65537), W.ERR_UNSUPPORTED),
    (dict(num_pages=(1 << 24) + 1), W.ERR_UNSUPPORTED),
    (dict(num_pages=1 << 24, kv_heads=4), W.ERR_UNSUPPORTED),  # 2^31 rows a layer
    (dict(max_pages=1 << 28), W.ERR_UNSUPPORTED), (dict(num_slots=65536, max_pages=1 << 15), W.ERR_UNSUPPORTED),
    (dict(page_table=2 * A + 4), W.ERR_ALIGNMENT),
    (dict(seq_len=4 * A + 16), W.ERR_INVALID_ARG),  # inside page_refs
]


@pytest.mark.parametrize("change,want", BAD_CACHES)
def test_bad_caches(L, change, want):
    c = ctypes.byref(cache(**change))
    assert L.w4a16_kv_extend(c, 7 * A, 8 * A, 2, None) == want
    assert L.w4a16_kv_fork(c, 7 * A, 8 * A, 2, None) == want
    assert L.w4a16_kv_trim(c, 7 * A, None, 2, None) == want
    assert L.w4a16_kv_compact(c, None) == want
    assert L.w4a16_kv_write(c, 0, 7 * A, 8 * A, 9 * A, 2, 4, 4, None) == want
    assert L.w4a16_attention_decode(c, 0, 7 * A, 8 * A, 2, 4, 100, 9 * A, 10 * A, None) == want


def test_null_cache(L):
    assert L.w4a16_kv_compact(None, None) == W.ERR_INVALID_ARG
    assert L.w4a16_kv_trim(None, 7 * A, None, 2, None) == W.ERR_INVALID_ARG


def test_page_lists(L):
    c = ctypes.byref(cache())
    for f in (L.w4a16_kv_extend, L.w4a16_kv_fork, L.w4a16_kv_trim):
        assert f(c, None, 8 * A, 2, None) == W.ERR_INVALID_ARG
        assert f(c, 7 * A, 8 * A, 0, None) == W.ERR_INVALID_ARG
        assert f(c, 7 * A, 8 * A, 9, None) == W.ERR_INVALID_ARG      # more than the slots
        assert f(c, 7 * A + 4, 8 * A, 2, None) == W.ERR_ALIGNMENT
        assert f(c, 7 * A, 3 * A, 2, None) == W.ERR_INVALID_ARG      # in seq_len
        assert f(c, 2 * A + 16, 8 * A, 2, None) == W.ERR_INVALID_ARG  # in the table
    assert L.w4a16_kv_extend(c, 7 * A, None, 2, None) == W.ERR_INVALID_ARG
    assert L.w4a16_kv_fork(c, 7 * A, None, 2, None) == W.ERR_INVALID_ARG


@pytest.mark.parametrize("args,want", [
    ((-1, 7 * A, 8 * A, 9 * A, 2, 4, 4), W.ERR_INVALID_ARG), ((2, 7 * A, 8 * A, 9 * A, 2, 4, 4), W.ERR_INVALID_ARG),
    ((0, None, 8 * A, 9 * A, 2, 4, 4), W.ERR_INVALID_ARG), ((0, 7 * A, None, 9 * A, 2, 4, 4), W.ERR_INVALID_ARG),
    ((0, 7 * A, 8 * A, None, 2, 4, 4), W.ERR_INVALID_ARG), ((0, 7 * A, 8 * A, 9 * A, 0, 4, 4), W.ERR_INVALID_ARG),
    ((0, 7 * A, 8 * A, 9 * A, 2, 0, 4), W.ERR_INVALID_ARG), ((0, 7 * A, 8 * A, 9 * A, 2, 4, -1), W.ERR_INVALID_ARG),
    ((0, 7 * A + 2, 8 * A, 9 * A, 2, 4, 4), W.ERR_ALIGNMENT), ((0, A + 64, 8 * A, 9 * A, 2, 4, 4), W.ERR_INVALID_ARG),
    ((0, 7 * A, 8 * A, 9 * A, 2, (1 << 31) - 1, 4), W.ERR_UNSUPPORTED),
    ((0, 7 * A, 8 * A, 9 * A, 2, 4, 65536), W.ERR_UNSUPPORTED),
])
def test_write_arguments(L, args, want):
    assert L.w4a16_kv_write(ctypes.byref(cache()), *args, None) == want


@pytest.mark.parametrize("args,want", [
    ((-1, 7 * A, 8 * A, 2, 4, 9, 9 * A, 10 * A), W.ERR_INVALID_ARG),
    ((2, 7 * A, 8 * A, 2, 4, 9, 9 * A, 10 * A), W.ERR_INVALID_ARG),
    ((0, None, 8 * A, 2, 4, 9, 9 * A, 10 * A), W.ERR_INVALID_ARG),
    ((0, 7 * A, None, 2, 4, 9, 9 * A, 10 * A), W.ERR_INVALID_ARG),
    ((0, 7 * A, 8 * A, 2, 4, 9, None, 10 * A), W.ERR_INVALID_ARG),
    ((0, 7 * A, 8 * A, 2, 4, 9, 9 * A, None), W.ERR_INVALID_ARG),
    ((0, 7 * A, 8 * A, 0, 4, 9, 9 * A, 10 * A), W.ERR_INVALID_ARG),
    ((0, 7 * A, 8 * A, 2, 6, 9, 9 * A, 10 * A), W.ERR_INVALID_ARG),   # 6 heads on 4
    ((0, 7 * A, 8 * A, 2, 4, 0, 9 * A, 10 * A), W.ERR_INVALID_ARG),
    ((0, 7 * A, 8 * A, 9, 4, 9, 9 * A, 10 * A), W.ERR_UNSUPPORTED),   # more rows than slots
    ((0, 7 * A, 8 * A, 2, 65536, 9, 9 * A, 10 * A), W.ERR_UNSUPPORTED),
])
def test_decode_arguments(L, args, want):
    assert L.w4a16_attention_decode(ctypes.byref(cache()), *args, None) == want


def test_sizes(L):
    assert L.w4a16_kv_scratch_bytes(100, 8) > 0 and L.w4a16_kv_scratch_bytes(100, 8) % 16 == 0
    assert L.w4a16_kv_scratch_bytes(0, 8) == L.w4a16_kv_scratch_bytes(100, 65537) == 0
    n = ctypes.c_int64()
    assert L.w4a16_attention_decode_workspace(6, 4, ctypes.byref(n)) == W.ERR_INVALID_ARG
    assert L.w4a16_attention_decode_workspace(8, 4, None) == W.ERR_INVALID_ARG


def test_binding_refuses_what_it_can_see():
    import torch
    t = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError):
        W._need_list(t)  # not on the GPU
    with pytest.raises(ValueError):
        W.KVCache.from_tensors(torch.zeros((1, 2, 3, 1, 16, 128), dtype=torch.bfloat16), t.view(2, 2), t, t)


def test_status_string(L):
    assert "pages" in W.status_string(W.ERR_CAPACITY)
