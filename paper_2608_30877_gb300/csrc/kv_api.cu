// C ABI of the paged key-value cache (declared in include/w4a16.h): argument validation and
// dispatch.
#include "kv.h"
#include "layer.h"
#include "w4a16.h"

#include <cuda.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstdint>

namespace w4a16 {
namespace {

constexpr int64_t kMaxDim = (int64_t{1} << 31) - 1;

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// [p, p + bytes); empty where p is null.
struct Span {
    const void* p;
    int64_t bytes;
};
bool overlaps(const Span& a, const Span& b) {
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(a.p), b0 = reinterpret_cast<uintptr_t>(b.p);
    return a.p != nullptr && b.p != nullptr && a0 < b0 + static_cast<uintptr_t>(b.bytes) &&
           b0 < a0 + static_cast<uintptr_t>(a.bytes);
}

bool scratch_sizes_ok(int64_t num_pages, int64_t num_slots) {
    return num_pages > 0 && num_pages <= kKvMaxPages && num_slots > 0 && num_slots <= kKvMaxSlots;
}
int64_t scratch_bytes(int64_t num_pages, int64_t num_slots) {
    const int list = kv_scratch_list(static_cast<int>(num_pages), static_cast<int>(num_slots));
    return (4 * (kKvScratchHeader + kKvScratchLists * static_cast<int64_t>(list) + num_slots) + 15) / 16 * 16;
}

// A cache's buffers, for the overlap checks.
struct CacheSpans {
    Span s[6];
};

int check_cache(const w4a16_kv_cache* c, CacheSpans* spans) {
    if (c == nullptr || c->pages == nullptr || c->page_table == nullptr || c->seq_len == nullptr ||
        c->page_refs == nullptr || c->scratch == nullptr)
        return W4A16_ERR_INVALID_ARG;
    if (c->layers <= 0 || c->num_pages <= 0 || c->kv_heads <= 0 || c->page_tokens <= 0 ||
        c->head_dim <= 0 || c->num_slots <= 0 || c->max_pages <= 0)
        return W4A16_ERR_INVALID_ARG;
    if (c->kv_bits != 16 && c->kv_bits != 8) return W4A16_ERR_INVALID_ARG;
    if ((c->exponents != nullptr) != (c->kv_bits == 8)) return W4A16_ERR_INVALID_ARG;
    if (c->head_dim != kKvHeadDim) return W4A16_ERR_UNSUPPORTED;
    if (c->page_tokens != 16 && c->page_tokens != 32 && c->page_tokens != 64 && c->page_tokens != 128)
        return W4A16_ERR_UNSUPPORTED;
    if (!scratch_sizes_ok(c->num_pages, c->num_slots) || c->layers > 65535 || c->kv_heads > 65535 ||
        c->max_pages > kMaxDim / c->page_tokens || c->num_slots * c->max_pages > kMaxDim ||
        2 * c->num_pages * c->kv_heads > kMaxDim / c->page_tokens)
        return W4A16_ERR_UNSUPPORTED;
    const void* all[6] = {c->pages, c->exponents, c->page_table, c->seq_len, c->page_refs, c->scratch};
    for (const void* p : all)
        if (!aligned16(p)) return W4A16_ERR_ALIGNMENT;
    const int64_t rows = c->layers * 2 * c->num_pages * c->kv_heads * c->page_tokens;
    const int64_t bytes[6] = {rows * c->head_dim * (c->kv_bits / 8), rows,
                              c->num_slots * c->max_pages * 4, c->num_slots * 4, c->num_pages * 4,
                              scratch_bytes(c->num_pages, c->num_slots)};
    for (int i = 0; i < 6; ++i) {
        spans->s[i] = {all[i], bytes[i]};
        for (int j = 0; j < i; ++j)
            if (overlaps(spans->s[i], spans->s[j])) return W4A16_ERR_INVALID_ARG;
    }
    return W4A16_OK;
}

// An argument next to the cache: 16-byte aligned and outside the cache's buffers.
int check_argument(const CacheSpans& c, const Span& a) {
    if (!aligned16(a.p)) return W4A16_ERR_ALIGNMENT;
    for (const Span& s : c.s)
        if (overlaps(a, s)) return W4A16_ERR_INVALID_ARG;
    return W4A16_OK;
}

KvView view_of(const w4a16_kv_cache& c, int* status) {
    KvView v;
    v.pages = static_cast<uint8_t*>(c.pages);
    v.exponents = static_cast<uint8_t*>(c.exponents);
    v.table = static_cast<int32_t*>(c.page_table);
    v.seq_len = static_cast<int32_t*>(c.seq_len);
    v.refs = static_cast<int32_t*>(c.page_refs);
    v.scratch = static_cast<int32_t*>(c.scratch);
    v.refused = v.scratch + kKvScratchHeader +
                kKvScratchLists * static_cast<int64_t>(kv_scratch_list(static_cast<int>(c.num_pages),
                                                                       static_cast<int>(c.num_slots)));
    v.status = status;
    v.layers = static_cast<int>(c.layers);
    v.num_pages = static_cast<int>(c.num_pages);
    v.kv_heads = static_cast<int>(c.kv_heads);
    v.page_shift = 0;
    while ((int64_t{1} << v.page_shift) < c.page_tokens) ++v.page_shift;
    v.num_slots = static_cast<int>(c.num_slots);
    v.max_pages = static_cast<int>(c.max_pages);
    v.row_bytes = static_cast<int>(c.head_dim * (c.kv_bits / 8));
    return v;
}

// Arguments of a page operation over n list entries; b may be null where `optional`.
int check_lists(const w4a16_kv_cache* cache, const void* a, const void* b, bool optional, int64_t n) {
    CacheSpans spans;
    int rc = check_cache(cache, &spans);
    if (rc != W4A16_OK) return rc;
    if (a == nullptr || (b == nullptr && !optional) || n <= 0 || n > cache->num_slots)
        return W4A16_ERR_INVALID_ARG;
    rc = check_argument(spans, {a, n * 4});
    if (rc != W4A16_OK) return rc;
    return check_argument(spans, {b, n * 4});
}

int status_of(cudaError_t e) { return e == cudaSuccess ? W4A16_OK : W4A16_ERR_CUDA; }

}  // namespace
}  // namespace w4a16

using namespace w4a16;

extern "C" int64_t w4a16_kv_scratch_bytes(int64_t num_pages, int64_t num_slots) {
    return scratch_sizes_ok(num_pages, num_slots) ? scratch_bytes(num_pages, num_slots) : 0;
}

extern "C" int w4a16_kv_extend(const w4a16_kv_cache* cache, const void* slots_i32, const void* add_i32,
                               int64_t n, void* stream) {
    int rc = check_lists(cache, slots_i32, add_i32, false, n);
    if (rc != W4A16_OK) return rc;
    LibraryState st;
    rc = library_state(&st);
    if (rc != W4A16_OK) return rc;
    return status_of(launch_kv_extend(view_of(*cache, st.status), static_cast<const int32_t*>(slots_i32),
                                      static_cast<const int32_t*>(add_i32), static_cast<int>(n),
                                      st.sm_count, static_cast<cudaStream_t>(stream)));
}

extern "C" int w4a16_kv_fork(const w4a16_kv_cache* cache, const void* parents_i32,
                             const void* children_i32, int64_t n, void* stream) {
    int rc = check_lists(cache, parents_i32, children_i32, false, n);
    if (rc != W4A16_OK) return rc;
    LibraryState st;
    rc = library_state(&st);
    if (rc != W4A16_OK) return rc;
    return status_of(launch_kv_fork(view_of(*cache, st.status), static_cast<const int32_t*>(parents_i32),
                                    static_cast<const int32_t*>(children_i32), static_cast<int>(n),
                                    static_cast<cudaStream_t>(stream)));
}

extern "C" int w4a16_kv_trim(const w4a16_kv_cache* cache, const void* slots_i32, const void* keep_i32,
                             int64_t n, void* stream) {
    int rc = check_lists(cache, slots_i32, keep_i32, true, n);
    if (rc != W4A16_OK) return rc;
    LibraryState st;
    rc = library_state(&st);
    if (rc != W4A16_OK) return rc;
    return status_of(launch_kv_trim(view_of(*cache, st.status), static_cast<const int32_t*>(slots_i32),
                                    static_cast<const int32_t*>(keep_i32), static_cast<int>(n),
                                    static_cast<cudaStream_t>(stream)));
}

extern "C" int w4a16_kv_compact(const w4a16_kv_cache* cache, void* stream) {
    CacheSpans spans;
    int rc = check_cache(cache, &spans);
    if (rc != W4A16_OK) return rc;
    LibraryState st;
    rc = library_state(&st);
    if (rc != W4A16_OK) return rc;
    return status_of(launch_kv_compact(view_of(*cache, st.status), st.sm_count,
                                       static_cast<cudaStream_t>(stream)));
}

extern "C" int w4a16_kv_write(const w4a16_kv_cache* cache, int64_t layer, const void* qkv_bf16,
                              const void* seq_start_i32, const void* slots_i32, int64_t nseq, int64_t M,
                              int64_t H, void* stream) {
    CacheSpans spans;
    int rc = check_cache(cache, &spans);
    if (rc != W4A16_OK) return rc;
    if (qkv_bf16 == nullptr || seq_start_i32 == nullptr || slots_i32 == nullptr || layer < 0 ||
        layer >= cache->layers || nseq <= 0 || M <= 0 || H < 0)
        return W4A16_ERR_INVALID_ARG;
    if (M > kMaxDim - 16 || nseq > kMaxDim / 2 || H > 65535) return W4A16_ERR_UNSUPPORTED;
    rc = check_argument(spans, {qkv_bf16, M * (H + 2 * cache->kv_heads) * cache->head_dim * 2});
    if (rc != W4A16_OK) return rc;
    rc = check_argument(spans, {seq_start_i32, (nseq + 1) * 4});
    if (rc != W4A16_OK) return rc;
    rc = check_argument(spans, {slots_i32, nseq * 4});
    if (rc != W4A16_OK) return rc;
    LibraryState st;
    rc = library_state(&st);
    if (rc != W4A16_OK) return rc;
    const KvWriteParams p{static_cast<const uint16_t*>(qkv_bf16), static_cast<const int32_t*>(seq_start_i32),
                          static_cast<const int32_t*>(slots_i32), static_cast<int>(layer),
                          static_cast<int>(nseq), static_cast<int>(M), static_cast<int>(H)};
    return status_of(launch_kv_write(view_of(*cache, st.status), p, st.sm_count, static_cast<cudaStream_t>(stream)));
}

extern "C" int w4a16_kv_rotary(const w4a16_kv_cache* cache, void* qkv_bf16, const void* seq_start_i32,
                               const void* slots_i32, int64_t nseq, int64_t M, int64_t H, const void* turns_u64,
                               int64_t rot_dim, int layout, float factor, void* stream) {
    CacheSpans spans;
    int rc = check_cache(cache, &spans);
    if (rc != W4A16_OK) return rc;
    if (qkv_bf16 == nullptr || slots_i32 == nullptr || turns_u64 == nullptr || nseq <= 0 || M <= 0 || H < 0 ||
        rot_dim <= 0 || rot_dim > cache->head_dim || !std::isfinite(factor) ||
        (layout != W4A16_ROTARY_HALF && layout != W4A16_ROTARY_PAIRS) || (seq_start_i32 == nullptr && nseq != M))
        return W4A16_ERR_INVALID_ARG;
    if (M > kMaxDim - 16 || nseq > kMaxDim / 2 || H > 65535 || rot_dim % 16 != 0) return W4A16_ERR_UNSUPPORTED;
    const Span args[4] = {{qkv_bf16, M * (H + 2 * cache->kv_heads) * cache->head_dim * 2},
                          {seq_start_i32, (nseq + 1) * 4},
                          {slots_i32, nseq * 4},
                          {turns_u64, rot_dim / 2 * 8}};
    for (int i = 0; i < 4; ++i) {
        rc = check_argument(spans, args[i]);
        if (rc != W4A16_OK) return rc;
        if (i > 0 && overlaps(args[0], args[i])) return W4A16_ERR_INVALID_ARG;
    }
    LibraryState st;
    rc = library_state(&st);
    if (rc != W4A16_OK) return rc;
    RotaryParams p;
    p.qkv = static_cast<uint16_t*>(qkv_bf16);
    p.seq_start = static_cast<const int32_t*>(seq_start_i32);
    p.first = static_cast<const int32_t*>(slots_i32);
    p.turns = static_cast<const uint64_t*>(turns_u64);
    p.status = st.status;
    p.M = static_cast<int>(M);
    p.nseq = static_cast<int>(nseq);
    p.H = static_cast<int>(H);
    p.kv_heads = static_cast<int>(cache->kv_heads);
    p.d = kKvHeadDim;
    p.rot = static_cast<int>(rot_dim);
    p.factor = factor;
    p.pairs = layout == W4A16_ROTARY_PAIRS;
    const KvView view = view_of(*cache, st.status);
    return status_of(launch_rotary(&view, p, st.sm_count, static_cast<cudaStream_t>(stream)));
}

extern "C" int w4a16_attention_decode_workspace(int64_t H, int64_t kv_heads, int64_t* bytes) {
    if (bytes == nullptr || H <= 0 || kv_heads <= 0 || H % kv_heads != 0) return W4A16_ERR_INVALID_ARG;
    if (H > 65535) return W4A16_ERR_UNSUPPORTED;
    LibraryState st;
    const int rc = library_state(&st);
    if (rc != W4A16_OK) return rc;
    *bytes = decode_workspace_bytes(static_cast<int>(H), static_cast<int>(kv_heads), st.sm_count);
    return W4A16_OK;
}

extern "C" int w4a16_attention_decode(const w4a16_kv_cache* cache, int64_t layer, const void* qkv_bf16,
                                      const void* slots_i32, int64_t n, int64_t H, int64_t window,
                                      void* out_bf16, void* workspace, void* stream) {
    CacheSpans spans;
    int rc = check_cache(cache, &spans);
    if (rc != W4A16_OK) return rc;
    if (qkv_bf16 == nullptr || slots_i32 == nullptr || out_bf16 == nullptr || workspace == nullptr ||
        layer < 0 || layer >= cache->layers || n <= 0 || H <= 0 || H % cache->kv_heads != 0 || window <= 0)
        return W4A16_ERR_INVALID_ARG;
    if (n > cache->num_slots || H > 65535) return W4A16_ERR_UNSUPPORTED;
    LibraryState st;
    rc = library_state(&st);
    if (rc != W4A16_OK) return rc;
    const Span args[4] = {{qkv_bf16, n * (H + 2 * cache->kv_heads) * cache->head_dim * 2},
                          {slots_i32, n * 4},
                          {out_bf16, n * H * cache->head_dim * 2},
                          {workspace, decode_workspace_bytes(static_cast<int>(H),
                                                             static_cast<int>(cache->kv_heads), st.sm_count)}};
    for (int i = 0; i < 4; ++i) {
        rc = check_argument(spans, args[i]);
        if (rc != W4A16_OK) return rc;
        for (int j = 2; j < i; ++j)
            if (overlaps(args[i], args[j])) return W4A16_ERR_INVALID_ARG;
    }
    for (int i = 0; i < 2; ++i)
        if (overlaps(args[i], args[2]) || overlaps(args[i], args[3])) return W4A16_ERR_INVALID_ARG;
    DecodeParams p;
    p.qkv = static_cast<const uint16_t*>(qkv_bf16);
    p.slots = static_cast<const int32_t*>(slots_i32);
    p.out = static_cast<uint16_t*>(out_bf16);
    p.workspace = workspace;
    p.layer = static_cast<int>(layer);
    p.n = static_cast<int>(n);
    p.H = static_cast<int>(H);
    p.window = window > kMaxDim ? static_cast<int>(kMaxDim) : static_cast<int>(window);
    p.scale = 1.0f / sqrtf(static_cast<float>(kKvHeadDim));
    p.wait_ns = wait_limit_ns();
    const KvView view = view_of(*cache, st.status);
    CacheMaps maps;
    rc = encode_cache(&maps, view, p.layer);
    if (rc != W4A16_OK) return rc;
    return status_of(launch_attention_decode(maps, view, p, st.sm_count, static_cast<cudaStream_t>(stream)));
}
