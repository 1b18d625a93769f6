// Keys and values of a packed batch's tokens into the cache's pages.
//
// Rows of the fused projection hold a token's keys and values of all heads in one run;
// in a page a head's tokens lie in one run.  16 threads move a row of 128 values in
// 16-byte pieces (and reduce its largest value for the 8-bit form).  Bound by HBM: each
// value is read once and written once.
#include <cuda_runtime.h>
#include <cstdint>

#include "kv.h"
#include "kv_row.cuh"
#include "ptx.cuh"

namespace w4a16 {

namespace {

constexpr int kThreads = 256;
constexpr int kTokens = 16;  // tokens of a CTA
constexpr int kBatch = 4;    // rows that 16 threads have under way

// Where token m of the packed batch goes: its page and place there; page -1 outside every
// sequence or for an entry of -1, -2 for an error.
__device__ __forceinline__ void token_place(const KvView& kv, const KvWriteParams& p, int m, int* page,
                                            int* at) {
    *page = -1;
    int lo = 0, hi = p.nseq;  // the last sequence that starts at m or before
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (p.seq_start[mid] <= m) lo = mid; else hi = mid - 1;
    }
    if (lo >= p.nseq || p.seq_start[lo] > m) return;
    const int begin = p.seq_start[lo], end = p.seq_start[lo + 1], slot = p.slots[lo];
    if (slot == -1) return;
    *page = -2;
    if (slot < 0 || slot >= kv.num_slots) return;
    const int len = kv.seq_len[slot];
    if (begin < 0 || end > p.M || m >= end || len < end - begin ||
        len > static_cast<int64_t>(kv.max_pages) << kv.page_shift)
        return;
    const int pos = len - end + m;
    const int found = kv.table[static_cast<int64_t>(slot) * kv.max_pages + (pos >> kv.page_shift)];
    if (found < 0 || found >= kv.num_pages) return;
    *page = found;
    *at = pos & ((1 << kv.page_shift) - 1);
}

template <bool E4M3>
__global__ void __launch_bounds__(kThreads) kv_write_kernel(const KvView kv, const KvWriteParams p) {
    __shared__ int pages[kTokens], places[kTokens];
    const int m0 = blockIdx.x * kTokens;
    grid_launch_dependents();
    grid_wait();
    if (threadIdx.x < kTokens) {
        int page = -1, at = 0;
        if (m0 + threadIdx.x < p.M) token_place(kv, p, m0 + threadIdx.x, &page, &at);
        if (page == -2) record_status(kv.status, 1 /* W4A16_ERR_INVALID_ARG */);
        pages[threadIdx.x] = page;
        places[threadIdx.x] = at;
    }
    // a table that decreases anywhere is an error, also where no token shows it
    for (int64_t s = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; s < p.nseq;
         s += static_cast<int64_t>(gridDim.x) * kThreads)
        if (p.seq_start[s] > p.seq_start[s + 1] || p.seq_start[s] < 0 || p.seq_start[s + 1] > p.M)
            record_status(kv.status, 1);
    __syncthreads();
    const int lane16 = threadIdx.x & 15;
    const int rows = 2 * kv.kv_heads;  // of a token
    const int64_t width = static_cast<int64_t>(p.H + rows) * kKvHeadDim;
    // (kBatch rows' loads under way together: one at a time, 13000 tokens of 8 heads took 32 us)
    for (int r0 = threadIdx.x >> 4; r0 < kTokens * rows; r0 += kBatch * (kThreads / 16)) {
        uint4 v[kBatch];
        int64_t row[kBatch], exponent[kBatch];
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            const int r = r0 + b * (kThreads / 16);
            const int t = r < kTokens * rows ? r / rows : 0;
            const int which = (r - t * rows) / kv.kv_heads, head = r - t * rows - which * kv.kv_heads;
            row[b] = -1;
            if (r >= kTokens * rows || pages[t] < 0) continue;  // (the same for the row's 16 threads)
            v[b] = __ldg(reinterpret_cast<const uint4*>(
                p.qkv + (m0 + t) * width +
                (p.H + which * kv.kv_heads + head) * static_cast<int64_t>(kKvHeadDim)) + lane16);
            row[b] = kv_row(kv, p.layer, which, pages[t], head, places[t]);
            exponent[b] = kv_exponent(kv, p.layer, which, pages[t], head, places[t]);
        }
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            if (row[b] < 0) continue;
            if constexpr (!E4M3) {
                reinterpret_cast<uint4*>(kv.pages)[row[b] * 16 + lane16] = v[b];
            } else {
                uint2 codes;
                const int e = e4m3_row_of_16(v[b], &codes);
                reinterpret_cast<uint2*>(kv.pages)[row[b] * 16 + lane16] = codes;
                if (lane16 == 0) kv.exponents[exponent[b]] = static_cast<uint8_t>(e + 127);
            }
        }
    }
}

}  // namespace

cudaError_t launch_kv_write(const KvView& kv, const KvWriteParams& p, cudaStream_t stream) {
    const int grid = (p.M + kTokens - 1) / kTokens;
    return launch_overlapped(kv.exponents != nullptr ? kv_write_kernel<true> : kv_write_kernel<false>, grid, kThreads,
                             0, stream, kv, p);
}

}  // namespace w4a16
