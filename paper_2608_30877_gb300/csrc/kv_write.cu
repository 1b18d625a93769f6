// Keys and values of a packed batch's tokens into the cache's pages.
//
// Rows of the fused projection hold a token's keys and values of all heads in one run;
// in a page a head's tokens lie in one run.  A CTA takes 8 tokens; 16 threads move a row of 128
// values in 16-byte pieces (and reduce its largest value for the 8-bit form), several rows
// under way together.  Bound by HBM: each value is read once and written once.  A row's
// addresses are sums of 32-bit offsets: with divisions and 64-bit products per row the
// issue slots were the bound (13000 tokens of 8 heads in 8 bits 32 us, now 22; 39000 of 96 heads
// in bf16 600, now 576, 97% of the copy bandwidth).  Tokens / rows under way / CTAs an SM, both
// in us: 8 / 4 / 6 576 and 24, 16 / 4 / 4 577 and 23, 8 / 2 / 8 593 and 22, 32 / 4 / 4 622 and 28.
#include <cuda_runtime.h>
#include <cstdint>

#include "kv.h"
#include "kv_row.cuh"
#include "ptx.cuh"

namespace w4a16 {

namespace {

constexpr int kThreads = 256;
constexpr int kTokens = 8;  // tokens of a CTA
constexpr int kStarts = 1024;  // a sequence table of up to so many sequences is searched in shared memory

// Where token m of the packed batch goes: its page and place there; page -1 outside every
// sequence or for an entry of -1, -2 for an error.
__device__ __forceinline__ void token_place(const KvView& kv, const KvWriteParams& p, const int32_t* starts, int m,
                                            int* page, int* at) {
    *page = -1;
    int lo = 0, hi = p.nseq;  // the last sequence that starts at m or before
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (starts[mid] <= m) lo = mid; else hi = mid - 1;
    }
    if (lo >= p.nseq || starts[lo] > m) return;
    const int begin = starts[lo], end = starts[lo + 1], slot = p.slots[lo];
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
__global__ void __launch_bounds__(kThreads, E4M3 ? 8 : 6) kv_write_kernel(const KvView kv, const KvWriteParams p) {
    constexpr int kBatch = E4M3 ? 2 : 4;  // rows that 16 threads have under way
    __shared__ int rows_at[kTokens];       // of a token: its row of head 0, -1 if it is left out
    __shared__ int32_t starts[kStarts + 1];
    const int m0 = blockIdx.x * kTokens;
    grid_launch_dependents();
    grid_wait();
    const bool staged = p.nseq <= kStarts;
    if (staged) {
        for (int i = threadIdx.x; i <= p.nseq; i += kThreads) starts[i] = p.seq_start[i];
        __syncthreads();
    }
    if (threadIdx.x < kTokens) {
        int page = -1, at = 0;
        if (m0 + threadIdx.x < p.M)
            token_place(kv, p, staged ? starts : p.seq_start, m0 + threadIdx.x, &page, &at);
        if (page == -2) record_status(kv.status, 1 /* W4A16_ERR_INVALID_ARG */);
        // (a layer's rows are fewer than 2^31)
        rows_at[threadIdx.x] = page < 0 ? -1 : ((page * kv.kv_heads) << kv.page_shift) + at;
    }
    // a table that decreases anywhere is an error, also where no token shows it
    for (int64_t s = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; s < p.nseq;
         s += static_cast<int64_t>(gridDim.x) * kThreads)
        if (p.seq_start[s] > p.seq_start[s + 1] || p.seq_start[s] < 0 || p.seq_start[s + 1] > p.M)
            record_status(kv.status, 1);
    __syncthreads();
    const int lane16 = threadIdx.x & 15;
    const int rows = 2 * kv.kv_heads;  // of a token
    const int64_t width = static_cast<int64_t>(p.H + rows) * (kKvHeadDim / 8);  // in 16-byte pieces
    const uint4* const src = reinterpret_cast<const uint4*>(p.qkv) + m0 * width + p.H * (kKvHeadDim / 8) + lane16;
    const int value_rows = (kv.num_pages * kv.kv_heads) << kv.page_shift;  // from a key to its value
    uint8_t* const pages = kv.pages + 2 * static_cast<int64_t>(p.layer) * value_rows * kv.row_bytes;
    uint8_t* const exponents =
        E4M3 ? kv.exponents + 2 * static_cast<int64_t>(p.layer) * value_rows : nullptr;
    // these 16 threads' next row: row r of token t, keys of all heads and then values
    int t = (threadIdx.x >> 4) / rows, r = (threadIdx.x >> 4) - t * rows;
    while (t < kTokens) {
        uint4 v[kBatch];
        int row[kBatch], which[kBatch];
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            row[b] = -1;
            if (t < kTokens && rows_at[t] >= 0) {
                v[b] = __ldcs(src + t * width + r * (kKvHeadDim / 8));
                which[b] = r >= kv.kv_heads;
                row[b] = rows_at[t] + ((r - (which[b] ? kv.kv_heads : 0)) << kv.page_shift);
            }
            r += kThreads / 16;
            while (r >= rows && t < kTokens) {
                r -= rows;
                ++t;
            }
        }
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            if (row[b] < 0) continue;  // (the same for the row's 16 threads)
            const int64_t to = (static_cast<int64_t>(row[b]) + (which[b] ? value_rows : 0)) * 16 + lane16;
            if constexpr (!E4M3) {
                reinterpret_cast<uint4*>(pages)[to] = v[b];
            } else {
                uint2 codes;
                const int e = e4m3_row_of_16(v[b], &codes);
                reinterpret_cast<uint2*>(pages)[to] = codes;
                if (lane16 == 0) exponents[2 * static_cast<int64_t>(row[b]) + which[b]] = static_cast<uint8_t>(e + 127);
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
