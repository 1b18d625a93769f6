// Keys and values of a packed batch's tokens into the cache's pages.
//
// Rows of the fused projection hold a token's keys and values of all heads in one run;
// in a page a head's tokens lie in one run.  A CTA takes 1 to 32 tokens (few heads, many tokens);
// 16 threads move a row of 128 values in 16-byte pieces (and reduce its largest value for the 8-bit
// form), several rows under way together.  Bound by HBM: each value is read once and written
// once; 39000 tokens of 96 heads take 561 us (6.8 TB/s, the copy bandwidth), in 8 bits 509 (83%).  Short
// calls are bound by the way to a token's place: three loads in a row before the first row (13000
// tokens of 8 heads in 8 bits 20 us, 13 at the copy bandwidth).  A row's addresses are sums of
// 32-bit offsets: with divisions and 64-bit products per row the issue slots were the bound.
// Rows under way / CTAs an SM in 8 bits, 13000 tokens of 8 heads and 39000 of 96: 2 / 8 20 and
// 505 us, 4 / 6 22 and 541, 4 / 5 21 and 522, 2 / 6 21 and 552; in bf16 4 / 6 576, 2 / 8 593.  The first
// rows loaded ahead of the places took registers and time (22.9, 560).
#include <cuda_runtime.h>
#include <cstdint>

#include "kv.h"
#include "kv_row.cuh"
#include "ptx.cuh"

namespace w4a16 {

namespace {

constexpr int kThreads = 256;
constexpr int kTokens = 32;  // of a CTA, at most
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
    const bool refused = growth_refused(kv, true, slot);  // (beside the length: a load of any_refused first takes 0.9 us)
    if (refused || begin < 0 || end > p.M || m >= end || len < end - begin ||
        len > static_cast<int64_t>(kv.max_pages) << kv.page_shift)
        return;
    const int pos = len - end + m;
    const int found = kv.table[static_cast<int64_t>(slot) * kv.max_pages + (pos >> kv.page_shift)];
    if (found < 0 || found >= kv.num_pages) return;
    *page = found;
    *at = pos & ((1 << kv.page_shift) - 1);
}

constexpr int kCheckSlots = kStarts * 32;  // of a checking CTA

// Whether a slot from `from` on is twice among the sequences with rows, by one CTA with a bit for each
// slot.  (Every CTA comparing its tokens' slots with the list, which would tell it to leave them out,
// took 9 us of 508 with 64 sequences of 96 heads and 1800 with 60000 sequences of one token.)
__device__ __noinline__ void check_slots(const int32_t* slots, const int32_t* seq_start, int nseq, int from, int to,
                                         uint32_t* bits, int* status) {
    constexpr int kSide = 2;  // pieces of the lists that a thread has under way
    for (int i = threadIdx.x; i < kStarts; i += kThreads) bits[i] = 0;
    __syncthreads();
    auto claim = [&](int slot, int begin, int end) {
        if (begin >= end || slot < from || slot >= to) return;
        const uint32_t bit = 1u << ((slot - from) & 31);
        if (atomicOr(&bits[(slot - from) >> 5], bit) & bit) record_status(status, 1 /* W4A16_ERR_INVALID_ARG */);
    };
    const int whole = nseq & ~3;
    for (int64_t i0 = 4 * threadIdx.x; i0 < whole; i0 += 4 * kThreads * kSide) {
        int4 s[kSide], b[kSide];
        int e[kSide];
#pragma unroll
        for (int k = 0; k < kSide; ++k) {
            const int64_t i = i0 + 4 * kThreads * k;
            if (i < whole) {
                s[k] = *reinterpret_cast<const int4*>(slots + i);
                b[k] = *reinterpret_cast<const int4*>(seq_start + i);
                e[k] = seq_start[i + 4];
            }
        }
#pragma unroll
        for (int k = 0; k < kSide; ++k)
            if (i0 + 4 * kThreads * k < whole) {
                claim(s[k].x, b[k].x, b[k].y);
                claim(s[k].y, b[k].y, b[k].z);
                claim(s[k].z, b[k].z, b[k].w);
                claim(s[k].w, b[k].w, e[k]);
            }
    }
    const int i = whole + static_cast<int>(threadIdx.x);
    if (i < nseq) claim(slots[i], seq_start[i], seq_start[i + 1]);
}

// The first CTAs, one for each kCheckSlots slots, check the list of slots; the others move `tokens`
// tokens each.
template <bool E4M3>
__global__ void __launch_bounds__(kThreads, E4M3 ? 8 : 6) kv_write_kernel(const KvView kv, const KvWriteParams p,
                                                                             const int tokens) {
    constexpr int kBatch = E4M3 ? 2 : 4;  // rows that 16 threads have under way
    __shared__ int rows_at[kTokens];       // of a token: its row of head 0, -1 if it is left out
    __shared__ int32_t starts[kStarts + 1];
    const int checks = (kv.num_slots + kCheckSlots - 1) / kCheckSlots;
    const int block = static_cast<int>(blockIdx.x) - checks;
    const int m0 = block * tokens;
    grid_launch_dependents();
    grid_wait();
    if (block < 0) {
        const int from = static_cast<int>(blockIdx.x) * kCheckSlots;
        check_slots(p.slots, p.seq_start, p.nseq, from, min(from + kCheckSlots, kv.num_slots),
                    reinterpret_cast<uint32_t*>(starts), kv.status);
        return;
    }
    const bool staged = p.nseq <= kStarts;
    if (staged) {
        for (int i = threadIdx.x; i <= p.nseq; i += kThreads) starts[i] = p.seq_start[i];
        __syncthreads();
    }
    if (threadIdx.x < tokens) {
        int page = -1, at = 0;
        if (m0 + threadIdx.x < p.M)
            token_place(kv, p, staged ? starts : p.seq_start, m0 + threadIdx.x, &page, &at);
        if (page == -2) record_status(kv.status, 1 /* W4A16_ERR_INVALID_ARG */);
        // (a layer's rows are fewer than 2^31)
        rows_at[threadIdx.x] = page < 0 ? -1 : ((page * kv.kv_heads) << kv.page_shift) + at;
    }
    // a table that decreases anywhere is an error, also where no token shows it
    for (int64_t s = static_cast<int64_t>(block) * kThreads + threadIdx.x; s < p.nseq;
         s += static_cast<int64_t>(gridDim.x - checks) * kThreads)
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
    while (t < tokens) {
        uint4 v[kBatch];
        int row[kBatch], which[kBatch];
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            row[b] = -1;
            if (t < tokens && rows_at[t] >= 0) {
                v[b] = __ldcs(src + t * width + r * (kKvHeadDim / 8));
                which[b] = r >= kv.kv_heads;
                row[b] = rows_at[t] + ((r - (which[b] ? kv.kv_heads : 0)) << kv.page_shift);
            }
            r += kThreads / 16;
            while (r >= rows && t < tokens) {
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

cudaError_t launch_kv_write(const KvView& kv, const KvWriteParams& p, int sm_count, cudaStream_t stream) {
    // At most 64 pairs of rows to a CTA, and a CTA for each SM if there are tokens for it.  (us, with 64 /
    // 128 / 768 pairs: 39000 tokens of 96 heads 561 / 561 / 576, in 8 bits 508 / 508 / 505, 40 of 32
    // heads 4.2 / 5.7 / 8.9, one of 96 4.7 / 4.7 / 13; with 32 pairs 13000 of 8 heads in 8 bits 21.2
    // and not 20.1.  One head, 64000 tokens: 32 tokens to a CTA 11.6, 8 21.8.)
    int tokens = kTokens;
    while (tokens > 1 && (tokens * kv.kv_heads > 64 || static_cast<int64_t>(tokens) * sm_count > p.M)) tokens /= 2;
    const int grid = static_cast<int>((static_cast<int64_t>(p.M) + tokens - 1) / tokens) +
                     (kv.num_slots + kCheckSlots - 1) / kCheckSlots;
    return launch_overlapped(kv.exponents != nullptr ? kv_write_kernel<true> : kv_write_kernel<false>, grid, kThreads,
                             0, stream, kv, p, tokens);
}

}  // namespace w4a16
