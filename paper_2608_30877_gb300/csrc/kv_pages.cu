// Page operations of the key-value cache: growth with copy on write, sharing, release
// and compaction.
//
// A page is free if no sequence refers to it; the free pages are found by scanning the
// reference counts, lowest index first, so there is no list to keep in step with them and
// every result is a function of the tables alone (integer atomics commute).  Each
// operation runs its checks before its first change, so an error leaves the cache as it was.
// One CTA plans; what has to be copied (an extend's shared last pages, a compaction's
// moved pages) goes to a list in the scratch buffer that a second kernel works off over
// the whole GPU.  Bound by latency but for the copies, which HBM bounds.
#include <cuda_runtime.h>
#include <cstdint>

#include "kv.h"
#include "kv_row.cuh"
#include "ptx.cuh"

namespace w4a16 {

namespace {

constexpr int kThreads = 1024;
constexpr int kInvalid = 1;   // W4A16_ERR_INVALID_ARG
constexpr int kCapacity = 7;  // W4A16_ERR_CAPACITY
// A copy's source page and, from this bit on, its tokens (fewer than a page's 128 at most).
constexpr int kTokenShift = 24;
static_assert(kKvMaxPages == 1 << kTokenShift);

// The scratch buffer's lists: copied pages, and growth's plan and free pages or
// compaction's map, which never live at the same time as one another.
struct Lists {
    KvScratch* head;
    int32_t *src, *dst, *a, *b;
};
__device__ __forceinline__ Lists lists_of(const KvView& kv) {
    const int n = kv_scratch_list(kv.num_pages, kv.num_slots);
    int32_t* p = kv.scratch + kKvScratchHeader;
    return {reinterpret_cast<KvScratch*>(kv.scratch), p, p + n, p + 2 * n, p + 3 * n};
}

struct PlanShared {
    uint32_t seen[kKvMaxSlots / 32];
    int warp[kThreads / 32];
    int total;
    int error;
    int copies;
};

// Exclusive sum over the CTA's threads in thread order, and the total; all threads call it.
__device__ __forceinline__ int block_scan(int v, PlanShared& sh, int* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int inc = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int t = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += t;
    }
    if (lane == 31) sh.warp[warp] = inc;
    __syncthreads();
    if (warp == 0) {
        int w = sh.warp[lane];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int t = __shfl_up_sync(0xffffffffu, w, o);
            if (lane >= o) w += t;
        }
        sh.warp[lane] = w;
    }
    __syncthreads();
    const int before = warp > 0 ? sh.warp[warp - 1] : 0;
    *total = sh.warp[kThreads / 32 - 1];
    __syncthreads();
    return before + inc - v;
}

__device__ __forceinline__ void plan_begin(const KvView& kv, PlanShared& sh) {
    for (int i = threadIdx.x; i < (kv.num_slots + 31) / 32; i += kThreads) sh.seen[i] = 0;
    if (threadIdx.x == 0) sh.error = sh.copies = 0;
    __syncthreads();
    grid_launch_dependents();
    grid_wait();
}
// Whether the slot is within range and new to the call.
__device__ __forceinline__ bool claim_slot(const KvView& kv, PlanShared& sh, int slot) {
    if (slot < 0 || slot >= kv.num_slots) return false;
    const uint32_t bit = 1u << (slot & 31);
    return (atomicOr(&sh.seen[slot >> 5], bit) & bit) == 0;
}
__device__ __forceinline__ bool length_ok(const KvView& kv, int len) {
    return len >= 0 && len <= static_cast<int64_t>(kv.max_pages) << kv.page_shift;
}
__device__ __forceinline__ int pages_of(const KvView& kv, int len) {
    return (len + (1 << kv.page_shift) - 1) >> kv.page_shift;
}
__device__ __forceinline__ int32_t* entries_of(const KvView& kv, int slot) {
    return kv.table + static_cast<int64_t>(slot) * kv.max_pages;
}
__device__ __forceinline__ bool page_ok(const KvView& kv, int page) {
    return page >= 0 && page < kv.num_pages;
}

// The slot's last page if the sequence is to get a copy of it, else -1; false for a bad index.
__device__ __forceinline__ bool shared_last(const KvView& kv, int slot, int len, int add, int* page) {
    *page = -1;
    if (add <= 0 || (len & ((1 << kv.page_shift) - 1)) == 0) return true;
    const int last = entries_of(kv, slot)[len >> kv.page_shift];
    if (!page_ok(kv, last)) return false;
    if (kv.refs[last] > 1) *page = last;
    return true;
}

__global__ void __launch_bounds__(kThreads)
    kv_extend_kernel(const KvView kv, const int32_t* __restrict__ slots,
                     const int32_t* __restrict__ add, int n) {
    __shared__ PlanShared sh;
    const Lists ls = lists_of(kv);
    const int tid = threadIdx.x;
    plan_begin(kv, sh);
    // pages that each entry needs, as offsets into the pages to allocate (list a)
    int need_all = 0;
    bool too_many = false;
    for (int i0 = 0; i0 < n; i0 += kThreads) {
        const int i = i0 + tid;
        int need = 0;
        if (i < n && slots[i] != -1) {
            const int slot = slots[i], grow = add[i];
            int error = 0, copy = -1;
            if (!claim_slot(kv, sh, slot) || grow < 0) {
                error = kInvalid;
            } else {
                const int len = kv.seq_len[slot];
                const int64_t to = static_cast<int64_t>(len) + grow;
                if (!length_ok(kv, len) || !shared_last(kv, slot, len, grow, &copy))
                    error = kInvalid;
                else if (to > static_cast<int64_t>(kv.max_pages) << kv.page_shift)
                    error = kCapacity;
                else
                    need = pages_of(kv, static_cast<int>(to)) - pages_of(kv, len) + (copy >= 0);
            }
            if (error != 0) atomicCAS(&sh.error, 0, error);
        }
        int sum;
        const int before = block_scan(need, sh, &sum);
        if (i < n) ls.a[i] = need_all + before;
        too_many |= sum > kv.num_pages - need_all;  // (no overflow: need_all stays below)
        if (too_many) break;
        need_all += sum;
    }
    // the lowest free pages, in order (list b)
    int found = 0;
    if (!too_many) {
        // kRun counts a thread and pass, which a pool of 16000 pages takes once
        constexpr int kRun = 16;
        for (int p0 = 0; p0 < kv.num_pages && found < need_all; p0 += kThreads * kRun) {
            const int begin = p0 + tid * kRun;
            uint32_t free = 0;
            if (begin + kRun <= kv.num_pages) {
                int4 v[kRun / 4];
#pragma unroll
                for (int k = 0; k < kRun / 4; ++k) v[k] = reinterpret_cast<const int4*>(kv.refs + begin)[k];
#pragma unroll
                for (int k = 0; k < kRun / 4; ++k)
                    free |= ((v[k].x == 0) | (v[k].y == 0) << 1 | (v[k].z == 0) << 2 | (v[k].w == 0) << 3) << 4 * k;
            } else {
                for (int k = 0; begin + k < kv.num_pages; ++k) free |= (kv.refs[begin + k] == 0) << k;
            }
            int sum;
            int rank = found + block_scan(__popc(free), sh, &sum);
            for (; free != 0 && rank < need_all; free &= free - 1, ++rank) ls.b[rank] = begin + __ffs(free) - 1;
            found += sum;
        }
    }
    __syncthreads();
    if (sh.error != 0 || too_many || found < need_all) {
        if (tid == 0) {
            record_status(kv.status, sh.error != 0 ? sh.error : kCapacity);
            ls.head->copies = 0;
            ls.head->moved = -1;
        }
        return;
    }
    // what to copy, before any count changes
    for (int i = tid; i < n; i += kThreads) {
        const int slot = slots[i];
        int copy = -1;
        if (slot != -1) shared_last(kv, slot, kv.seq_len[slot], add[i], &copy);
        if (copy >= 0) {
            const int c = atomicAdd(&sh.copies, 1);  // (the copies' order does not matter)
            ls.src[c] = copy | (kv.seq_len[slot] & ((1 << kv.page_shift) - 1)) << kTokenShift;
            ls.dst[c] = i;
        }
    }
    __syncthreads();
    for (int c = tid; c < sh.copies; c += kThreads)
        atomicSub(&kv.refs[ls.src[c] & (kKvMaxPages - 1)], 1);
    // page r of the allocated ones belongs to the last entry whose offset is at most r
    for (int r = tid; r < need_all; r += kThreads) {
        int lo = 0, hi = n - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (ls.a[mid] <= r) lo = mid; else hi = mid - 1;
        }
        const int slot = slots[lo];
        const int need = (lo + 1 < n ? ls.a[lo + 1] : need_all) - ls.a[lo];
        const int has = pages_of(kv, kv.seq_len[slot] + add[lo]);
        const int page = ls.b[r];
        entries_of(kv, slot)[has - need + r - ls.a[lo]] = page;
        kv.refs[page] = 1;
    }
    __syncthreads();
    for (int c = tid; c < sh.copies; c += kThreads) ls.dst[c] = ls.b[ls.a[ls.dst[c]]];
    for (int i = tid; i < n; i += kThreads)
        if (slots[i] != -1) kv.seq_len[slots[i]] += add[i];
    if (tid == 0) {
        ls.head->copies = sh.copies;
        ls.head->moved = -1;
    }
}

__global__ void __launch_bounds__(kThreads)
    kv_fork_kernel(const KvView kv, const int32_t* __restrict__ parents,
                   const int32_t* __restrict__ children, int n) {
    __shared__ PlanShared sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    plan_begin(kv, sh);
    for (int i = tid; i < n; i += kThreads) {
        if (children[i] == -1) continue;
        const int parent = parents[i];
        if (!claim_slot(kv, sh, children[i]) || kv.seq_len[children[i]] != 0 || parent < 0 ||
            parent >= kv.num_slots || !length_ok(kv, kv.seq_len[parent]))
            sh.error = kInvalid;
    }
    __syncthreads();
    for (int i = warp; i < n && sh.error == 0; i += kThreads / 32) {
        if (children[i] == -1) continue;
        const int parent = parents[i];
        bool ok = (sh.seen[parent >> 5] >> (parent & 31) & 1) == 0;  // (a child of this call)
        const int pages = pages_of(kv, kv.seq_len[parent]);
        for (int e = lane; e < pages; e += 32) ok &= page_ok(kv, entries_of(kv, parent)[e]);
        if (!ok) sh.error = kInvalid;
    }
    __syncthreads();
    if (sh.error != 0) {
        if (tid == 0) record_status(kv.status, sh.error);
        return;
    }
    for (int i = warp; i < n; i += kThreads / 32) {
        if (children[i] == -1) continue;
        const int len = kv.seq_len[parents[i]], pages = pages_of(kv, len);
        const int32_t* from = entries_of(kv, parents[i]);
        int32_t* to = entries_of(kv, children[i]);
        for (int e = lane; e < pages; e += 32) {
            const int page = from[e];
            to[e] = page;
            atomicAdd(&kv.refs[page], 1);
        }
        if (lane == 0) kv.seq_len[children[i]] = len;
    }
}

__global__ void __launch_bounds__(kThreads)
    kv_trim_kernel(const KvView kv, const int32_t* __restrict__ slots,
                   const int32_t* __restrict__ keep, int n) {
    __shared__ PlanShared sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    plan_begin(kv, sh);
    for (int i = tid; i < n; i += kThreads) {
        const int slot = slots[i];
        if (slot == -1) continue;
        const int left = keep != nullptr ? keep[i] : 0;
        if (!claim_slot(kv, sh, slot) || !length_ok(kv, kv.seq_len[slot]) || left < 0 ||
            left > kv.seq_len[slot])
            sh.error = kInvalid;
    }
    __syncthreads();
    for (int i = warp; i < n && sh.error == 0; i += kThreads / 32) {
        if (slots[i] == -1) continue;
        const int pages = pages_of(kv, kv.seq_len[slots[i]]);
        for (int e = pages_of(kv, keep != nullptr ? keep[i] : 0) + lane; e < pages; e += 32)
            if (!page_ok(kv, entries_of(kv, slots[i])[e])) sh.error = kInvalid;
    }
    __syncthreads();
    if (sh.error != 0) {
        if (tid == 0) record_status(kv.status, sh.error);
        return;
    }
    for (int i = warp; i < n; i += kThreads / 32) {
        if (slots[i] == -1) continue;
        const int left = keep != nullptr ? keep[i] : 0;
        const int pages = pages_of(kv, kv.seq_len[slots[i]]);
        for (int e = pages_of(kv, left) + lane; e < pages; e += 32)
            atomicSub(&kv.refs[entries_of(kv, slots[i])[e]], 1);
        __syncwarp();
        if (lane == 0) kv.seq_len[slots[i]] = left;
    }
}

__global__ void __launch_bounds__(kThreads) kv_compact_kernel(const KvView kv) {
    __shared__ PlanShared sh;
    const Lists ls = lists_of(kv);
    const int tid = threadIdx.x;
    plan_begin(kv, sh);
    int live = 0;
    for (int p0 = 0; p0 < kv.num_pages; p0 += kThreads) {
        const int p = p0 + tid;
        live += __syncthreads_count(p < kv.num_pages && kv.refs[p] > 0);
    }
    // the sequences' entries are within range, or nothing moves
    for (int s = tid >> 5; s < kv.num_slots; s += kThreads / 32) {
        const int len = kv.seq_len[s];
        if (!length_ok(kv, len)) {
            sh.error = kInvalid;
            continue;
        }
        for (int e = tid & 31; e < pages_of(kv, len); e += 32)
            if (!page_ok(kv, entries_of(kv, s)[e])) sh.error = kInvalid;
    }
    __syncthreads();
    if (sh.error != 0) {
        if (tid == 0) {
            record_status(kv.status, sh.error);
            ls.head->copies = 0;
            ls.head->moved = -1;
        }
        return;
    }
    int movers = 0, holes = 0;
    for (int p0 = 0; p0 < kv.num_pages; p0 += kThreads) {
        const int p = p0 + tid;
        const bool used = p < kv.num_pages && kv.refs[p] > 0;
        const int mover = used && p >= live, hole = !used && p < live;
        int sum;
        const int m = block_scan(mover, sh, &sum);
        if (mover) ls.src[movers + m] = p;
        movers += sum;
        const int h = block_scan(hole, sh, &sum);
        if (hole) ls.dst[holes + h] = p;
        holes += sum;
    }
    __syncthreads();
    for (int c = tid; c < movers; c += kThreads) {
        const int from = ls.src[c], to = ls.dst[c];
        ls.b[from] = to;  // the map
        kv.refs[to] = kv.refs[from];
        kv.refs[from] = 0;
    }
    if (tid == 0) {
        ls.head->copies = movers;
        ls.head->moved = live;
    }
}

// The listed pages' tokens in every layer, and after a compaction the tables' entries.  A
// warp copies a head's tokens of one layer's keys or values, which lie in one run.
__global__ void __launch_bounds__(256) kv_copy_kernel(const KvView kv) {
    constexpr int kBatch = 8;  // 16-byte pieces that a thread has under way
    const Lists ls = lists_of(kv);
    grid_launch_dependents();
    grid_wait();
    const int lane = threadIdx.x & 31, T = 1 << kv.page_shift;
    const int64_t warp = blockIdx.x * 8 + (threadIdx.x >> 5), warps = gridDim.x * 8;
    const int copies = ls.head->copies, moved = ls.head->moved;
    const int64_t runs = static_cast<int64_t>(copies) * kv.layers * 2 * kv.kv_heads;
    for (int64_t w = warp; w < runs; w += warps) {
        const int head = static_cast<int>(w % kv.kv_heads);
        const int64_t rest = w / kv.kv_heads;
        const int which = static_cast<int>(rest & 1);
        const int layer = static_cast<int>((rest >> 1) % kv.layers);
        const int c = static_cast<int>((rest >> 1) / kv.layers);
        const int page = ls.src[c] & (kKvMaxPages - 1);
        const int tokens = moved >= 0 ? T : ls.src[c] >> kTokenShift;
        const uint4* from = reinterpret_cast<const uint4*>(
            kv.pages + kv_row(kv, layer, which, page, head, 0) * kv.row_bytes);
        uint4* to = reinterpret_cast<uint4*>(
            kv.pages + kv_row(kv, layer, which, ls.dst[c], head, 0) * kv.row_bytes);
        const int units = tokens * (kv.row_bytes / 16);
        for (int u0 = lane; u0 < units; u0 += 32 * kBatch) {
            uint4 v[kBatch];
#pragma unroll
            for (int b = 0; b < kBatch; ++b)
                if (u0 + 32 * b < units) v[b] = __ldcs(from + u0 + 32 * b);
#pragma unroll
            for (int b = 0; b < kBatch; ++b)
                if (u0 + 32 * b < units) __stcs(to + u0 + 32 * b, v[b]);
        }
        if (kv.exponents != nullptr && which == 0) {
            const uint16_t* ef = reinterpret_cast<const uint16_t*>(
                kv.exponents + kv_exponent(kv, layer, 0, page, head, 0));
            uint16_t* et = reinterpret_cast<uint16_t*>(
                kv.exponents + kv_exponent(kv, layer, 0, ls.dst[c], head, 0));
            for (int t = lane; t < tokens; t += 32) et[t] = ef[t];
        }
    }
    if (moved < 0) return;
    for (int64_t s = warp; s < kv.num_slots; s += warps) {
        const int pages = pages_of(kv, kv.seq_len[s]);
        int32_t* entry = entries_of(kv, static_cast<int>(s));
        for (int e = lane; e < pages; e += 32)
            if (entry[e] >= moved) entry[e] = ls.b[entry[e]];
    }
}

cudaError_t launch_copies(const KvView& kv, int sm_count, cudaStream_t stream) {
    return launch_overlapped(kv_copy_kernel, sm_count * 8, 256, 0, stream, kv);
}

}  // namespace

cudaError_t launch_kv_extend(const KvView& kv, const int32_t* slots, const int32_t* add, int n,
                             int sm_count, cudaStream_t stream) {
    const cudaError_t e = launch_overlapped(kv_extend_kernel, 1, kThreads, 0, stream, kv, slots, add, n);
    return e != cudaSuccess ? e : launch_copies(kv, sm_count, stream);
}

cudaError_t launch_kv_fork(const KvView& kv, const int32_t* parents, const int32_t* children, int n,
                           cudaStream_t stream) {
    return launch_overlapped(kv_fork_kernel, 1, kThreads, 0, stream, kv, parents, children, n);
}

cudaError_t launch_kv_trim(const KvView& kv, const int32_t* slots, const int32_t* keep, int n,
                           cudaStream_t stream) {
    return launch_overlapped(kv_trim_kernel, 1, kThreads, 0, stream, kv, slots, keep, n);
}

cudaError_t launch_kv_compact(const KvView& kv, int sm_count, cudaStream_t stream) {
    const cudaError_t e = launch_overlapped(kv_compact_kernel, 1, kThreads, 0, stream, kv);
    return e != cudaSuccess ? e : launch_copies(kv, sm_count, stream);
}

}  // namespace w4a16
