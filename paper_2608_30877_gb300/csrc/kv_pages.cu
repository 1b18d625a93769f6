// Page operations of the key-value cache: growth with copy on write, sharing, release
// and compaction.
//
// A page is free if no sequence refers to it; the free pages are found by scanning the
// reference counts, lowest index first, so there is no list to keep in step with them and
// every result is a function of the tables alone (integer atomics commute).  Each
// operation runs its checks before its first change, so an error leaves the cache as it was; growth
// that is refused marks its slots in the scratch buffer, and what would store the tokens
// that were not added (writes, decode attention) leaves marked slots alone.
// One CTA plans; what has to be copied (an extend's shared last pages, a compaction's
// moved pages) goes to a list in the scratch buffer that a second kernel works off over
// the whole GPU.  Bound by latency but for the copies, which HBM bounds: a thread takes a list
// entry and all pages of a chunk of entries are worked off side by side, so that a call is a
// chain of four or five loads (with a warp for each entry, one after another, 512 sequences
// took 11 us a call).
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
    int32_t *src, *dst;     // what the copy kernel copies
    int32_t *offset, *copy; // growth, by entry: its first allocated page, its page to copy or -1
    int32_t* page;          // growth: the free pages; compaction: where a page has gone
};
__device__ __forceinline__ Lists lists_of(const KvView& kv) {
    const int n = kv_scratch_list(kv.num_pages, kv.num_slots);
    int32_t* p = kv.scratch + kKvScratchHeader;
    return {reinterpret_cast<KvScratch*>(kv.scratch), p, p + n, p + 2 * n, p + 3 * n, p + 4 * n};
}

struct PlanShared {
    uint32_t seen[kKvMaxSlots / 32];
    int64_t warp[kThreads / 32];
    int error;
    int copies;
    // a chunk of list entries: slot, first page entry, and where its pages start among the chunk's
    int slot[kThreads], other[kThreads], first[kThreads], start[kThreads];
    int large[kThreads], larges;
};

// Sum over the CTA's threads before this one, and the total; all threads call it.
__device__ __forceinline__ int64_t block_scan(int64_t v, PlanShared& sh, int64_t* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int64_t inc = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t t = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += t;
    }
    if (lane == 31) sh.warp[warp] = inc;
    __syncthreads();
    if (warp == 0) {
        int64_t w = sh.warp[lane];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t t = __shfl_up_sync(0xffffffffu, w, o);
            if (lane >= o) w += t;
        }
        sh.warp[lane] = w;
    }
    __syncthreads();
    const int64_t before = warp > 0 ? sh.warp[warp - 1] : 0;
    *total = sh.warp[kThreads / 32 - 1];
    __syncthreads();
    return before + inc - v;
}

// Calls use(k, e, load(k, e)) for page entry e of chunk entry k, over the pages [first, first +
// count) of each thread's chunk entry (of `entries`).  Where an entry has 16 pages or more on
// average a warp takes an entry, else the pages are spread evenly over the CTA by a search for
// each (64 entries of 63 pages 9 us a call against 12, 512 of at most one 8 against 11);
// kSide of a thread's searches and loads are under way together.
template <typename Load, typename Use>
__device__ __forceinline__ void each_page(PlanShared& sh, int first, int count, int entries, Load load, Use use) {
    constexpr int kSide = 4;
    int64_t all;
    const int before = static_cast<int>(block_scan(count, sh, &all));
    const int total = static_cast<int>(all);  // (at most the page table's entries)
    sh.first[threadIdx.x] = first;
    sh.start[threadIdx.x] = before;
    __syncthreads();
    if (total >= 16 * static_cast<int64_t>(entries)) {
        for (int k = threadIdx.x >> 5; k < entries; k += kThreads / 32) {
            const int from = sh.first[k], n = (k + 1 < kThreads ? sh.start[k + 1] : total) - sh.start[k];
            for (int e0 = threadIdx.x & 31; e0 < n; e0 += 32 * kSide) {
                int page[kSide];
#pragma unroll
                for (int s = 0; s < kSide; ++s)
                    if (e0 + 32 * s < n) page[s] = load(k, from + e0 + 32 * s);
#pragma unroll
                for (int s = 0; s < kSide; ++s)
                    if (e0 + 32 * s < n) use(k, from + e0 + 32 * s, page[s]);
            }
        }
        __syncthreads();
        return;
    }
    for (int64_t r0 = threadIdx.x; r0 < total; r0 += kThreads * kSide) {
        int k[kSide], e[kSide], page[kSide];
#pragma unroll
        for (int s = 0; s < kSide; ++s) k[s] = 0;
        // the last entry that starts at r or before
        for (int step = kThreads / 2; step > 0; step >>= 1)
#pragma unroll
            for (int s = 0; s < kSide; ++s)
                if (sh.start[k[s] + step] <= r0 + s * kThreads) k[s] += step;
#pragma unroll
        for (int s = 0; s < kSide; ++s) {
            const int r = static_cast<int>(r0) + s * kThreads;
            e[s] = sh.first[k[s]] + r - sh.start[k[s]];
            if (r < total) page[s] = load(k[s], e[s]);
        }
#pragma unroll
        for (int s = 0; s < kSide; ++s)
            if (r0 + s * kThreads < total) use(k[s], e[s], page[s]);
    }
    __syncthreads();
}

// Whether an entry has been found wrong.  All threads call it before each pass over the lists: the pass
// may set the flag, so no thread begins one before every thread has read it.
__device__ __forceinline__ bool plan_failed(const PlanShared& sh) { return __syncthreads_or(sh.error) != 0; }

__device__ __forceinline__ void plan_begin(const KvView& kv, PlanShared& sh) {
    for (int i = threadIdx.x; i < (kv.num_slots + 31) / 32; i += kThreads) sh.seen[i] = 0;
    if (threadIdx.x == 0) sh.error = sh.copies = sh.larges = 0;
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

// A slot's mark, set or taken away; `any`: whether there was one when the call began.
__device__ __forceinline__ void mark_refused(const KvView& kv, int slot) {
    if (atomicExch(&kv.refused[slot], kKvRefused) != kKvRefused) atomicAdd(&lists_of(kv).head->refused, 1);
}
__device__ __forceinline__ void unmark(const KvView& kv, bool any, int slot) {
    if (any && atomicExch(&kv.refused[slot], 0) == kKvRefused) atomicSub(&lists_of(kv).head->refused, 1);
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
    kv_extend_kernel(const KvView kv, const int32_t* slots,
                     const int32_t* add, int n) {
    __shared__ PlanShared sh;
    const Lists ls = lists_of(kv);
    const int tid = threadIdx.x;
    plan_begin(kv, sh);
    // kRun counts a thread and pass: a pool of 16000 pages takes one, under way from the start
    constexpr int kRun = 16;
    auto load_run = [&](int p0, int4 (&v)[kRun / 4]) {
        const int begin = p0 + tid * kRun;
#pragma unroll
        for (int k = 0; k < kRun / 4; ++k) {
            v[k] = make_int4(1, 1, 1, 1);
            if (begin + 4 * k + 4 <= kv.num_pages) {
                v[k] = reinterpret_cast<const int4*>(kv.refs + begin)[k];
            } else {
                const int left = kv.num_pages - begin - 4 * k;
                if (left > 0) v[k].x = kv.refs[begin + 4 * k];
                if (left > 1) v[k].y = kv.refs[begin + 4 * k + 1];
                if (left > 2) v[k].z = kv.refs[begin + 4 * k + 2];
            }
        }
    };
    int4 run[kRun / 4];
    load_run(0, run);
    const bool any = any_refused(kv);
    // pages that each entry needs, as offsets into the pages to allocate
    int64_t need_all = 0;
    for (int i0 = 0; i0 < n; i0 += kThreads) {
        const int i = i0 + tid;
        int need = 0, copy = -1;
        if (i < n && slots[i] != -1) {
            const int slot = slots[i], grow = add[i];
            int error = 0;
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
        int64_t sum;
        const int64_t before = need_all + block_scan(need, sh, &sum);
        if (i < n) {
            ls.offset[i] = static_cast<int>(before < kv.num_pages ? before : kv.num_pages);
            ls.copy[i] = copy;
        }
        need_all += sum;
    }
    // the lowest free pages, in order
    int64_t found = 0;
    for (int p0 = 0; p0 < kv.num_pages && found < need_all && need_all <= kv.num_pages; p0 += kThreads * kRun) {
        if (p0 > 0) load_run(p0, run);
        uint32_t free = 0;
#pragma unroll
        for (int k = 0; k < kRun / 4; ++k)
            free |= ((run[k].x == 0) | (run[k].y == 0) << 1 | (run[k].z == 0) << 2 | (run[k].w == 0) << 3) << 4 * k;
        int64_t sum;
        int64_t rank = found + block_scan(__popc(free), sh, &sum);
        for (; free != 0 && rank < need_all; free &= free - 1, ++rank)
            ls.page[rank] = p0 + tid * kRun + __ffs(free) - 1;
        found += sum;
    }
    __syncthreads();
    if (sh.error != 0 || found < need_all) {
        // what follows in the same step stores nothing for the sequences that were to grow
        for (int i = tid; i < n; i += kThreads)
            if (slots[i] >= 0 && slots[i] < kv.num_slots && add[i] != 0) mark_refused(kv, slots[i]);
        if (tid == 0) {
            record_status(kv.status, sh.error != 0 ? sh.error : kCapacity);
            ls.head->copies = 0;
            ls.head->moved = -1;
        }
        return;
    }
    // nothing above has changed the cache; each entry's pages, many of them by the whole CTA
    constexpr int kOwn = 16;
    for (int i0 = 0; i0 < n; i0 += kThreads) {
        const int i = i0 + tid;
        if (i < n && slots[i] != -1) {
            const int slot = slots[i], len = kv.seq_len[slot], to = len + add[i];
            const int offset = ls.offset[i], copy = ls.copy[i];
            const int first = pages_of(kv, len) - (copy >= 0), need = pages_of(kv, to) - first;
            if (copy >= 0) {
                const int c = atomicAdd(&sh.copies, 1);  // (the copies' order does not matter)
                ls.src[c] = copy | (len & ((1 << kv.page_shift) - 1)) << kTokenShift;
                ls.dst[c] = ls.page[offset];
                atomicSub(&kv.refs[copy], 1);
            }
            for (int k = 0; k < need && k < kOwn; ++k) {
                const int page = ls.page[offset + k];
                entries_of(kv, slot)[first + k] = page;
                kv.refs[page] = 1;
            }
            if (need > kOwn) {
                const int l = atomicAdd(&sh.larges, 1);
                sh.slot[l] = slot;
                sh.first[l] = first;
                sh.start[l] = offset;
                sh.large[l] = need;
            }
            kv.seq_len[slot] = to;
            unmark(kv, any, slot);
        }
        __syncthreads();
        for (int l = 0; l < sh.larges; ++l)
            for (int k = kOwn + tid; k < sh.large[l]; k += kThreads) {
                const int page = ls.page[sh.start[l] + k];
                entries_of(kv, sh.slot[l])[sh.first[l] + k] = page;
                kv.refs[page] = 1;
            }
        __syncthreads();
        if (tid == 0) sh.larges = 0;
        __syncthreads();
    }
    if (tid == 0) {
        ls.head->copies = sh.copies;
        ls.head->moved = -1;
    }
}

__global__ void __launch_bounds__(kThreads)
    kv_fork_kernel(const KvView kv, const int32_t* parents,
                   const int32_t* children, int n) {
    __shared__ PlanShared sh;
    const int tid = threadIdx.x;
    plan_begin(kv, sh);
    const bool any = any_refused(kv);
    for (int i = tid; i < n; i += kThreads) {
        if (children[i] == -1) continue;
        const int parent = parents[i];
        if (!claim_slot(kv, sh, children[i]) || kv.seq_len[children[i]] != 0 || parent < 0 ||
            parent >= kv.num_slots || !length_ok(kv, kv.seq_len[parent]))
            sh.error = kInvalid;
    }
    __syncthreads();
    // checks every page, then shares them; a chunk of entries at a time
    for (int pass = 0; pass < 2 && !plan_failed(sh); ++pass) {
        for (int i0 = 0; i0 < n; i0 += kThreads) {
            const int i = i0 + tid;
            int len = 0, child = -1;
            if (i < n && children[i] != -1) {
                const int parent = parents[i];
                child = children[i];
                // (a parent that is a child of this call)
                if (sh.seen[parent >> 5] >> (parent & 31) & 1) sh.error = kInvalid;
                len = kv.seq_len[parent];
                sh.slot[tid] = parent;
                sh.other[tid] = child;
            }
            auto load = [&](int k, int e) { return entries_of(kv, sh.slot[k])[e]; };
            each_page(sh, 0, pages_of(kv, len), min(n - i0, kThreads), load, [&](int k, int e, int page) {
                if (pass == 0) {
                    if (!page_ok(kv, page)) sh.error = kInvalid;
                } else {
                    entries_of(kv, sh.other[k])[e] = page;
                    atomicAdd(&kv.refs[page], 1);
                }
            });
            if (pass == 1 && child >= 0) {
                kv.seq_len[child] = len;
                unmark(kv, any, child);
            }
        }
    }
    if (sh.error != 0 && tid == 0) record_status(kv.status, sh.error);
}

__global__ void __launch_bounds__(kThreads)
    kv_trim_kernel(const KvView kv, const int32_t* slots,
                   const int32_t* keep, int n) {
    __shared__ PlanShared sh;
    const int tid = threadIdx.x;
    plan_begin(kv, sh);
    const bool any = any_refused(kv);
    // checks every entry and page, then gives the pages back; a chunk of entries at a time
    for (int pass = 0; pass < 2 && !plan_failed(sh); ++pass) {
        for (int i0 = 0; i0 < n; i0 += kThreads) {
            const int i = i0 + tid;
            int first = 0, count = 0, slot = -1, left = 0;
            if (i < n && slots[i] != -1) {
                slot = slots[i];
                left = keep != nullptr ? keep[i] : 0;
                if (pass == 0 && !claim_slot(kv, sh, slot)) {
                    sh.error = kInvalid;
                } else {
                    const int len = kv.seq_len[slot];
                    if (!length_ok(kv, len) || left < 0 || left > len) {
                        sh.error = kInvalid;
                    } else {
                        first = pages_of(kv, left);
                        count = pages_of(kv, len) - first;
                    }
                }
                sh.slot[tid] = slot;
            }
            auto load = [&](int k, int e) { return entries_of(kv, sh.slot[k])[e]; };
            each_page(sh, first, count, min(n - i0, kThreads), load, [&](int, int, int page) {
                if (pass == 0) {
                    if (!page_ok(kv, page)) sh.error = kInvalid;
                } else {
                    atomicSub(&kv.refs[page], 1);
                }
            });
            if (pass == 1 && slot >= 0) {
                kv.seq_len[slot] = left;
                unmark(kv, any, slot);
            }
        }
    }
    if (sh.error != 0 && tid == 0) record_status(kv.status, sh.error);
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
        int64_t sum;
        // (both counts in one scan: a pass has at most kThreads of each)
        const int64_t before = block_scan(mover + (static_cast<int64_t>(hole) << 32), sh, &sum);
        if (mover) ls.src[movers + static_cast<int>(before & 0xFFFFFFFF)] = p;
        if (hole) ls.dst[holes + static_cast<int>(before >> 32)] = p;
        movers += static_cast<int>(sum & 0xFFFFFFFF);
        holes += static_cast<int>(sum >> 32);
    }
    __syncthreads();
    for (int c = tid; c < movers; c += kThreads) {
        const int from = ls.src[c], to = ls.dst[c];
        ls.page[from] = to;
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
                if (u0 + 32 * b < units) v[b] = __ldcg(from + u0 + 32 * b);
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
            if (entry[e] >= moved) entry[e] = ls.page[entry[e]];
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
