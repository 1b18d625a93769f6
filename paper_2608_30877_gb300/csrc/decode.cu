// Attention of one new token per sequence over the paged key-value cache.
//
// out = sum_j softmax_j(q . k_j / sqrt(128)) v_j in one pass over keys and values, with the
// running maximum and sum of the softmax in fp32.  It does 1 to 16 multiplications per byte,
// so HBM bounds it; the design keeps the memory busy whatever the batch looks like:
//
//  * Units.  The keys that a row sees, cut into tiles of 32 KB of keys and values (64 tokens
//    in bf16, 128 in e4m3), times the key heads, form one list over the whole batch, and
//    each CTA takes an equal run of it.  A row's length is thus split over as many CTAs as
//    its share of the bytes, and short rows share a CTA.  Everything follows from the
//    lengths on the device, so that a captured graph serves growing sequences.
//  * Stages.  One warp walks the run: it looks pages up in the table, and brings the pieces of
//    a tile by TMA into a ring of three stages (192 KB in flight on an SM's two CTAs), with
//    the row's queries and the new token's key and value.
//  * Products.  Four warps split a tile's keys, 16 at a time: S^T = K Q^T and O^T += V^T P^T by
//    warp-level MMAs whose A operand is the cache (16 keys or 16 values' dimensions) and whose
//    N = 8 columns are the queries of a key head, so that few queries waste few columns.  The
//    tensor pipe is nearly idle at this; the tcgen05 form would want 128 rows.  The warps'
//    maxima, sums and outputs are their own until the end of an item (row and head), where
//    they meet in the stage that was read last.
//  * More than 16 queries of a key head: the warps split the columns instead of the keys, up
//    to 64, then further items.
//  * Join.  A CTA's first and last items may continue in other CTAs: each then writes its
//    part to the workspace, and the last one to finish, found by a counter that wraps
//    to zero, adds them up in the order of the CTAs, so that the result has the same bits every time.
//
// 8-bit cache: codes are exact in fp16, where the products are taken.  A row of q is scaled by
// a power of two to the top of fp16's range; a key's exponent goes to its score; a value's
// exponent to its weight, and the weights that multiply the codes are relative to the largest
// of these products, whose running maximum a column keeps next to its scores'.
#include <cuda.h>
#include <cuda_runtime.h>
#include <cstdint>

#include "kv.h"
#include "kv_row.cuh"
#include "ptx.cuh"

namespace w4a16 {

namespace {

constexpr int kWarps = 4;                    // consumers
constexpr int kThreads = (kWarps + 1) * 32;  // and the producer
constexpr int kStages = 3;
constexpr int kHalfStage = 16384;            // a tile's keys, or its values
constexpr int kStageBytes = 2 * kHalfStage;
constexpr int kMaxCols = 64;                 // query columns of an item
constexpr int kCtasPerSm = 2;
constexpr int kInvalid = 1;                  // W4A16_ERR_INVALID_ARG
// e4m3: fp16 weights go up to 2^12, so that the least of them is 2^-36 of the largest
constexpr float kWeightTop = 12.0f;

// How the queries of a key head (the group) are laid over columns and warps.
struct Columns {
    int group;  // queries of a key head
    int block;  // columns of an item: 8, 16, 32 or 64
    int blocks; // items of a key head
    int warps;  // warps side by side in the columns: 1, 2 or 4
};
__host__ __device__ inline Columns columns_of(int group) {
    Columns c;
    c.group = group;
    c.block = group <= 8 ? 8 : group <= 16 ? 16 : group <= 32 ? 32 : kMaxCols;
    c.blocks = (group + c.block - 1) / c.block;
    c.warps = c.block <= 16 ? 1 : c.block / 16;
    return c;
}
__host__ __device__ inline int used_columns(int group) { return group < kMaxCols ? group : kMaxCols; }

// A part in the workspace: the outputs of its columns, then their sums, maxima, and the
// maxima that the outputs are relative to (e4m3; else the same).
__host__ __device__ inline int part_floats(int cols) { return cols * (kKvHeadDim + 3); }

// What the producer says about a stage.
struct Unit {
    int row, head, block, key0;  // the tile's first key
    int low, len;                // keys that the row sees
    int flags;
    int first_cta, parts;        // of the item, with kLast
    int page, at;                // the new token's place, with kNew
    int pad;
};
constexpr int kFirst = 1;    // the item's first unit in this CTA
constexpr int kLast = 2;     // and its last
constexpr int kNew = 4;      // the tile has the new token
constexpr int kBad = 8;      // a page index out of range
constexpr int kQSlotShift = 4;

struct Shared {
    uint64_t full[kStages], empty[kStages], met;
    Unit unit[kStages];
    alignas(16) uint16_t fresh[kStages][2][kKvHeadDim];           // the new token's key and value
    alignas(16) uint8_t exponents[kStages][2 * 128];  // e4m3: a tile's (key, value) pairs
    float part_l[kWarps][16], part_m[kWarps][16], part_w[kWarps][16];
    int64_t warp_sum[kThreads / 32];
    int64_t start_base;
    int start_row;
    int is_last;
    int abort;
};

struct DecodeArgs {
    KvView kv;
    DecodeParams p;
    Columns cols;
    int window;
};

__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t half_pair(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float bf16_lo(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t v) { return __uint_as_float(v & 0xFFFF0000u); }

__device__ __forceinline__ void ldsm_x4(uint32_t addr, uint32_t (&v)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3])
                 : "r"(addr)
                 : "memory");
}
__device__ __forceinline__ void ldsm_x4_trans(uint32_t addr, uint32_t (&v)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3])
                 : "r"(addr)
                 : "memory");
}
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t v) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
template <bool E4M3>
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (E4M3)
        asm volatile(
            "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
            "{%8, %9}, {%0, %1, %2, %3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile(
            "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
            "{%8, %9}, {%0, %1, %2, %3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// The consumers' barrier, bounded like every wait; false if the CTA gave up.
__device__ __forceinline__ bool consumers_meet(Shared& sh, uint32_t& phase, int* status, uint64_t wait_ns) {
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(smem_u32(&sh.met));
    const bool ok = wait_warp(smem_u32(&sh.met), phase, &sh.abort, status, wait_ns);
    phase ^= 1;
    return ok;
}
__device__ __forceinline__ void fence_proxy_async() {
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}
// Untiled copy; addresses and size multiples of 16 bytes.
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
        "l"(src), "r"(bytes), "r"(bar)
        : "memory");
}

// Byte of 16-byte unit `unit` of a tile's row in the 128-byte swizzle; a bf16 row is two
// halves of 128 bytes, a half tile of 64 rows apart.
template <bool E4M3>
__device__ __forceinline__ uint32_t tile_byte(int row, int unit) {
    const uint32_t base = E4M3 ? 0 : static_cast<uint32_t>(unit >> 3) * 8192u;
    return base + row * 128u + (((unit & 7) ^ (row & 7)) << 4);
}

// A row's slot and the keys it sees; no keys for padding, an empty sequence or bad data.
struct Row {
    int slot, len, low, first, tiles;  // first: its first tile
};
template <bool E4M3>
__device__ __forceinline__ Row row_of(const DecodeArgs& a, int i, bool* bad) {
    constexpr int kTile = E4M3 ? 128 : 64;
    Row r{a.p.slots[i], 0, 0, 0, 0};
    *bad = r.slot < -1 || r.slot >= a.kv.num_slots;
    if (*bad || r.slot < 0) return r;
    const int len = a.kv.seq_len[r.slot];
    *bad = len < 0 || len > static_cast<int64_t>(a.kv.max_pages) << a.kv.page_shift;
    if (*bad || len == 0) return r;
    r.len = len;
    r.low = len > a.window ? len - a.window : 0;
    r.first = r.low / kTile;
    r.tiles = (len - 1) / kTile + 1 - r.first;
    return r;
}

// The CTA whose run has unit u: runs start at c * units / ctas, rounded down.
__device__ __forceinline__ int cta_of(int64_t u, int64_t units, int64_t ctas) {
    return static_cast<int>(((u + 1) * ctas - 1) / units);
}

template <bool E4M3>
__device__ void produce(const DecodeArgs& a, const CUtensorMap* map, Shared& sh, uint32_t stages,
                        uint32_t queries, int64_t units, int64_t ctas, int64_t u0, int64_t u1) {
    constexpr int kTile = E4M3 ? 128 : 64;
    const KvView& kv = a.kv;
    const int lane = threadIdx.x & 31;
    const int box_shift = kv.page_shift < (E4M3 ? 7 : 6) ? kv.page_shift : (E4M3 ? 7 : 6);
    const int box_rows = 1 << box_shift;
    const int halves = E4M3 ? 1 : 2;
    const int boxes = (kTile >> box_shift) * halves * 2;  // of a stage, at most 16
    const int items = kv.kv_heads * a.cols.blocks;        // of a row
    const int64_t width = static_cast<int64_t>(a.p.H + 2 * kv.kv_heads) * kKvHeadDim;
    // this lane's box: values or keys, half of the row, place in the tile
    const int which = lane & 1, half = (lane >> 1) % halves, box = (lane >> 1) / halves;

    int row = sh.start_row;
    int64_t base = sh.start_base;
    bool bad;
    Row r = row_of<E4M3>(a, row, &bad);
    int item = static_cast<int>((u0 - base) / r.tiles);
    int tile = static_cast<int>((u0 - base) - static_cast<int64_t>(item) * r.tiles);
    int ids = 0, ids_from = -1, ids_row = -1;  // 32 entries of the row's page list, a lane each
    int slot = 0;             // of the item's queries
    int since[2] = {0, 0};    // units since the one that read each query slot; 0: none
    int st = 0;
    uint32_t phase = 0;       // of the stage's barriers
    int64_t issued = 0;
    for (int64_t u = u0; u < u1; ++u, ++issued) {
        const bool first = u == u0 || tile == 0;
        if (issued >= kStages &&
            !wait_warp(smem_u32(&sh.empty[st]), phase ^ 1, &sh.abort, kv.status, a.p.wait_ns))
            break;
        if (first) {
            // The unit that read this slot's queries before has to be released.  One that is
            // kStages back or more is: its stage, or a later one's, was waited for.
            const int back = since[slot];
            if (back > 0 && back < kStages) {
                const int v = st - back;
                if (!wait_warp(smem_u32(&sh.empty[v < 0 ? v + kStages : v]), v < 0 ? phase ^ 1 : phase,
                               &sh.abort, kv.status, a.p.wait_ns))
                    break;
            }
            since[slot] = 0;
        }
        const int key0 = (r.first + tile) * kTile;
        // page list entries of the tile; a page's boxes never cross it
        const int e0 = key0 >> kv.page_shift;
        const int e1 = (min(key0 + kTile, r.len) - 1) >> kv.page_shift;
        if (ids_row != row || e0 < ids_from || e1 >= ids_from + 32) {
            ids_row = row;
            ids_from = e0;
            const int e = e0 + lane;
            ids = e <= (r.len - 1) >> kv.page_shift
                      ? __ldg(kv.table + static_cast<int64_t>(r.slot) * kv.max_pages + e) : 0;
        }
        const int head = item / a.cols.blocks, block = item - head * a.cols.blocks;
        const int key = key0 + box * box_rows;  // of this lane's box
        const bool mine = lane < boxes && key < r.len && key + box_rows > r.low;
        const int id = __shfl_sync(0xffffffffu, ids, ((key >> kv.page_shift) - ids_from) & 31);
        const bool id_ok = id >= 0 && id < kv.num_pages;
        const bool tile_bad = __any_sync(0xffffffffu, mine && !id_ok);
        const int loads = __popc(__ballot_sync(0xffffffffu, mine));
        const bool fresh = key0 + kTile >= r.len;
        const int last_id = __shfl_sync(0xffffffffu, ids, (((r.len - 1) >> kv.page_shift) - ids_from) & 31);
        const bool last = u + 1 == u1 || tile + 1 == r.tiles;
        const uint32_t bar = smem_u32(&sh.full[st]);
        const int q_cols = min(a.cols.block, a.cols.group - block * a.cols.block);
        if (lane == 0) {
            Unit& t = sh.unit[st];
            t.row = row;
            t.head = head;
            t.block = block;
            t.key0 = key0;
            t.low = r.low;
            t.len = r.len;
            t.flags = (first ? kFirst : 0) | (last ? kLast : 0) | (fresh ? kNew : 0) | (tile_bad ? kBad : 0) |
                      slot << kQSlotShift;
            if (last) {
                const int64_t begin = base + static_cast<int64_t>(item) * r.tiles;
                t.first_cta = cta_of(begin, units, ctas);
                t.parts = cta_of(begin + r.tiles - 1, units, ctas) - t.first_cta + 1;
            }
            t.page = last_id >= 0 && last_id < kv.num_pages ? last_id : -1;
            t.at = (r.len - 1) & ((1 << kv.page_shift) - 1);
            mbar_arrive_expect_tx(bar, loads * (box_rows * 128u) + (first ? q_cols * 256u : 0u) +
                                           (fresh ? 512u : 0u));
            const uint16_t* qkv = a.p.qkv + row * width;
            if (first)
                bulk_load(queries + slot * a.cols.block * 256,
                          qkv + (static_cast<int64_t>(head) * a.cols.group + block * a.cols.block) * kKvHeadDim,
                          q_cols * 256, bar);
            if (fresh) {
                bulk_load(smem_u32(sh.fresh[st][0]), qkv + (a.p.H + head) * static_cast<int64_t>(kKvHeadDim), 256,
                          bar);
                bulk_load(smem_u32(sh.fresh[st][1]),
                          qkv + (a.p.H + kv.kv_heads + head) * static_cast<int64_t>(kKvHeadDim), 256, bar);
            }
        }
        __syncwarp();
        if (mine) {
            const int32_t at = key & ((1 << kv.page_shift) - 1);
            const int32_t c1 = static_cast<int32_t>(
                (((static_cast<int64_t>(which) * kv.num_pages + (id_ok ? id : 0)) * kv.kv_heads + head)
                 << kv.page_shift) + at);
            const uint32_t dst = stages + st * kStageBytes + which * kHalfStage + half * 8192u +
                                 box * box_rows * 128u;
            if (dbg_check(tma_box_ok(dst, box_rows * 128u, 1024, stages, stages + kStages * kStageBytes, half * 64,
                                     E4M3 ? 1 : 2), kv.status))
                tma_load_2d(dst, map, bar, half * 64, c1);
        }
        if constexpr (E4M3) {
            // (key, value) exponents, eight tokens to a lane; every lane arrives
            const int k8 = key0 + lane * 8;
            const int id8 = __shfl_sync(0xffffffffu, ids, ((k8 >> kv.page_shift) - ids_from) & 31);
            if (lane < kTile / 8 && k8 < r.len && k8 + 8 > r.low) {
                const int64_t from = kv_exponent(kv, a.p.layer, 0, id8 >= 0 && id8 < kv.num_pages ? id8 : 0, head,
                                                 k8 & ((1 << kv.page_shift) - 1));
                asm volatile("cp.async.ca.shared.global [%0], [%1], 16;" ::"r"(
                                 smem_u32(&sh.exponents[st][lane * 16])),
                             "l"(kv.exponents + from)
                             : "memory");
            }
            asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
        }
        if (issued == 0 && !short_limit_ok(bar, 0, &sh.abort, kv.status, a.p.wait_ns)) {
            ++issued;
            break;
        }
        // the next unit
        if (since[0] > 0 || (first && slot == 0)) ++since[0];
        if (since[1] > 0 || (first && slot == 1)) ++since[1];
        if (++st == kStages) {
            st = 0;
            phase ^= 1;
        }
        if (++tile == r.tiles) {
            tile = 0;
            slot ^= 1;
            if (++item == items && u + 1 < u1) {
                item = 0;
                base += static_cast<int64_t>(items) * r.tiles;
                do {  // (there are units left, so that a row has them)
                    r = row_of<E4M3>(a, ++row, &bad);
                } while (r.tiles == 0 && row + 1 < a.p.n);
                if (r.tiles == 0) {  // (unless the lengths changed during the call)
                    sh.abort = 1;
                    record_status(kv.status, kInvalid);
                    ++issued;
                    break;
                }
            }
        }
    }
    // the copies in flight, before the CTA may end (the consumers may have given up)
    for (int64_t i = issued > kStages ? issued - kStages : 0; i < issued; ++i)
        settle(smem_u32(&sh.full[i % kStages]), (i / kStages) & 1);
}

// The running softmax of a warp: two columns a thread in each of NT tiles of eight.
template <int NT>
struct State {
    float m[NT][2], l[NT][2], o[8][NT][4];
    float w[NT][2];  // e4m3: the largest score and value's exponent, which o is relative to
    bool bad;        // a page index was out of range
};

template <bool E4M3, int NT>
__device__ void consume(const DecodeArgs& a, Shared& sh, uint8_t* stage_mem, uint8_t* query_mem, int64_t u0,
                        int64_t u1) {
    constexpr int kTile = E4M3 ? 128 : 64;
    const KvView& kv = a.kv;
    const int lane = threadIdx.x & 31, warp = (threadIdx.x >> 5) - 1;
    const int g = lane >> 2, c = lane & 3;
    const int col_warp = warp % a.cols.warps, key_warp = warp / a.cols.warps, key_warps = kWarps / a.cols.warps;
    const float scale = a.p.scale * 1.4426950408889634f;
    State<NT> s;
    uint32_t q[8][NT][2];
    float q_scale[NT][2];  // of this thread's columns: the softmax's scale, and e4m3's of q
    int st = 0;
    uint32_t phase = 0, met = 0;
    for (int64_t u = u0; u < u1; ++u) {
        if (!wait_warp(smem_u32(&sh.full[st]), phase, &sh.abort, kv.status, a.p.wait_ns)) return;
        const Unit t = sh.unit[st];
        uint8_t* const tile = stage_mem + st * kStageBytes;
        const uint32_t keys = smem_u32(tile), values = keys + kHalfStage;
        if (t.flags & kFirst) {
            // Q as the B operand: column g of a tile of eight, in the order of K's dimensions
            const uint8_t* rows = query_mem + (t.flags >> kQSlotShift & 1) * a.cols.block * 256;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const uint8_t* row = rows + (col_warp * 8 * NT + nt * 8 + g) * 256;
                if constexpr (!E4M3) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        q[k][nt][0] = *reinterpret_cast<const uint32_t*>(row + k * 32 + c * 4);
                        q[k][nt][1] = *reinterpret_cast<const uint32_t*>(row + k * 32 + 16 + c * 4);
                    }
                    q_scale[nt][0] = q_scale[nt][1] = scale;
                } else {
                    uint2 v[8];
                    float top = 0.0f;
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        v[k] = *reinterpret_cast<const uint2*>(row + k * 32 + c * 8);
                        top = fmaxf(top, fmaxf(fmaxf(finite_abs(bf16_lo(v[k].x)), finite_abs(bf16_hi(v[k].x))),
                                               fmaxf(finite_abs(bf16_lo(v[k].y)), finite_abs(bf16_hi(v[k].y)))));
                    }
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                    // the largest to [2^14, 2^15): eight bits of mantissa stay exact down to 2^-31 of it
                    int e = static_cast<int>(__float_as_uint(top) >> 23) - 127 - 14;
                    e = e < -112 ? -112 : e;
                    const float f = power_of_two(-e);
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        q[k][nt][0] = half_pair(bf16_lo(v[k].x) * f, bf16_hi(v[k].x) * f);
                        q[k][nt][1] = half_pair(bf16_lo(v[k].y) * f, bf16_hi(v[k].y) * f);
                    }
                    // (column g's scale is needed by the threads of columns 2c and 2c + 1)
#pragma unroll
                    for (int j = 0; j < 2; ++j)
                        q_scale[nt][j] = scale * power_of_two(__shfl_sync(0xffffffffu, e, (2 * c + j) * 4));
                }
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 2; ++j) s.m[nt][j] = s.w[nt][j] = -INFINITY, s.l[nt][j] = 0.0f;
#pragma unroll
            for (int k = 0; k < 8; ++k)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int j = 0; j < 4; ++j) s.o[k][nt][j] = 0.0f;
            s.bad = false;
        }
        s.bad |= (t.flags & kBad) != 0;
        // The tile's ends: the new token's row is put in place, and values that no query sees
        // become zero (a weight of 0 does not keep a NaN out of a product).
        const bool edge = t.key0 < t.low || t.key0 + kTile >= t.len;
        if (edge) {
            for (int kg = warp; kg < kTile / 16; kg += kWarps) {
                const int k16 = t.key0 + kg * 16;
                if (k16 >= t.len || k16 + 16 <= t.low) continue;
                for (int i = lane; i < 16 * (E4M3 ? 8 : 16); i += 32) {
                    const int r = i >> (E4M3 ? 3 : 4), unit = i & (E4M3 ? 7 : 15);
                    if (k16 + r < t.low || k16 + r >= t.len)
                        *reinterpret_cast<uint4*>(tile + kHalfStage + tile_byte<E4M3>(kg * 16 + r, unit)) =
                            make_uint4(0, 0, 0, 0);
                }
                const int fresh = t.len - 1 - k16;
                if (fresh < 16 && fresh >= 0) {
                    const int r = kg * 16 + fresh;
                    const bool store = t.block == 0 && t.page >= 0 && !s.bad;
                    if constexpr (!E4M3) {
                        const int which = lane >> 4, unit = lane & 15;
                        const uint4 v = reinterpret_cast<const uint4*>(sh.fresh[st][which])[unit];
                        *reinterpret_cast<uint4*>(tile + which * kHalfStage + tile_byte<E4M3>(r, unit)) = v;
                        if (store)
                            reinterpret_cast<uint4*>(kv.pages)[kv_row(kv, a.p.layer, which, t.page, t.head, t.at) * 16 +
                                                               unit] = v;
                    } else {
#pragma unroll
                        for (int which = 0; which < 2; ++which) {
                            const uint2 v = reinterpret_cast<const uint2*>(sh.fresh[st][which])[lane];
                            float top = fmaxf(fmaxf(finite_abs(bf16_lo(v.x)), finite_abs(bf16_hi(v.x))),
                                              fmaxf(finite_abs(bf16_lo(v.y)), finite_abs(bf16_hi(v.y))));
#pragma unroll
                            for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                            const int e = e4m3_row_exponent(top);
                            const float f = power_of_two(-e);
                            const uint32_t codes = e4m3_quad(bf16_lo(v.x) * f, bf16_hi(v.x) * f, bf16_lo(v.y) * f,
                                                             bf16_hi(v.y) * f);
                            *reinterpret_cast<uint32_t*>(tile + which * kHalfStage + tile_byte<E4M3>(r, lane >> 2) +
                                                         (lane & 3) * 4) = codes;
                            if (lane == 0) sh.exponents[st][r * 2 + which] = static_cast<uint8_t>(e + 127);
                            if (store) {
                                reinterpret_cast<uint32_t*>(
                                    kv.pages)[kv_row(kv, a.p.layer, which, t.page, t.head, t.at) * 32 + lane] = codes;
                                if (lane == 0)
                                    kv.exponents[kv_exponent(kv, a.p.layer, which, t.page, t.head, t.at)] =
                                        static_cast<uint8_t>(e + 127);
                            }
                        }
                    }
                }
            }
            fence_proxy_async();  // (the stage's next contents come by TMA)
            __syncwarp();
            // others read what this warp mended
            if (a.cols.warps > 1 && !consumers_meet(sh, met, kv.status, a.p.wait_ns)) return;
        }
        for (int kg = key_warp; kg < kTile / 16; kg += key_warps) {
            const int k16 = t.key0 + kg * 16;
            if (k16 >= t.len || k16 + 16 <= t.low) continue;
            // scores of 16 keys: rows g and g + 8, columns 2c and 2c + 1
            float acc[2][NT][4];
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[i][nt][j] = 0.0f;
            if constexpr (!E4M3) {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    uint32_t f[4];
                    ldsm_x4(keys + tile_byte<E4M3>(kg * 16 + (lane & 15), 2 * k + (lane >> 4)), f);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma<E4M3>(acc[k & 1][nt], f, q[k][nt][0], q[k][nt][1]);
                }
            } else {
                // a 16-byte unit is 16 dimensions, of which a thread gets 4c .. 4c + 3
#pragma unroll
                for (int k = 0; k < 8; k += 2) {
                    uint32_t w[4];
                    ldsm_x4(keys + tile_byte<E4M3>(kg * 16 + (lane & 15), k + (lane >> 4)), w);
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const uint32_t f[4] = {e4m3_to_half2(static_cast<uint16_t>(w[2 * i])),
                                               e4m3_to_half2(static_cast<uint16_t>(w[2 * i + 1])),
                                               e4m3_to_half2(static_cast<uint16_t>(w[2 * i] >> 16)),
                                               e4m3_to_half2(static_cast<uint16_t>(w[2 * i + 1] >> 16))};
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) mma<E4M3>(acc[i][nt], f, q[k + i][nt][0], q[k + i][nt][1]);
                    }
                }
            }
            bool see[2] = {true, true};
            if (edge) {
                see[0] = k16 + g >= t.low && k16 + g < t.len;
                see[1] = k16 + g + 8 >= t.low && k16 + g + 8 < t.len;
            }
            float key_scale[2] = {1.0f, 1.0f}, value_exp[2] = {0.0f, 0.0f};
            if constexpr (E4M3) {
                const uint8_t* pairs = sh.exponents[st] + (kg * 16 + g) * 2;
                const uint32_t e0 = *reinterpret_cast<const uint16_t*>(pairs);
                const uint32_t e1 = *reinterpret_cast<const uint16_t*>(pairs + 16);
                key_scale[0] = __uint_as_float((e0 & 0xFFu) << 23);
                key_scale[1] = __uint_as_float((e1 & 0xFFu) << 23);
                value_exp[0] = static_cast<float>(static_cast<int>(e0 >> 8) - 127);
                value_exp[1] = static_cast<float>(static_cast<int>(e1 >> 8) - 127);
            }
            float alpha[NT][2];  // what the new maxima make of o
            uint32_t b[NT][2];
            bool moved = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float x[4], p[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float v = acc[0][nt][j] + acc[1][nt][j];
                    x[j] = see[j >> 1] ? v * (E4M3 ? key_scale[j >> 1] * q_scale[nt][j & 1] : q_scale[nt][j & 1])
                                       : -INFINITY;
                }
                // the running maximum of a column: v over the group's keys and what it was
                auto raise = [&](float v, float& was, float* scale_old) {
                    v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 4));
                    v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 8));
                    v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 16));
                    v = fmaxf(v, was);
                    const float base = v == -INFINITY ? 0.0f : v;
                    *scale_old = ex2(was - base);
                    moved |= v != was;
                    was = v;
                    return base;
                };
                float scale_l[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float base = raise(fmaxf(x[j], x[j + 2]), s.m[nt][j], &scale_l[j]);
                    p[j] = ex2(x[j] - base);
                    p[j + 2] = ex2(x[j + 2] - base);
                    alpha[nt][j] = scale_l[j];
                }
                // keys 2c, 2c + 1 of column g: the transpose of what this thread holds
                uint32_t w0, w1;
                if constexpr (!E4M3) {
                    w0 = bf16_pair(p[0], p[1]);
                    w1 = bf16_pair(p[2], p[3]);
                    // (the sum of the rounded weights, so that they add up to one)
                    s.l[nt][0] = s.l[nt][0] * scale_l[0] + (bf16_lo(w0) + bf16_lo(w1));
                    s.l[nt][1] = s.l[nt][1] * scale_l[1] + (bf16_hi(w0) + bf16_hi(w1));
                } else {
                    s.l[nt][0] = s.l[nt][0] * scale_l[0] + (p[0] + p[2]);
                    s.l[nt][1] = s.l[nt][1] * scale_l[1] + (p[1] + p[3]);
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        // (an unseen key's score is -inf whatever its exponent)
                        const float y0 = x[j] + value_exp[0], y1 = x[j + 2] + value_exp[1];
                        const float base = raise(fmaxf(y0, y1), s.w[nt][j], &alpha[nt][j]) - kWeightTop;
                        p[j] = ex2(y0 - base);
                        p[j + 2] = ex2(y1 - base);
                    }
                    w0 = half_pair(p[0], p[1]);
                    w1 = half_pair(p[2], p[3]);
                }
                b[nt][0] = transpose_8x8(w0);
                b[nt][1] = transpose_8x8(w1);
            }
            if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
                for (int k = 0; k < 8; ++k)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int j = 0; j < 4; ++j) s.o[k][nt][j] *= alpha[nt][j & 1];
            }
            if constexpr (!E4M3) {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    uint32_t f[4];
                    ldsm_x4_trans(values + tile_byte<E4M3>(kg * 16 + (lane & 7) + ((lane >> 4) << 3),
                                                           2 * k + (lane >> 3 & 1)), f);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma<E4M3>(s.o[k][nt], f, b[nt][0], b[nt][1]);
                }
            } else {
                // rows g and g + 8 of a tile are dimensions 2g and 2g + 1 of its 16
#pragma unroll
                for (int k = 0; k < 8; k += 2) {
                    uint32_t w[4];
                    ldsm_x4_trans(values + tile_byte<E4M3>(kg * 16 + (lane & 15), k + (lane >> 4)), w);
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const uint32_t lo = __byte_perm(w[2 * i], 0, 0x3120);
                        const uint32_t hi = __byte_perm(w[2 * i + 1], 0, 0x3120);
                        const uint32_t f[4] = {e4m3_to_half2(static_cast<uint16_t>(lo)),
                                               e4m3_to_half2(static_cast<uint16_t>(lo >> 16)),
                                               e4m3_to_half2(static_cast<uint16_t>(hi)),
                                               e4m3_to_half2(static_cast<uint16_t>(hi >> 16))};
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) mma<E4M3>(s.o[k + i][nt], f, b[nt][0], b[nt][1]);
                    }
                }
            }
        }
        if (t.flags & kLast) {
            // The warps' parts meet in the stage, which all have read: [warp][16 columns][128],
            // a column turned by eight values per pair so that a store's lanes hit all banks.
            float* const meet = reinterpret_cast<float*>(tile);
            if (!consumers_meet(sh, met, kv.status, a.p.wait_ns)) return;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    float l = s.l[nt][j];
                    l += __shfl_xor_sync(0xffffffffu, l, 4);
                    l += __shfl_xor_sync(0xffffffffu, l, 8);
                    l += __shfl_xor_sync(0xffffffffu, l, 16);
                    const int col = nt * 8 + 2 * c + j;
                    if (g == 0) {
                        sh.part_l[warp][col] = l;
                        sh.part_m[warp][col] = s.m[nt][j];
                        sh.part_w[warp][col] = E4M3 ? s.w[nt][j] : s.m[nt][j];
                    }
#pragma unroll
                    for (int k = 0; k < 8; ++k)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const int d = E4M3 ? 16 * k + 2 * g + i : 16 * k + g + 8 * i;
                            meet[(warp * 8 * NT + col) * kKvHeadDim + ((d + 8 * (col >> 1)) & 127)] =
                                s.o[k][nt][2 * i + j];
                        }
                }
            if (!consumers_meet(sh, met, kv.status, a.p.wait_ns)) return;
            const int tid = threadIdx.x - 32, d = tid;  // a thread to a dimension
            const int cols = min(a.cols.block, a.cols.group - t.block * a.cols.block);
            const int max_cols = used_columns(a.cols.group);
            float* const parts = reinterpret_cast<float*>(
                static_cast<uint8_t*>(a.p.workspace) + static_cast<int64_t>(gridDim.x) * 4);
            const int64_t stride = part_floats(max_cols);
            const bool whole = t.parts == 1;
            float* const part =
                parts + (2 * static_cast<int64_t>(blockIdx.x) + (t.first_cta == static_cast<int>(blockIdx.x))) * stride;
            uint16_t* const out =
                a.p.out + (static_cast<int64_t>(t.row) * a.p.H + static_cast<int64_t>(t.head) * a.cols.group +
                           t.block * a.cols.block) * kKvHeadDim;
            auto finite = [](float m) { return m == -INFINITY ? 0.0f : m; };
            // an output from its sum, relative to 2^w, and the weights' sum, relative to 2^m
            auto output = [&](float o, float l, float m, float w, bool bad) {
                float v = o / l;
                // (in two steps: an exponent may be -120, and ex2 flushes below 2^-126)
                if constexpr (E4M3) v = v * ex2(-kWeightTop) * ex2(finite(w) - finite(m));
                return bad ? uint16_t{0} : static_cast<uint16_t>(bf16_pair(v, 0.0f));
            };
            for (int col = 0; col < cols; ++col) {
                const int cw = col / (8 * NT), in = col - cw * 8 * NT;
                float m = -INFINITY, w = -INFINITY, l = 0.0f, o = 0.0f;
                for (int k = 0; k < key_warps; ++k) {
                    m = fmaxf(m, sh.part_m[k * a.cols.warps + cw][in]);
                    w = fmaxf(w, sh.part_w[k * a.cols.warps + cw][in]);
                }
                for (int k = 0; k < key_warps; ++k) {
                    const int i = k * a.cols.warps + cw;
                    l += ex2(sh.part_m[i][in] - finite(m)) * sh.part_l[i][in];
                    o += ex2(sh.part_w[i][in] - finite(w)) *
                         meet[(i * 8 * NT + in) * kKvHeadDim + ((d + 8 * (in >> 1)) & 127)];
                }
                if (whole) {
                    out[col * kKvHeadDim + d] = output(o, l, m, w, s.bad);
                } else {
                    part[col * kKvHeadDim + d] = o;
                    if (d == 0) {
                        float* const stats = part + max_cols * kKvHeadDim + col;
                        stats[0] = s.bad ? -1.0f : l;  // (a sum is never negative: marks a bad page index)
                        stats[max_cols] = m;
                        stats[2 * max_cols] = w;
                    }
                }
            }
            if (whole) {
                if (s.bad && tid == 0) record_status(kv.status, kInvalid);
            } else {
                __threadfence();
                if (!consumers_meet(sh, met, kv.status, a.p.wait_ns)) return;
                if (tid == 0) {
                    unsigned int* const count = static_cast<unsigned int*>(a.p.workspace) + t.first_cta;
                    sh.is_last = atomicInc(count, t.parts - 1) == static_cast<unsigned int>(t.parts - 1);
                }
                if (!consumers_meet(sh, met, kv.status, a.p.wait_ns)) return;
                if (sh.is_last) {
                    __threadfence();
                    // part k is of CTA first_cta + k: its last item for k = 0, else its first
                    auto at = [&](int k) {
                        return parts + (2 * static_cast<int64_t>(t.first_cta + k) + (k == 0)) * stride;
                    };
                    for (int col = 0; col < cols; ++col) {
                        const int stats = max_cols * kKvHeadDim + col;
                        float m = -INFINITY, w = -INFINITY, l = 0.0f, o = 0.0f;
                        bool bad = false;
                        for (int k = 0; k < t.parts; ++k) {
                            m = fmaxf(m, __ldcg(at(k) + stats + max_cols));
                            w = fmaxf(w, __ldcg(at(k) + stats + 2 * max_cols));
                        }
                        for (int k = 0; k < t.parts; ++k) {
                            const float pl = __ldcg(at(k) + stats);
                            bad |= pl < 0.0f;
                            l += ex2(__ldcg(at(k) + stats + max_cols) - finite(m)) * pl;
                            o += ex2(__ldcg(at(k) + stats + 2 * max_cols) - finite(w)) *
                                 __ldcg(at(k) + col * kKvHeadDim + d);
                        }
                        out[col * kKvHeadDim + d] = output(o, l, m, w, bad);
                        if (bad && tid == 0) record_status(kv.status, kInvalid);
                    }
                }
            }
            fence_proxy_async();
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&sh.empty[st]));
        if (++st == kStages) {
            st = 0;
            phase ^= 1;
        }
    }
}

template <bool E4M3, int NT>
__global__ void __launch_bounds__(kThreads, kCtasPerSm)
    attention_decode_kernel(const __grid_constant__ CUtensorMap map, const DecodeArgs a) {
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ Shared sh;
    // (the dynamic part starts past the static one: rounded up to the swizzle's 1024 bytes)
    const uint32_t raw = smem_u32(smem), up = (1024 - (raw & 1023)) & 1023;
    uint8_t* const stage_mem = smem + up;
    uint8_t* const query_mem = stage_mem + kStages * kStageBytes;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) {
        prefetch_tmap(&map);
        for (int i = 0; i < kStages; ++i) {
            mbar_init(smem_u32(&sh.full[i]), E4M3 ? 33 : 1);
            mbar_init(smem_u32(&sh.empty[i]), kWarps);
        }
        mbar_init(smem_u32(&sh.met), kWarps);
        sh.abort = 0;
        fence_mbar_init();
    }
    grid_launch_dependents();
    grid_wait();
    __syncthreads();

    // the batch's units, this CTA's run of them, and the row and its first unit where it starts
    const int items = a.kv.kv_heads * a.cols.blocks;
    int64_t units = 0;
    for (int i0 = 0; i0 < a.p.n; i0 += kThreads) {
        const int i = i0 + tid;
        int64_t v = 0;
        if (i < a.p.n) {
            bool bad;
            const Row r = row_of<E4M3>(a, i, &bad);
            v = static_cast<int64_t>(r.tiles) * items;
            if (i % gridDim.x == blockIdx.x && bad) record_status(a.kv.status, kInvalid);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        if (lane == 0) sh.warp_sum[warp] = v;
        __syncthreads();
        for (int w = 0; w < kThreads / 32; ++w) units += sh.warp_sum[w];
        __syncthreads();
    }
    // rows without keys are zero
    for (int i = blockIdx.x; i < a.p.n; i += gridDim.x) {
        bool bad;
        if (row_of<E4M3>(a, i, &bad).tiles > 0) continue;
        uint4* const out = reinterpret_cast<uint4*>(a.p.out + static_cast<int64_t>(i) * a.p.H * kKvHeadDim);
        for (int j = tid; j < a.p.H * (kKvHeadDim / 8); j += kThreads) out[j] = make_uint4(0, 0, 0, 0);
    }
    const int64_t ctas = units < gridDim.x ? units : gridDim.x;
    if (blockIdx.x >= ctas) return;
    const int64_t u0 = blockIdx.x * units / ctas, u1 = (blockIdx.x + 1) * units / ctas;
    int64_t before = 0;
    for (int i0 = 0; i0 < a.p.n && before <= u0; i0 += kThreads) {
        const int i = i0 + tid;
        int64_t v = 0;
        if (i < a.p.n) {
            bool bad;
            v = static_cast<int64_t>(row_of<E4M3>(a, i, &bad).tiles) * items;
        }
        int64_t sum = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t t = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += t;
        }
        if (lane == 31) sh.warp_sum[warp] = sum;
        __syncthreads();
        int64_t all = 0;
        for (int w = 0; w < kThreads / 32; ++w) {
            if (w == warp) sum += all + before;
            all += sh.warp_sum[w];
        }
        if (u0 < sum && u0 >= sum - v) {
            sh.start_row = i;
            sh.start_base = sum - v;
        }
        before += all;
        __syncthreads();
    }
    if (warp == 0)
        produce<E4M3>(a, &map, sh, smem_u32(stage_mem), smem_u32(query_mem), units, ctas, u0, u1);
    else
        consume<E4M3, NT>(a, sh, stage_mem, query_mem, u0, u1);
}

template <bool E4M3, int NT>
cudaError_t launch(const CUtensorMap& map, const DecodeArgs& a, int grid, cudaStream_t stream) {
    auto kern = attention_decode_kernel<E4M3, NT>;
    const int bytes = 1024 + kStages * kStageBytes + 2 * a.cols.block * 256;
    cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = kThreads;
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, kern, map, a);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

// A counter for each CTA, then two parts for each.
int64_t decode_workspace_bytes(int H, int kv_heads, int sm_count) {
    const int64_t ctas = static_cast<int64_t>(sm_count) * kCtasPerSm;
    const int64_t bytes = ctas * 4 + ctas * 2 * part_floats(used_columns(H / kv_heads)) * 4;
    return (bytes + 15) / 16 * 16;
}

int encode_cache(CUtensorMap* map, const KvView& kv, int layer) {
    const bool e4m3 = kv.exponents != nullptr;
    const int64_t rows = static_cast<int64_t>(2) * kv.num_pages * kv.kv_heads << kv.page_shift;
    const int most = e4m3 ? 128 : 64, tokens = 1 << kv.page_shift;
    return encode_rows(map, e4m3 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16,
                          kv.pages + layer * rows * kv.row_bytes, kKvHeadDim, rows, kv.row_bytes,
                          e4m3 ? 128 : 64, tokens < most ? tokens : most);
}

cudaError_t launch_attention_decode(const CUtensorMap& map, const KvView& kv, const DecodeParams& p, int sm_count,
                                    cudaStream_t stream) {
    const DecodeArgs a{kv, p, columns_of(p.H / kv.kv_heads), p.window};
    const int grid = sm_count * kCtasPerSm;
    const bool e4m3 = kv.exponents != nullptr, wide = a.cols.block > 8;
    return e4m3 ? (wide ? launch<true, 2>(map, a, grid, stream) : launch<true, 1>(map, a, grid, stream))
                : (wide ? launch<false, 2>(map, a, grid, stream) : launch<false, 1>(map, a, grid, stream));
}

}  // namespace w4a16
