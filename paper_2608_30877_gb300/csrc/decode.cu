// Attention of one new token per sequence over the paged key-value cache.
//
// out = sum_j softmax_j(q . k_j / sqrt(128)) v_j in one pass over keys and values, with the
// running maximum and sum of the softmax in fp32.  It does 1 to 16 multiplications per byte,
// so HBM bounds it; the design keeps the memory busy whatever the batch looks like:
//
//  * Units.  The keys that a row sees, cut into tiles of 32 KB of keys and values (64 tokens
//    in bf16, 128 in e4m3), times the key heads, form one list over the whole batch, and
//    each CTA takes a run of it with an equal share of the keys (rows end inside tiles: by
//    equal numbers of tiles the 64 rows of 200 to 1024 tokens kept an SM busy 72% of the
//    time).  A row's length is thus split over as many CTAs as its share of the bytes,
//    and short rows share a CTA.  Everything follows from the lengths on the device, so
//    that a captured graph serves growing sequences.
//  * Stages.  One warp walks the run: it looks pages up in the table, and brings the pieces of
//    a tile by TMA into a ring of three stages (192 KB in flight on an SM's two CTAs; with 17
//    and more queries of a key head one CTA fits, 96 KB), with the row's queries and the
//    new token's key and value.
//  * Products.  Four warps split a tile's keys, 16 at a time: S^T = K Q^T and O^T += V^T P^T by
//    warp-level MMAs whose A operand is the cache (16 keys or 16 values' dimensions) and whose
//    N = 8 columns are the queries of a key head, so that few queries waste few columns.  The
//    tensor pipe is nearly idle at this; the tcgen05 form would want 128 rows.  The warps'
//    maxima, sums and outputs are their own until the end of an item (row and head): each
//    leaves them in its own rows of the stage that it read last and goes on, and a sixth
//    warp adds them up, stores the result and releases the stage (with the four warps doing
//    that together, they stood still 1 us per item).
//  * More than 8 queries of a key head: the warps split the columns before the keys, up to 32
//    columns, then further items.  With 32 columns a CTA takes 121856 of an SM's 233472 bytes of shared
//    memory (108800 with 8, 113152 with 16), so that the grid of two per SM runs as two waves of one.
//    (16 columns in a warp passed the registers' limit on the 8-bit cache: 12 queries of a head 86 us, and
//    69 with 8, before small weights had products of their own; in bf16 100 either way, 32 queries 71
//    and 75, 64 queries 80 and 74.)
//  * Join.  A CTA's first and last items may continue in other CTAs: each then writes its
//    part to the workspace, and when all its work is done counts itself present for both
//    (one fence and one round trip for the two).  The last CTA of an item, found by a counter
//    that wraps to zero, adds the parts up in the order of the CTAs, so that the result has
//    the same bits every time.
//
// Measured: 64 rows of 200 to 1024 tokens and 96 heads in pages of 64 tokens 290 us (6.6 TB/s, 97%
// of the copy bandwidth), in 8 bits 156 (6.2 TB/s, 91%); 37 rows of 1 to 8192 tokens, 12 queries to
// each of 8 key heads 99 us (88%).  Calls of less than 50 us are bound by the way to the first
// tile (lengths, table, keys: four loads in a row, 3.5 us), by CTAs that end apart, and by the join
// (2 to 4 us): three contexts of up to 131072 tokens in 8 bits 43.5 us (30 at the copy bandwidth), one
// row of 333 tokens 9.6 (2.4).  Far from it, in us of 64 rows of 200 to 1024 tokens: 8 key heads of 12 queries
// each in 8 bits 39 (12), of 32 queries each 88 (25) and in 8 bits 98 (13).
//
// Weights.  They are rounded to bf16 next to bf16 values, since an MMA's operands are of one type, and
// the sum that divides the output is of the rounded ones: each is off by 2^-9 at most, as the output's
// own rounding is, and the outputs are off by 0.0021 of their norm where weights in fp32 leave 0.0017 (64
// pairs, against 64 bits).
//
// 8-bit cache.  Keys' and values' codes are converted to fp16, exactly, and multiplied with
// the queries in fp16 (scaled by a power of two, which keeps the bits of all that are 2^-24 of their
// row's largest or more; smaller ones are off by 2^-32 of that at most) and the weights in fp16.
// (Warp-level MMAs on e4m3 are no way around that: on this machine each takes 2 fp16 MMAs and the
// conversion of both operands.)  A key's exponent goes to its score, a value's exponent
// to its weight, and the weights that multiply the codes are relative to the largest of these
// products, whose running maximum a column keeps next to its scores'; small ones have MMAs of
// their own.
#include <cuda.h>
#include <cuda_runtime.h>
#include <cstdint>

#include "kv.h"
#include "kv_row.cuh"
#include "ptx.cuh"

namespace w4a16 {

namespace {

constexpr int kWarps = 4;                    // consumers
constexpr int kThreads = (kWarps + 2) * 32;  // the producer before them, the finisher after
constexpr int kStages = 3;
constexpr int kStageBytes = 32768;           // a tile's keys and values
constexpr int kWarpBytes = kStageBytes / kWarps;
constexpr int kValueOffset = 2048;           // from 16 keys' rows of 128 bytes to their values'
constexpr int kMaxCols = 32;                 // query columns of an item: eight a warp
constexpr int kQueryStride = 272;            // bytes between rows of q, on other banks
constexpr int kCtasPerSm = 2;
constexpr int kInvalid = 1;                  // W4A16_ERR_INVALID_ARG
// A column's maximum is raised, and what it has so far scaled down, only where a score passes
// it by this much (powers of two): rarely, and until then a warp's lanes need not agree on the
// largest score.
constexpr float kSlackBf16 = 8.0f, kSlackE4m3 = 3.0f;
// e4m3: fp16 weights go up to 2^(12.9 + 3).  Those below 2^-16, where fp16 has fewer bits than bf16, get
// products of their own, 2^24 times as large: where the keys with the large weights have values
// of 0 in a dimension, the small weights are all there is.  (One query: in the odd columns, at
// no cost.  Several: with weights over more than 2^29 in every step 64 rows of 8 key heads take 29
// us and not 26.)  What is less than 2^-61 of the largest vanishes.
constexpr float kWeightTop = 12.9f;
constexpr float kSmallScale = 16777216.0f;
__device__ __forceinline__ bool small_weight(float p) {  // 0 < p < 2^-16
    return __float_as_uint(p) - 1u < 0x377FFFFFu;
}
// The maximum of no scores.  (Not -inf, whose differences would be NaN.)
constexpr float kLeast = -3.0e38f;

// How the queries of a key head (the group) are laid over columns and warps.
struct Columns {
    int group;  // queries of a key head
    int block;  // columns of an item: 8, 16 or 32
    int blocks; // items of a key head
    int warps;  // warps side by side in the columns: 1, 2 or 4
};
inline Columns columns_of(int group) {
    Columns c;
    c.group = group;
    c.block = group <= 8 ? 8 : group <= 16 ? 16 : kMaxCols;
    c.blocks = (group + c.block - 1) / c.block;
    c.warps = c.block / 8;
    return c;
}
__host__ __device__ inline int used_columns(int group) { return group < kMaxCols ? group : kMaxCols; }

// A part in the workspace: the outputs of its columns, then for each its sum, its maximum and
// the maximum that the outputs are relative to (e4m3; else the same).
__host__ __device__ inline int part_floats(int cols) { return cols * (kKvHeadDim + 4); }

// The workspace's counters, one for each CTA.
__host__ __device__ inline int counter_bytes(int ctas) { return (ctas * 4 + 15) / 16 * 16; }

// (Positions go up to 2^31 - 16, and a tile may end at 2^31: comparisons take from the length, not add to
// a tile's first key.)
// What the producer says about a stage.
struct alignas(16) Unit {
    int row, head, block, key0;       // the tile's first key
    int low, len, flags;              // keys that the row sees
    int parts, first_cta;             // of the item, with kLast
    int page, at;                     // the new token's place, with kNew
};
constexpr int kFirst = 1;    // the item's first unit in this CTA
constexpr int kLast = 2;     // and its last
constexpr int kEnd = 16;     // the CTA's last unit
constexpr int kNew = 4;      // the tile has the new token
constexpr int kBad = 8;      // a page index out of range
constexpr int kQSlotShift = 5;

// A row's slot and the keys it sees; no keys for padding, an empty sequence or bad data.
struct Row {
    int slot, len, low;
    int first, tiles;  // its first tile, and how many
    int skip;          // groups of 16 keys of the first tile that it does not see
    int weight;        // of an item: the groups that it sees, and item_weight
};

// A part that the CTA has written: the item, and whether the CTA is to add it up.
struct Pending {
    int row, head, block, first_cta, parts;  // parts 0: none
    int join;
};

struct Shared {
    uint64_t full[kStages], empty[kStages], done[kStages], met, joined;
    Unit unit[kStages];
    alignas(16) uint16_t fresh[kStages][2][kKvHeadDim];           // the new token's key and value
    alignas(16) uint8_t exponents[kStages][2 * 128];  // e4m3: a tile's (key, value) pairs
    // an item's sums and maxima by stage, column and key warp (at most 64 of the two)
    alignas(16) float part_l[kStages][kMaxCols], part_m[kStages][kMaxCols], part_w[kStages][kMaxCols];
    Pending pending[2];  // the CTA's parts of items that others share
    int64_t warp_sum[kThreads / 32];
    int64_t bound[2];
    int64_t start_base;
    int start_row, start_item, start_into;
    Row start;
    int empty_rows;
    int twice;  // a slot is twice in the list
    int abort;
};

struct DecodeArgs {
    KvView kv;
    DecodeParams p;
    Columns cols;
    int item_weight;  // groups of 16 keys that an item costs as much as, beside its own
    int snap;         // groups from an item's end within which no part begins
    uint64_t grid_reciprocal;  // 2^64 / CTAs, rounded up
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
// Sixteen rows of 32 bytes' columns, transposed: register r of lane (g, c) has column
// g + 8 (r % 2) of rows 4c .. 4c + 3, + 16 from r = 2 on; a lane gives a row's address.
__device__ __forceinline__ void ldsm_bytes_trans(uint32_t addr, uint32_t (&v)[4]) {
    asm volatile("ldmatrix.sync.aligned.m16n16.x2.trans.shared.b8 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3])
                 : "r"(addr)
                 : "memory");
}
// The A operand from rows g and g + 8, four codes each: columns 2c, 2c + 1 and 2c + 8, 2c + 9.
__device__ __forceinline__ void codes_to_halves(uint32_t row, uint32_t row8, uint32_t (&f)[4]) {
    f[0] = e4m3_to_half2(static_cast<uint16_t>(row));
    f[1] = e4m3_to_half2(static_cast<uint16_t>(row8));
    f[2] = e4m3_to_half2(static_cast<uint16_t>(row >> 16));
    f[3] = e4m3_to_half2(static_cast<uint16_t>(row8 >> 16));
}
template <bool E4M3>
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (E4M3)
        asm(
            "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
            "{%8, %9}, {%0, %1, %2, %3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm(
            "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
            "{%8, %9}, {%0, %1, %2, %3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// The consumers' barrier, bounded like every wait; false if the CTA gave up.
__device__ __forceinline__ bool consumers_meet(Shared& sh, uint32_t& phase, int* status, uint64_t wait_ns) {
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(smem_u32(&sh.met));
    // (the others are a few instructions away: polls that do not suspend the warp)
    bool ok = false;
    for (int i = 0; i < 64 && !ok; ++i) ok = __all_sync(0xffffffffu, mbar_test_wait(smem_u32(&sh.met), phase));
    if (!ok) ok = wait_warp(smem_u32(&sh.met), phase, &sh.abort, status, wait_ns);
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

// A stage holds groups of 16 tokens; in each, for each half of the rows in bf16, the keys' 128
// bytes, then the values'.  A box is a number of groups of one page.  Byte of 16-byte unit
// `unit` of a tile's key row, in the 128-byte swizzle.
template <bool E4M3>
__device__ __forceinline__ uint32_t tile_byte(int row, int unit) {
    const uint32_t box = E4M3 ? (row >> 4) * 4096u : (row >> 4) * 8192u + (unit >> 3) * 4096u;
    return box + (row & 15) * 128u + (((unit & 7) ^ (row & 7)) << 4);
}
// Key of row `row` of a step's matrix `i` of 8 keys; e4m3: turned, so that both ways in which
// ldmatrix reads keys and values are without bank conflicts.
template <bool E4M3>
__device__ __forceinline__ int key_at(int row, int i) {
    return 8 * i + (E4M3 ? row ^ 4 * (i & 1) : row);
}
// One box; completion is signalled on `bar` as transaction bytes.
__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap* map, uint32_t bar, int32_t group) {
    asm volatile(
        "cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%2, %2, %2, %2, %3}], [%4];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(group), "r"(bar)
        : "memory");
}
// Quotient of numbers that are not negative: in 32 bits where they fit (a 64-bit division takes
// 300 clocks, and a short row's call had eight of them in a row).
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
    if (((a | b) >> 32) == 0) return static_cast<uint32_t>(a) / static_cast<uint32_t>(b);
    return a / b;
}

__device__ __forceinline__ bool length_ok(const DecodeArgs& a, int len) {
    return len >= 0 && len <= static_cast<int64_t>(a.kv.max_pages) << a.kv.page_shift;
}
template <bool E4M3>
__device__ __forceinline__ Row row_from(const DecodeArgs& a, int slot, int len) {
    constexpr int kGroups = E4M3 ? 8 : 4;  // of a tile
    Row r{slot, len, 0, 0, 0, 0, 0};
    if (len == 0) return r;
    r.low = len > a.p.window ? len - a.p.window : 0;
    const int begin = r.low / 16, end = (len - 1) / 16 + 1;
    r.first = begin / kGroups;
    r.tiles = (end - 1) / kGroups + 1 - r.first;
    r.skip = begin - r.first * kGroups;
    r.weight = end - begin + a.item_weight;
    return r;
}
template <bool E4M3>
__device__ __forceinline__ Row row_of(const DecodeArgs& a, bool any, int i, bool* bad) {
    const int slot = a.p.slots[i];
    *bad = slot < -1 || slot >= a.kv.num_slots;
    if (*bad || slot < 0) return Row{};
    const int len = a.kv.seq_len[slot];
    const bool refused = growth_refused(a.kv, any, slot);
    *bad = refused || !length_ok(a, len);
    return *bad ? Row{} : row_from<E4M3>(a, slot, len);
}
// Where tile t of an item starts in its weight.
template <bool E4M3>
__device__ __forceinline__ int tile_start(const Row& r, int t) {
    return t == 0 ? 0 : t * (E4M3 ? 8 : 4) - r.skip;
}

// CTA c has the tiles that start in [bound(c), bound(c + 1)), bound(c) = c * weight / ctas rounded
// down and, if that is at most `snap` groups from the start or the end of the item in which it
// falls, moved there: a part costs more than so many groups.  `snap` is at least a tile and
// an item's weight, and so are the bounds apart before they move; so each part of an item has a tile.
// A bound `into` groups into an item, moved.
__device__ __forceinline__ int snapped(int into, int weight, int snap) {
    return into <= snap ? 0 : weight - into <= snap ? weight : into;
}
// The parts of an item [begin, end), and the CTA of the first if there are more.
__device__ __forceinline__ int parts_of(int64_t begin, int64_t end, int64_t weight, int64_t ctas, int snap,
                                        int* first_cta) {
    // the bounds in (begin + snap, end - snap)
    if (end - begin <= 2 * snap) {
        *first_cta = 0;
        return 1;
    }
    const int64_t lo = quotient((begin + snap + 1) * ctas + weight - 1, weight);
    const int64_t hi = quotient((end - snap) * ctas - 1, weight);
    *first_cta = static_cast<int>(lo) - 1;
    return hi >= lo ? static_cast<int>(hi - lo) + 2 : 1;
}

template <bool E4M3>
__device__ void produce(const DecodeArgs& a, const CacheMaps& maps, Shared& sh, uint32_t stages,
                        uint32_t queries, int64_t weight, int64_t ctas, int64_t w1) {
    constexpr int kTile = E4M3 ? 128 : 64;
    const KvView& kv = a.kv;
    const int lane = threadIdx.x & 31;
    constexpr int kGroupBytes = kStageBytes / (kTile / 16);  // 16 tokens' keys and values
    const int items = kv.kv_heads * a.cols.blocks;        // of a row
    const int64_t width = static_cast<int64_t>(a.p.H + 2 * kv.kv_heads) * kKvHeadDim;
    // This lane's tokens of a tile: a group of 16, or in e4m3 eight, whose exponents it copies
    // (of a group the even lane loads the codes).
    constexpr int kLaneTokens = E4M3 ? 8 : 16;
    const bool has_tokens = lane < kTile / kLaneTokens, has_group = has_tokens && lane * kLaneTokens % 16 == 0;
    const int lane_key = has_tokens ? lane * kLaneTokens : 0;
    const int group = lane * kLaneTokens / 16, of_box = group & (maps.groups - 1);
    const uint8_t* const exponents = E4M3 ? kv.exponents + kv_exponent(kv, a.p.layer, 0, 0, 0, 0) : nullptr;

    int row = sh.start_row;
    int64_t base = sh.start_base;
    Row r = sh.start;
    int item = sh.start_item, tile = 0;
    const int rest = sh.start_into;
    while (tile < r.tiles && tile_start<E4M3>(r, tile) < rest) tile = max(tile + 1, (rest + r.skip) / (kTile / 16));
    bool begun = false, more = true;
    // Page list entries, a lane each: the row's first 32, the 32 that the tiles are in, and the
    // 32 after them; and the same of the rows that follow.  All are loaded ahead of their use:
    // a stop for each would be a microsecond, of the 1.5 that a tile takes.
    auto load_ids = [&](const Row& of, int from) {
        const int e = from + lane;
        return e <= (of.len - 1) >> kv.page_shift
                   ? __ldcg(kv.table + static_cast<int64_t>(of.slot) * kv.max_pages + e) : 0;
    };
    auto first_entry = [&](const Row& of) { return of.first * kTile >> kv.page_shift; };
    constexpr int kUnknown = -2, kNone = -1;
    int next_index = kUnknown, next_ids = 0, rows_from = kNone, slot_of = -1, len_of = 0;
    Row next{};
    const bool any = any_refused(kv);
    auto find_next = [&]() {  // the next row with keys
        next_index = kNone;
        for (int from = row + 1; from < a.p.n && next_index == kNone; from = rows_from + 32) {
            if (rows_from == kNone || from >= rows_from + 32) {
                rows_from = from;
                slot_of = from + lane < a.p.n ? __ldcg(a.p.slots + from + lane) : -1;
                const bool slot_ok = slot_of >= 0 && slot_of < kv.num_slots;
                len_of = slot_ok ? __ldcg(kv.seq_len + slot_of) : 0;
                const bool refused = slot_ok && growth_refused(kv, any, slot_of);
                if (refused || !length_ok(a, len_of)) len_of = 0;
            }
            const uint32_t have = __ballot_sync(0xffffffffu, len_of > 0 && rows_from + lane >= from);
            if (have == 0) continue;
            const int l = __ffs(have) - 1;
            next_index = rows_from + l;
            next = row_from<E4M3>(a, __shfl_sync(0xffffffffu, slot_of, l), __shfl_sync(0xffffffffu, len_of, l));
            next_ids = load_ids(next, first_entry(next));
        }
    };
    int slot = 0;             // of the item's queries
    int since[2] = {0, 0};    // units since the one that read each query slot; 0: none
    int st = 0;
    uint32_t phase = 0;       // of the stage's barriers
    int64_t issued = 0;
    bool cut = rest > 0;      // the item began in another CTA
    if (item == items) {  // (a bound moved to the end of the row)
        find_next();
        item = tile = 0;
        base += static_cast<int64_t>(items) * r.weight;
        row = next_index;
        r = next;
        more = next_index != kNone;
        next_index = kUnknown;
    }
    if (!more || tile >= r.tiles) {  // (only if the lengths changed during the call)
        sh.abort = 1;
        record_status(kv.status, kInvalid);
        return;
    }
    int head = item / a.cols.blocks, block = item - head * a.cols.blocks;
    int64_t begin = base + static_cast<int64_t>(item) * r.weight;  // of the item
    int ids_from = ((r.first + tile) * kTile) >> kv.page_shift;
    int ids = load_ids(r, ids_from), ids_first = load_ids(r, first_entry(r)), ids_after = load_ids(r, ids_from + 32);
    for (; more; ++issued) {
        const bool first = !begun || tile == 0;
        begun = true;
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
        // (32 entries are whole tiles, and a page's boxes never cross it)
        if (key0 >> kv.page_shift >= ids_from + 32) {
            ids = ids_after;
            ids_from += 32;
            ids_after = load_ids(r, ids_from + 32);
        }
        const uint32_t bar = smem_u32(&sh.full[st]);
        // The groups that the row sees, by boxes as large as a page allows, or each by itself at
        // the row's ends.
        const int key = key0 + lane_key;  // of this lane's tokens
        const int id = __shfl_sync(0xffffffffu, ids, ((key >> kv.page_shift) - ids_from) & 31);
        const bool id_ok = id >= 0 && id < kv.num_pages;
        const int32_t row_at = (((id_ok ? id : 0) * kv.kv_heads + head) << kv.page_shift) +
                               (key & ((1 << kv.page_shift) - 1));
        const bool mine = has_group && key < r.len && key + 16 > r.low;
        const bool whole = mine && key - (of_box - 1) * 16 > r.low && key + (maps.groups - 1 - of_box) * 16 < r.len;
        if (mine && (!whole || of_box == 0)) {
            const uint32_t dst = stages + st * kStageBytes + group * kGroupBytes;
            const int box_bytes = whole ? maps.groups * kGroupBytes : kGroupBytes;
            if (dbg_check(tma_box_ok(dst, box_bytes, 1024, stages, stages + kStages * kStageBytes, 0, 1), kv.status))
                load_box(dst, whole ? &maps.box : &maps.group, bar, row_at >> 4);
        }
        if constexpr (E4M3) {  // (key, value) exponents; every lane arrives
            if (has_tokens && key < r.len && key + 8 > r.low)
                asm volatile("cp.async.ca.shared.global [%0], [%1], 16;" ::"r"(
                                 smem_u32(&sh.exponents[st][lane * 16])),
                             "l"(exponents + 2 * static_cast<int64_t>(row_at))
                             : "memory");
            asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
        }
        const int loads = __popc(__ballot_sync(0xffffffffu, mine));
        const bool tile_bad = __any_sync(0xffffffffu, mine && !id_ok);
        uint32_t bytes = loads * kGroupBytes;
        const uint16_t* const qkv = a.p.qkv + row * width;
        if (first) {
            const int q_cols = min(a.cols.block, a.cols.group - block * a.cols.block);
            for (int i = lane; i < q_cols; i += 32)
                bulk_load(queries + (slot * a.cols.block + i) * kQueryStride,
                          qkv + (static_cast<int64_t>(head) * a.cols.group + block * a.cols.block + i) * kKvHeadDim,
                          256, bar);
            bytes += q_cols * 256;
        }
        const bool fresh = key0 >= r.len - kTile;
        int page = -1;
        if (fresh) {
            if (lane < 2)
                bulk_load(smem_u32(sh.fresh[st][lane]),
                          qkv + (a.p.H + lane * kv.kv_heads + head) * static_cast<int64_t>(kKvHeadDim), 256, bar);
            bytes += 512;
            page = __shfl_sync(0xffffffffu, ids, (((r.len - 1) >> kv.page_shift) - ids_from) & 31);
            if (page >= kv.num_pages) page = -1;
        }
        // whether the item goes on in this CTA, and the CTA after it
        const bool ends = begin + r.weight <= w1;
        const bool last = tile + 1 == r.tiles || (!ends && begin + tile_start<E4M3>(r, tile + 1) >= w1);
        more = !last || begin + r.weight < w1;
        if (lane == 0) {
            Unit& t = sh.unit[st];
            t.row = row;
            t.head = head;
            t.block = block;
            t.key0 = key0;
            t.low = r.low;
            t.len = r.len;
            t.flags = (first ? kFirst : 0) | (last ? kLast : 0) | (fresh ? kNew : 0) | (tile_bad ? kBad : 0) |
                      (more ? 0 : kEnd) | slot << kQSlotShift;
            t.parts = 1;
            t.first_cta = 0;
            if (last && (cut || !ends)) t.parts = parts_of(begin, begin + r.weight, weight, ctas, a.snap, &t.first_cta);
            t.page = page;
            t.at = (r.len - 1) & ((1 << kv.page_shift) - 1);
            // (after the copies: the phase waits for this arrival)
            mbar_arrive_expect_tx(bar, bytes);
        }
        __syncwarp();
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
            cut = false;
            begin += r.weight;
            if (++block == a.cols.blocks) {
                block = 0;
                ++head;
            }
            if (++item == items && more) {
                if (next_index == kUnknown) find_next();
                if (next_index == kNone) {  // (only if the lengths changed during the call)
                    sh.abort = 1;
                    record_status(kv.status, kInvalid);
                    ++issued;
                    break;
                }
                item = head = 0;
                row = next_index;
                r = next;
                next_index = kUnknown;
                ids_first = next_ids;
                ids_from = kNone;
            }
            if (ids_from != first_entry(r)) {
                ids = ids_first;
                ids_from = first_entry(r);
                ids_after = load_ids(r, ids_from + 32);
            }
        }
        // (once the stages are all under way)
        if (next_index == kUnknown && issued + 1 >= kStages) find_next();
    }
    // the copies in flight, before the CTA may end (the consumers may have given up)
    for (int64_t i = issued > kStages ? issued - kStages : 0; i < issued; ++i)
        settle(smem_u32(&sh.full[i % kStages]), (i / kStages) & 1);
}

// What makes an output of a sum relative to 2^w, with weights whose sum is l relative to 2^m.
// In two factors, to be multiplied with the sum one after the other: a value's exponent may be -120, and
// with a sum of weights in the thousands their product would be a subnormal of a few bits.
template <bool E4M3>
__device__ __forceinline__ float2 output_scale(float l, float m, float w) {
    return E4M3 ? make_float2(1.0f / l * ex2(-kWeightTop), ex2(w - m)) : make_float2(1.0f / l, 1.0f);
}
template <bool E4M3>
__device__ __forceinline__ float scaled(float sum, float2 scale) {
    return E4M3 ? sum * scale.x * scale.y : sum * scale.x;
}

// A column of a warp's output lies in the warp's own rows of the stage, which no other warp
// reads while the columns are not split; its dimensions are turned so that the lanes of
// a store hit different banks.
__device__ __forceinline__ uint32_t meet_byte(int warp, int col) { return warp * kWarpBytes + col * 512; }
__device__ __forceinline__ int meet_turn(int col) { return 8 * (col >> 1 & 3); }

__device__ __forceinline__ uint16_t* output_of(const DecodeArgs& a, int row, int head, int block) {
    return a.p.out + (static_cast<int64_t>(row) * a.p.H + static_cast<int64_t>(head) * a.cols.group +
                      block * a.cols.block) * kKvHeadDim;
}
__device__ __forceinline__ int columns_in(const DecodeArgs& a, int block) {
    return min(a.cols.block, a.cols.group - block * a.cols.block);
}
__device__ __forceinline__ float* parts_in(const DecodeArgs& a) {
    return reinterpret_cast<float*>(static_cast<uint8_t*>(a.p.workspace) + counter_bytes(gridDim.x));
}

// The items that this CTA adds up, after its last unit, by all warps that computed.  Part 0 of
// an item is its CTA's last item, the others their CTAs' first, and they are added in this
// order.  Sixteen lanes take a column, eight outputs each; a lane has a part's statistics, and the
// outputs of kBatch parts are under way together.  One compact copy of the code: every CTA runs
// it once at most, and fetching it is a good part of its time (13 parts of 8 columns: a thread per output
// that walked columns and parts 35 us, a warp per column 20, this inlined and with 16 parts 6).
template <bool E4M3>
__device__ __noinline__ void join_pending(const float* parts, uint16_t* out, int H, int group, int block,
                                          const Pending* pending, int* status, int mine, int groups) {
    constexpr int kBatch = 8;
    const int lane = threadIdx.x & 31, l16 = lane & 15, max_cols = used_columns(group);
    const int64_t stride = part_floats(max_cols);
    int cols[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) cols[i] = pending[i].join ? min(block, group - pending[i].block * block) : 0;
#pragma unroll 1
    for (int i0 = 0; i0 < cols[0] + cols[1]; i0 += groups) {
        // (a warp's halves may have columns of two items, or one of them none)
        const int i = i0 + mine;
        const Pending& p = pending[i >= cols[0]];
        const int col = i < cols[0] ? i : i - cols[0], n = i < cols[0] + cols[1] ? p.parts : 0;
        const int longest = max(n, __shfl_xor_sync(0xffffffffu, n, 16));
        const float* const first = parts + (2 * p.first_cta + 1) * stride;  // then every second, from one before
        auto part = [&](int k) { return k == 0 ? first : first + (2 * k - 1) * stride; };
        auto stats = [&](int k) {
            return k < n ? __ldcg(reinterpret_cast<const float4*>(part(k) + max_cols * kKvHeadDim) + col)
                         : make_float4(0.0f, kLeast, kLeast, 0.0f);
        };
        float m = kLeast, top = kLeast, l = 0.0f;
        float4 s = stats(l16);
        bool bad = false;
        float sum[8] = {}, f = 0.0f;
#pragma unroll 1
        for (int k0 = 0; k0 < longest; k0 += kBatch) {
            float4 v[kBatch][2];
#pragma unroll
            for (int b = 0; b < kBatch; ++b)
                if (k0 + b < n) {
                    const float4* from = reinterpret_cast<const float4*>(part(k0 + b) + col * kKvHeadDim) + 2 * l16;
                    v[b][0] = __ldcg(from);
                    v[b][1] = __ldcg(from + 1);
                }
            if (k0 == 0) {  // (with the first outputs on their way)
                m = s.y;
                top = s.z;
#pragma unroll 1
                for (int k = 16; k < longest; k += 16) {
                    const float4 t = stats(k + l16);
                    m = fmaxf(m, t.y);
                    top = fmaxf(top, t.z);
                }
#pragma unroll
                for (int o = 8; o > 0; o >>= 1) {
                    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                }
            }
            if (k0 % 16 == 0) {
                if (k0 > 0) s = stats(k0 + l16);
                bad |= s.x < 0.0f;
                l += s.x * ex2(s.y - m);
                f = ex2(s.z - top);
            }
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
                const float w = __shfl_sync(0xffffffffu, f, (lane & 16) | ((k0 + b) & 15));
                if (k0 + b < n) {
                    sum[0] += w * v[b][0].x;
                    sum[1] += w * v[b][0].y;
                    sum[2] += w * v[b][0].z;
                    sum[3] += w * v[b][0].w;
                    sum[4] += w * v[b][1].x;
                    sum[5] += w * v[b][1].y;
                    sum[6] += w * v[b][1].z;
                    sum[7] += w * v[b][1].w;
                }
            }
        }
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
        bad = (__ballot_sync(0xffffffffu, bad) >> (lane & 16) & 0xFFFFu) != 0;
        if (n == 0) continue;
        const float2 scale = output_scale<E4M3>(l, m, top);
#pragma unroll
        for (int k = 0; k < 8; ++k) sum[k] = scaled<E4M3>(sum[k], scale);
        uint4 o = make_uint4(bf16_pair(sum[0], sum[1]), bf16_pair(sum[2], sum[3]), bf16_pair(sum[4], sum[5]),
                             bf16_pair(sum[6], sum[7]));
        if (bad) {
            o = make_uint4(0, 0, 0, 0);
            if (l16 == 0) record_status(status, kInvalid);
        }
        reinterpret_cast<uint4*>(
            out + (static_cast<int64_t>(p.row) * H + static_cast<int64_t>(p.head) * group + p.block * block + col) *
                      kKvHeadDim)[l16] = o;
    }
}

// The finisher: follows the stages, and at an item's end adds up what the warps left there.
template <bool E4M3>
__device__ void finish(const DecodeArgs& a, Shared& sh, const uint8_t* stage_mem) {
    const KvView& kv = a.kv;
    const int lane = threadIdx.x & 31;
    const int key_warps = kWarps / a.cols.warps, max_cols = used_columns(a.cols.group);
    int st = 0;
    uint32_t phase = 0, done_phase = 0;  // done_phase: a bit for each stage
    bool bad = false;
    for (;;) {
        if (!wait_warp(smem_u32(&sh.full[st]), phase, &sh.abort, kv.status, a.p.wait_ns)) return;
        const Unit& t = sh.unit[st];
        const int flags = t.flags;
        if (flags & kFirst) bad = false;
        bad |= (flags & kBad) != 0;
        if (flags & kLast) {
            if (!wait_warp(smem_u32(&sh.done[st]), done_phase >> st & 1, &sh.abort, kv.status, a.p.wait_ns)) return;
            done_phase ^= 1u << st;
            const uint8_t* const tile = stage_mem + st * kStageBytes;
            const int cols = columns_in(a, t.block);
            const bool whole = t.parts == 1;
            const int slot = t.first_cta == static_cast<int>(blockIdx.x);
            float* const part = parts_in(a) + (2 * static_cast<int64_t>(blockIdx.x) + slot) * part_floats(max_cols);
            uint16_t* const out = output_of(a, t.row, t.head, t.block);
#pragma unroll 2
            for (int col = 0; col < cols; ++col) {
                const int cw = col / 8, in = col % 8, turned = (4 * lane + meet_turn(in)) & 127;
                float4 x[kWarps];
                float ls[kWarps], ms[kWarps], ws[kWarps];
#pragma unroll
                for (int k = 0; k < kWarps; ++k) {
                    const bool has = k < key_warps;
                    const int at = col * key_warps + (has ? k : 0);
                    x[k] = *reinterpret_cast<const float4*>(
                        tile + meet_byte((has ? k : 0) * a.cols.warps + cw, in) + turned * 4);
                    ls[k] = has ? sh.part_l[st][at] : 0.0f;
                    ms[k] = has ? sh.part_m[st][at] : kLeast;
                    ws[k] = E4M3 && has ? sh.part_w[st][at] : ms[k];
                }
                // (a warp without keys: a maximum of kLeast and a sum of 0)
                const float m = fmaxf(fmaxf(ms[0], ms[1]), fmaxf(ms[2], ms[3]));
                const float w = E4M3 ? fmaxf(fmaxf(ws[0], ws[1]), fmaxf(ws[2], ws[3])) : m;
                float l = 0.0f;
                float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
                for (int k = 0; k < kWarps; ++k) {
                    const float f = ex2(ms[k] - m);
                    l += f * ls[k];
                    const float h = k >= key_warps ? 0.0f : E4M3 ? ex2(ws[k] - w) : f;
                    if (k < key_warps) {
                        o.x += h * x[k].x;
                        o.y += h * x[k].y;
                        o.z += h * x[k].z;
                        o.w += h * x[k].w;
                    }
                }
                if (whole) {
                    const float2 f = output_scale<E4M3>(l, m, w);
                    reinterpret_cast<uint2*>(out + col * kKvHeadDim)[lane] =
                        bad ? make_uint2(0, 0)
                            : make_uint2(bf16_pair(scaled<E4M3>(o.x, f), scaled<E4M3>(o.y, f)),
                                         bf16_pair(scaled<E4M3>(o.z, f), scaled<E4M3>(o.w, f)));
                } else {
                    reinterpret_cast<float4*>(part + col * kKvHeadDim)[lane] = o;
                    if (lane == 0)  // (a sum is never negative: marks a bad page index)
                        reinterpret_cast<float4*>(part + max_cols * kKvHeadDim)[col] =
                            make_float4(bad ? -1.0f : l, m, w, 0.0f);
                }
            }
            if (lane == 0) {
                if (whole) {
                    if (bad) record_status(kv.status, kInvalid);
                } else {
                    sh.pending[slot] = {t.row, t.head, t.block, t.first_cta, t.parts, 0};
                }
            }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&sh.empty[st]));
        if (flags & kEnd) break;
        if (++st == kStages) {
            st = 0;
            phase ^= 1;
        }
    }
    if (sh.pending[0].parts == 0 && sh.pending[1].parts == 0) {
        if (lane == 0) mbar_arrive(smem_u32(&sh.joined));
        return;
    }
    __syncwarp();
    if (lane < 2 && sh.pending[lane].parts > 0) {
        // (releases this CTA's part, which the warp wrote, and acquires the others')
        const uint32_t last = sh.pending[lane].parts - 1;
        uint32_t* const count = static_cast<uint32_t*>(a.p.workspace) + sh.pending[lane].first_cta;
        uint32_t was;
        asm volatile("atom.acq_rel.gpu.global.inc.u32 %0, [%1], %2;" : "=r"(was) : "l"(count), "r"(last) : "memory");
        sh.pending[lane].join = was == last;
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&sh.joined));
    if (sh.pending[0].join || sh.pending[1].join)
        join_pending<E4M3>(parts_in(a), a.p.out, a.p.H, a.cols.group, a.cols.block, sh.pending, kv.status,
                           2 * kWarps + (lane >> 4), 2 * (kWarps + 1));
}

// The tile's ends: the new token's row is put in place, as the cache holds it, and stored, and
// values that no query sees become zero (a weight of 0 does not keep a NaN out of a product).
template <bool E4M3>
__device__ __forceinline__ void mend_tile(const DecodeArgs& a, Shared& sh, int st, uint8_t* tile, int warp, int lane,
                                       bool store_ok) {
    constexpr int kTile = E4M3 ? 128 : 64;
    const KvView& kv = a.kv;
    const Unit& t = sh.unit[st];
    constexpr int kStep = kTile / kWarps;  // the keys that this warp mends
    const int key = t.key0 + warp * kStep;
    if (key < t.len && key > t.low - kStep) {
        for (int i = lane; i < kStep * (E4M3 ? 8 : 16); i += 32) {
            const int r = i >> (E4M3 ? 3 : 4), unit = i & (E4M3 ? 7 : 15);
            if (key + r < t.low || key + r >= t.len)
                *reinterpret_cast<uint4*>(tile + kValueOffset + tile_byte<E4M3>(warp * kStep + r, unit)) =
                    make_uint4(0, 0, 0, 0);
        }
        const int fresh = t.len - 1 - key;
        if (fresh < kStep && fresh >= 0) {
            // half a warp has the key, the other half the value, eight dimensions a lane
            const int r = warp * kStep + fresh, which = lane >> 4, unit = lane & 15;
            const bool store = store_ok && t.block == 0 && t.page >= 0;
            const int64_t row = kv_row(kv, a.p.layer, which, max(t.page, 0), t.head, t.at);
            const uint4 v = reinterpret_cast<const uint4*>(sh.fresh[st][which])[unit];
            if constexpr (!E4M3) {
                *reinterpret_cast<uint4*>(tile + which * kValueOffset + tile_byte<E4M3>(r, unit)) = v;
                if (store) reinterpret_cast<uint4*>(kv.pages)[row * 16 + unit] = v;
            } else {
                uint2 codes;
                const int e = e4m3_row_of_16(v, &codes);
                *reinterpret_cast<uint2*>(tile + which * kValueOffset + tile_byte<E4M3>(r, unit >> 1) + (unit & 1) * 8) =
                    codes;
                if (unit == 0) sh.exponents[st][r * 2 + which] = static_cast<uint8_t>(e + 127);
                if (store) {
                    reinterpret_cast<uint2*>(kv.pages)[row * 16 + unit] = codes;
                    if (unit == 0)
                        kv.exponents[kv_exponent(kv, a.p.layer, which, t.page, t.head, t.at)] =
                            static_cast<uint8_t>(e + 127);
                }
            }
        }
    }
    fence_proxy_async();  // (the stage's next contents come by TMA)
    __syncwarp();
}

// The running softmax of a warp's eight columns: two a thread.
struct State {
    float m[2], l[2], o[8][4];
    float w[2];  // e4m3: the largest score and value's exponent, which o is relative to
    bool bad;    // a page index was out of range
};

template <bool E4M3, bool ONE>
__device__ void consume(const DecodeArgs& a, Shared& sh, uint8_t* stage_mem, uint8_t* query_mem) {
    constexpr int kTile = E4M3 ? 128 : 64;
    constexpr int kStep = kTile / kWarps, kGroups = kStep / 16, kRows = 2 * kGroups;  // a warp's keys at a time
    const KvView& kv = a.kv;
    const int lane = threadIdx.x & 31, warp = (threadIdx.x >> 5) - 1;
    const int g = lane >> 2, c = lane & 3;
    const int col_warp = warp % a.cols.warps, key_warp = warp / a.cols.warps, key_warps = kWarps / a.cols.warps;
    const float scale = a.p.scale * 1.4426950408889634f;
    // This lane's row of an ldmatrix within a group of 16 keys (bytes, transposed: of the step's 32
    // keys).  Matrices of keys are (rows 0 .. 7, unit 0), (8 .. 15, 0), (0 .. 7, 1), (8 .. 15, 1); of
    // transposed values with the middle two exchanged; of transposed bytes rows 4c .. 4c + 3
    // are keys 2c, 2c + 1 of one matrix of 8 and of the next, in the order that the weights have.
    // Steps along the dimensions flip bits of the address.
    const uint32_t key_off = tile_byte<E4M3>(key_at<E4M3>(lane & 7, lane >> 3 & 1), lane >> 4);
    const uint32_t value_off =
        E4M3 ? tile_byte<E4M3>(key_at<E4M3>((lane >> 1 & 6) + (lane & 1), 2 * (lane >> 4) + (lane >> 1 & 1)), 0)
             : tile_byte<E4M3>((lane & 7) + ((lane >> 4) << 3), lane >> 3 & 1);
    int st = 0;
    uint32_t phase = 0, met = 0;
    auto wait = [&]() { return wait_warp(smem_u32(&sh.full[st]), phase, &sh.abort, kv.status, a.p.wait_ns); };
    auto release = [&]() {
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&sh.empty[st]));
        if (++st == kStages) {
            st = 0;
            phase ^= 1;
        }
    };
    for (;;) {  // an item
        if (!wait()) return;
        State s;
        uint32_t q[8][2];
        float q_scale[2];  // e4m3: of this thread's columns, the softmax's scale and that of q
        // Q as the B operand: column g of a tile of eight, in the order of K's dimensions
        const uint8_t* const row = query_mem + ((sh.unit[st].flags >> kQSlotShift & 1) * a.cols.block +
                                                (ONE ? 0 : col_warp * 8 + g)) * kQueryStride;
        if constexpr (!E4M3) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                q[k][0] = *reinterpret_cast<const uint32_t*>(row + k * 32 + c * 4);
                q[k][1] = *reinterpret_cast<const uint32_t*>(row + k * 32 + 16 + c * 4);
            }
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
            const int e = e4m3_row_exponent(top);
            const float f = power_of_two(-e);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float x[4] = {bf16_lo(v[k].x) * f, bf16_hi(v[k].x) * f, bf16_lo(v[k].y) * f,
                                    bf16_hi(v[k].y) * f};
                q[k][0] = half_pair(x[0], x[1]);
                q[k][1] = half_pair(x[2], x[3]);
            }
            // (column g's scale is needed by the threads of columns 2c and 2c + 1)
#pragma unroll
            for (int j = 0; j < 2; ++j)
                q_scale[j] = scale * power_of_two(__shfl_sync(0xffffffffu, e, (2 * c + j) * 4));
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) s.m[j] = s.w[j] = kLeast, s.l[j] = 0.0f;
#pragma unroll
        for (int k = 0; k < 8; ++k)
#pragma unroll
            for (int j = 0; j < 4; ++j) s.o[k][j] = 0.0f;
        s.bad = false;
        // whether this thread's columns are of queries
        const int queries = columns_in(a, sh.unit[st].block) - col_warp * 8;
        const bool used[2] = {2 * c < queries, 2 * c + 1 < queries};
        int flags;
        uint8_t* tile;
        for (;;) {  // a unit of it
            flags = sh.unit[st].flags;
            const int key0 = sh.unit[st].key0, low = sh.unit[st].low, len = sh.unit[st].len;
            tile = stage_mem + st * kStageBytes;
            const uint32_t keys = smem_u32(tile), values = keys + kValueOffset;
            s.bad |= (flags & kBad) != 0;
            const bool edge = key0 < low || key0 >= len - kTile;
            if (edge) {
                mend_tile<E4M3>(a, sh, st, tile, warp, lane, !s.bad);
                // others read what this warp mended
                if (a.cols.warps > 1 && !consumers_meet(sh, met, kv.status, a.p.wait_ns)) return;
            }
            for (int step = key_warp; step < kWarps; step += key_warps) {
                const int key = key0 + step * kStep;
                if (key >= len || key <= low - kStep) continue;
                // scores of the step's matrices of 8 keys: row g, columns 2c and 2c + 1
                float acc[2][4];  // e4m3: of two groups; bf16: of even and odd dimensions
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[i][j] = 0.0f;
                if constexpr (!E4M3) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        uint32_t f[4];
                        ldsm_x4(((keys + key_off + step * kWarpBytes) ^ ((k & 3) << 5)) + (k >> 2) * 4096, f);
                        mma<E4M3>(acc[k & 1], f, q[k][0], q[k][1]);
                    }
                } else {
#pragma unroll
                    for (int k = 0; k < 8; k += 2)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            uint32_t w[4], f[4];
                            ldsm_x4((keys + key_off + step * kWarpBytes + i * 4096) ^ (k << 4), w);
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                codes_to_halves(w[2 * h], w[2 * h + 1], f);
                                mma<E4M3>(acc[i], f, q[k + h][0], q[k + h][1]);
                            }
                        }
                }
                constexpr float kSlack = E4M3 ? kSlackE4m3 : kSlackBf16;
                uint32_t b[kGroups][2];  // the weights as the B operand
                bool added = false;      // products with values done
                // a column's maximum over its lanes, if that passes what it was; the factor for what
                // is relative to the old one
                auto raise = [&](float v, float& was) {
                    if constexpr (ONE) {
                        v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 1));
                        v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 2));
                    }
                    v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 4));
                    v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 8));
                    v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 16));
                    const float to = v > was + kSlack ? v : was, f = ex2(was - to);
                    was = to;
                    return f;
                };
                if constexpr (ONE) {
                    // One query, the same in every column: lane (g, c) has row g of all matrices, and
                    // takes that of matrix c (bf16: c % 2, in two lanes alike).
                    const int r = c % kRows, in = key_at<E4M3>(g, r), at = key + in;
                    float x = acc[0][0] + (E4M3 ? 0.0f : acc[1][0]);
                    const float x1 = acc[0][2] + (E4M3 ? 0.0f : acc[1][2]);
                    if (r == 1) x = x1;
                    if (E4M3 && r == 2) x = acc[1][0];
                    if (E4M3 && r == 3) x = acc[1][2];
                    float y = 0.0f;
                    if constexpr (E4M3) {
                        const uint32_t e =
                            *reinterpret_cast<const uint16_t*>(sh.exponents[st] + (step * kStep + in) * 2);
                        x *= __uint_as_float((e & 0xFFu) << 23) * q_scale[0];
                        y = static_cast<float>(static_cast<int>(e >> 8) - 127);
                    } else {
                        x *= scale;
                    }
                    if (edge && (at < low || at >= len)) x = -INFINITY;
                    y += x;
                    if (__any_sync(0xffffffffu, x > s.m[0] + kSlack || (E4M3 && y > s.w[0] + kSlack))) {
                        float f = raise(x, s.m[0]);
                        s.l[0] *= f;
                        if constexpr (E4M3) f = raise(y, s.w[0]);
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            s.o[k][0] *= f;
                            s.o[k][2] *= f;
                            if constexpr (E4M3) {
                                s.o[k][1] *= f;
                                s.o[k][3] *= f;
                            }
                        }
                    }
                    float p = ex2(x - s.m[0]);
                    if constexpr (E4M3) {
                        s.l[0] += p;
                        p = ex2(y - s.w[0] + kWeightTop);
                    } else {
                        // (the rounded weights' sum, so that they add up to one)
                        s.l[0] += bf16_lo(bf16_pair(p, 0.0f));
                    }
                    // rows g and g + 1 in the lanes of even g, then rows 2c and 2c + 1 everywhere
                    if constexpr (E4M3) {  // (the small ones to the odd columns)
                        const bool small = small_weight(p);
                        const float next = __shfl_xor_sync(0xffffffffu, p, 4);
                        const bool next_small = small_weight(next);
                        const uint32_t pair = half_pair(small ? 0.0f : p, next_small ? 0.0f : next);
#pragma unroll
                        for (int i = 0; i < kRows; ++i) b[i >> 1][i & 1] = __shfl_sync(0xffffffffu, pair, 8 * c + i);
                        if (__any_sync(0xffffffffu, small)) {
                            const uint32_t low = half_pair(small ? p * kSmallScale : 0.0f,
                                                           next_small ? next * kSmallScale : 0.0f);
#pragma unroll
                            for (int i = 0; i < kRows; ++i) {
                                const uint32_t l = __shfl_sync(0xffffffffu, low, 8 * c + i);
                                if (g & 1) b[i >> 1][i & 1] = l;
                            }
                        } else if (g & 1) {
#pragma unroll
                            for (int i = 0; i < kRows; ++i) b[i >> 1][i & 1] = 0;
                        }
                    } else {
                        const uint32_t pair = bf16_pair(p, __shfl_xor_sync(0xffffffffu, p, 4));
#pragma unroll
                        for (int i = 0; i < kRows; ++i) b[i >> 1][i & 1] = __shfl_sync(0xffffffffu, pair, 8 * c + i);
                    }
                } else {
                    // row g of each matrix, as it comes out of the products: e4m3 with the keys'
                    // exponents, before the columns' factors
                    float x[kRows][2], value_exp[kRows] = {};
#pragma unroll
                    for (int i = 0; i < kRows; ++i) {
                        float key_scale = 1.0f;
                        if constexpr (E4M3) {
                            const uint32_t e =
                                *reinterpret_cast<const uint16_t*>(sh.exponents[st] + (step * kStep + key_at<E4M3>(g, i)) * 2);
                            key_scale = __uint_as_float((e & 0xFFu) << 23);
                            value_exp[i] = static_cast<float>(static_cast<int>(e >> 8) - 127);
                        }
#pragma unroll
                        for (int j = 0; j < 2; ++j)
                            x[i][j] = E4M3 ? acc[i >> 1][(i & 1) * 2 + j] * key_scale
                                           : acc[0][i * 2 + j] + acc[1][i * 2 + j];
                    }
                    if (edge) {
#pragma unroll
                        for (int i = 0; i < kRows; ++i) {
                            const int at = key + key_at<E4M3>(g, i);
                            if (at >= low && at < len) continue;
                            x[i][0] = x[i][1] = -INFINITY;
                        }
                    }
                    auto factor = [&](int j) { return E4M3 ? q_scale[j] : scale; };
                    // this thread's largest score of a column, and with the value's exponent
                    auto largest = [&](int j) {
                        float v = x[0][j];
#pragma unroll
                        for (int i = 1; i < kRows; ++i) v = fmaxf(v, x[i][j]);
                        return v * factor(j);
                    };
                    auto largest_value = [&](int j) {
                        float v = fmaf(x[0][j], factor(j), value_exp[0]);
#pragma unroll
                        for (int i = 1; i < kRows; ++i) v = fmaxf(v, fmaf(x[i][j], factor(j), value_exp[i]));
                        return v;
                    };
                    bool over = false;
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        over |= largest(j) > s.m[j] + kSlack;
                        if constexpr (E4M3) over |= largest_value(j) > s.w[j] + kSlack;
                    }
                    if (__any_sync(0xffffffffu, over)) {
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            float f = raise(largest(j), s.m[j]);
                            s.l[j] *= f;
                            if constexpr (E4M3) f = raise(largest_value(j), s.w[j]);
#pragma unroll
                            for (int k = 0; k < 8; ++k) {
                                s.o[k][j] *= f;
                                s.o[k][j + 2] *= f;
                            }
                        }
                    }
                    bool small = false;
                    // rows 2c, 2c + 1 of column g: the transpose of what this thread holds
                    auto weight = [&](int i, int j) {
                        return E4M3 ? ex2(fmaf(x[i][j], factor(j), value_exp[i]) + (kWeightTop - s.w[j]))
                                    : ex2(fmaf(x[i][j], factor(j), -s.m[j]));
                    };
#pragma unroll
                    for (int i = 0; i < kRows; ++i) {
                        const float p[2] = {weight(i, 0), weight(i, 1)};
                        const uint32_t w = E4M3 ? half_pair(p[0], p[1]) : bf16_pair(p[0], p[1]);
                        if constexpr (E4M3) {
#pragma unroll
                            for (int j = 0; j < 2; ++j) {
                                s.l[j] += ex2(fmaf(x[i][j], factor(j), -s.m[j]));
                                small |= used[j] && small_weight(p[j]);
                            }
                        } else {  // (the rounded weights' sum, so that they add up to one)
                            s.l[0] += bf16_lo(w);
                            s.l[1] += bf16_hi(w);
                        }
                        b[i >> 1][i & 1] = transpose_8x8(w);
                    }
                    if constexpr (E4M3) {
                        if (__any_sync(0xffffffffu, small)) {
                            uint32_t lo[kGroups][2];
#pragma unroll
                            for (int i = 0; i < kRows; ++i) {
                                const float p[2] = {weight(i, 0), weight(i, 1)};
                                const bool is[2] = {small_weight(p[0]), small_weight(p[1])};
                                lo[i >> 1][i & 1] = transpose_8x8(
                                    half_pair(is[0] ? p[0] * kSmallScale : 0.0f, is[1] ? p[1] * kSmallScale : 0.0f));
                                b[i >> 1][i & 1] =
                                    transpose_8x8(half_pair(is[0] ? 0.0f : p[0], is[1] ? 0.0f : p[1]));
                            }
                            added = true;
#pragma unroll
                            for (int k = 0; k < 8; ++k) {
                                uint32_t w[4], f[4];
                                float d[4] = {};
                                ldsm_bytes_trans((values + value_off + step * kWarpBytes) ^ (k << 4), w);
#pragma unroll
                                for (int i = 0; i < kGroups; ++i) {
                                    codes_to_halves(w[2 * i], w[2 * i + 1], f);
                                    mma<E4M3>(s.o[k], f, b[i][0], b[i][1]);
                                    mma<E4M3>(d, f, lo[i][0], lo[i][1]);
                                }
#pragma unroll
                                for (int j = 0; j < 4; ++j) s.o[k][j] = fmaf(d[j], 1.0f / kSmallScale, s.o[k][j]);
                            }
                        }
                    }
                }
                if constexpr (!E4M3) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        uint32_t f[4];
                        ldsm_x4_trans(((values + value_off + step * kWarpBytes) ^ ((k & 3) << 5)) + (k >> 2) * 4096, f);
                        mma<E4M3>(s.o[k], f, b[0][0], b[0][1]);
                    }
                } else if (!added) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        uint32_t w[4], f[4];
                        ldsm_bytes_trans((values + value_off + step * kWarpBytes) ^ (k << 4), w);
#pragma unroll
                        for (int i = 0; i < kGroups; ++i) {
                            codes_to_halves(w[2 * i], w[2 * i + 1], f);
                            mma<E4M3>(s.o[k], f, b[i][0], b[i][1]);
                        }
                    }
                }
            }
            if (flags & kLast) break;
            release();
            if (!wait()) return;
        }
        if constexpr (E4M3 && ONE)
#pragma unroll
            for (int k = 0; k < 8; ++k)
#pragma unroll
                for (int i = 0; i < 4; i += 2) s.o[k][i] = fmaf(s.o[k][i + 1], 1.0f / kSmallScale, s.o[k][i]);
        // what this warp has of the item, into its rows of the stage
        if (a.cols.warps > 1 && !consumers_meet(sh, met, kv.status, a.p.wait_ns)) return;  // (others read them)
#pragma unroll
        for (int j = 0; j < (ONE ? 1 : 2); ++j) {
            float l = s.l[j];
            if constexpr (ONE) {
                l += __shfl_xor_sync(0xffffffffu, l, 1);
                if constexpr (E4M3) l += __shfl_xor_sync(0xffffffffu, l, 2);
            }
            l += __shfl_xor_sync(0xffffffffu, l, 4);
            l += __shfl_xor_sync(0xffffffffu, l, 8);
            l += __shfl_xor_sync(0xffffffffu, l, 16);
            const int col = 2 * c + j;
            if (g == 0) {
                const int at = (col_warp * 8 + col) * key_warps + key_warp;
                sh.part_l[st][at] = l;
                sh.part_m[st][at] = s.m[j];
                if constexpr (E4M3) sh.part_w[st][at] = s.w[j];
            }
            if (ONE && c > 0) continue;
            uint8_t* const to = tile + meet_byte(warp, col);
#pragma unroll
            for (int k = 0; k < 8; ++k)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int d = 16 * k + g + 8 * i;
                    *reinterpret_cast<float*>(to + ((d + meet_turn(col)) & 127) * 4) = s.o[k][2 * i + j];
                }
        }
        fence_proxy_async();  // (the stage's next contents come by TMA)
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&sh.done[st]));
        release();
        if (flags & kEnd) break;
    }
    if (!wait_warp(smem_u32(&sh.joined), 0, &sh.abort, kv.status, a.p.wait_ns)) return;
    if (sh.pending[0].join || sh.pending[1].join)
        join_pending<E4M3>(parts_in(a), a.p.out, a.p.H, a.cols.group, a.cols.block, sh.pending, kv.status,
                           2 * warp + (lane >> 4), 2 * (kWarps + 1));
}

template <bool E4M3, bool ONE>
__global__ void __launch_bounds__(kThreads, kCtasPerSm)
    attention_decode_kernel(const __grid_constant__ CacheMaps maps, const __grid_constant__ DecodeArgs a) {
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ Shared sh;
    // (the dynamic part starts past the static one: rounded up to the swizzle's 1024 bytes)
    const uint32_t raw = smem_u32(smem), up = (1024 - (raw & 1023)) & 1023;
    uint8_t* const stage_mem = smem + up;
    uint8_t* const query_mem = stage_mem + kStages * kStageBytes;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) {
        prefetch_tmap(&maps.box);
        prefetch_tmap(&maps.group);
        for (int i = 0; i < kStages; ++i) {
            mbar_init(smem_u32(&sh.full[i]), E4M3 ? 33 : 1);
            mbar_init(smem_u32(&sh.empty[i]), kWarps + 1);
            mbar_init(smem_u32(&sh.done[i]), kWarps);
        }
        mbar_init(smem_u32(&sh.met), kWarps);
        mbar_init(smem_u32(&sh.joined), 1);
        sh.pending[0] = sh.pending[1] = Pending{};
        sh.start_base = sh.start_row = sh.start_item = sh.start_into = sh.empty_rows = sh.twice = 0;
        sh.bound[0] = sh.bound[1] = 0;
        sh.start = Row{};
        sh.abort = 0;
        fence_mbar_init();
    }
    // (a bit for each slot, at most 8 KB, before the stages' first copies)
    uint32_t* const seen = reinterpret_cast<uint32_t*>(stage_mem);
    static_assert(kKvMaxSlots / 8 <= kStageBytes);
    for (int i = tid; i < (a.kv.num_slots + 31) / 32; i += kThreads) seen[i] = 0;
    grid_launch_dependents();
    grid_wait();
    __syncthreads();

    // The batch's weight, this CTA's share of it, and the row where it starts.  (Each load is
    // a microsecond's part: a batch of up to kThreads rows is read once.)
    const int items = a.kv.kv_heads * a.cols.blocks;
    const bool any = any_refused(a.kv);
    auto seen_before = [&](int i) {  // (a list of one has none)
        const int slot = a.p.n > 1 && i < a.p.n ? a.p.slots[i] : -1;
        if (slot < 0 || slot >= a.kv.num_slots) return false;
        const uint32_t bit = 1u << (slot & 31);
        return (atomicOr(&seen[slot >> 5], bit) & bit) != 0;
    };
    auto weigh = [&](int i, Row* r) -> int64_t {
        *r = Row{};
        if (i >= a.p.n) return 0;
        bool bad;
        *r = row_of<E4M3>(a, any, i, &bad);
        if (r->tiles == 0 && i % gridDim.x == blockIdx.x) {
            sh.empty_rows = 1;
            if (bad) record_status(a.kv.status, kInvalid);
        }
        return static_cast<int64_t>(r->weight) * items;
    };
    // the sum of v over the threads before this one and its own, and over all
    auto scan = [&](int64_t v, int64_t* all) {
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t t = __shfl_up_sync(0xffffffffu, v, o);
            if (lane >= o) v += t;
        }
        if (lane == 31) sh.warp_sum[warp] = v;
        __syncthreads();
        *all = 0;
        for (int w = 0; w < kThreads / 32; ++w) {
            if (w == warp) v += *all;
            *all += sh.warp_sum[w];
        }
        return v;
    };
    Row r;
    bool again = seen_before(tid);
    int64_t all, weight = 0, v = weigh(tid, &r);
    if (again) sh.twice = 1;
    int64_t upto = scan(v, &all);
    weight = all;
    for (int i0 = kThreads; i0 < a.p.n; i0 += kThreads) {
        __syncthreads();
        Row other;
        again = seen_before(i0 + tid);
        const int64_t w = weigh(i0 + tid, &other);
        if (again) sh.twice = 1;
        scan(w, &all);
        weight += all;
    }
    if (a.p.n > 1) fence_proxy_async();  // (the slots' bits, before the copies)
    // Two rows of one slot would both be its last token: nothing is stored, and all rows are zero.
    const bool twice = sh.twice != 0;
    if (twice && blockIdx.x == 0 && tid == 0) record_status(a.kv.status, kInvalid);
    // rows without keys are zero
    if (sh.empty_rows || twice)
        for (int i = blockIdx.x; i < a.p.n; i += gridDim.x) {
            bool bad;
            if (!twice && row_of<E4M3>(a, any, i, &bad).tiles > 0) continue;
            uint4* const out = reinterpret_cast<uint4*>(a.p.out + static_cast<int64_t>(i) * a.p.H * kKvHeadDim);
            for (int j = tid; j < a.p.H * (kKvHeadDim / 8); j += kThreads) out[j] = make_uint4(0, 0, 0, 0);
        }
    if (weight == 0 || twice) return;
    // as many CTAs as leave each at least the most that lies between two tiles' starts
    const int apart = (E4M3 ? 8 : 4) + a.item_weight;
    const bool full = weight >= static_cast<int64_t>(apart) * gridDim.x;
    const int64_t ctas = full ? gridDim.x : weight < apart ? 1 : quotient(weight, apart);
    if (blockIdx.x >= ctas) return;
    // (a batch of any size: less than 2^48 groups, so the multiplication is exact)
    const int64_t w0 = full ? __umul64hi(blockIdx.x * weight, a.grid_reciprocal) : quotient(blockIdx.x * weight, ctas);
    const int64_t w1 = full ? __umul64hi((blockIdx.x + 1) * weight, a.grid_reciprocal)
                            : quotient((blockIdx.x + 1) * weight, ctas);
    int64_t before = 0;
    for (int i0 = 0;;) {
        const int64_t begin = before + upto - v, end = before + upto;
        if (begin <= w0 && w0 < end) {
            const int64_t item = quotient(w0 - begin, r.weight), at = begin + item * r.weight;
            const int into = snapped(static_cast<int>(w0 - at), r.weight, a.snap);
            sh.bound[0] = at + into;
            sh.start_row = i0 + tid;
            sh.start_base = begin;
            sh.start = r;
            sh.start_item = static_cast<int>(item) + (into == r.weight);
            sh.start_into = into == r.weight ? 0 : into;
        }
        if (begin <= w1 && w1 < end) {
            const int64_t at = begin + quotient(w1 - begin, r.weight) * r.weight;
            sh.bound[1] = at + snapped(static_cast<int>(w1 - at), r.weight, a.snap);
        }
        if (w1 == weight) sh.bound[1] = weight;
        if (i0 == 0 && a.p.n > kThreads) {
            __syncthreads();
            scan(v, &all);  // (the first block's again)
        }
        before += all;
        i0 += kThreads;
        if (i0 >= a.p.n || before > w1) break;
        __syncthreads();
        v = weigh(i0 + tid, &r);
        upto = scan(v, &all);
    }
    __syncthreads();
    if (sh.bound[0] == sh.bound[1]) return;
    if (warp == 0)
        produce<E4M3>(a, maps, sh, smem_u32(stage_mem), smem_u32(query_mem), weight, ctas, sh.bound[1]);
    else if (warp <= kWarps)
        consume<E4M3, ONE>(a, sh, stage_mem, query_mem);
    else
        finish<E4M3>(a, sh, stage_mem);
}

template <bool E4M3, bool ONE>
cudaError_t launch(const CacheMaps& maps, const DecodeArgs& a, int grid, cudaStream_t stream) {
    auto kern = attention_decode_kernel<E4M3, ONE>;
    const int bytes = 1024 + kStages * kStageBytes + 2 * a.cols.block * kQueryStride;
    cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != cudaSuccess) return e;
    return launch_overlapped(kern, grid, kThreads, bytes, stream, maps, a);
}

}  // namespace

// A counter for each CTA, then two parts for each.
int64_t decode_workspace_bytes(int H, int kv_heads, int sm_count) {
    const int64_t ctas = static_cast<int64_t>(sm_count) * kCtasPerSm;
    return counter_bytes(static_cast<int>(ctas)) + ctas * 2 * part_floats(used_columns(H / kv_heads)) * 4;
}

int encode_cache(CacheMaps* maps, const KvView& kv, int layer) {
    const bool e4m3 = kv.exponents != nullptr;
    const uint64_t row = kv.row_bytes, groups = (static_cast<uint64_t>(kv.num_pages) * kv.kv_heads << kv.page_shift) / 16;
    const uint32_t halves = e4m3 ? 1 : 2, tile_groups = e4m3 ? 8 : 4, page_groups = (1u << kv.page_shift) / 16;
    maps->groups = static_cast<int>(page_groups < tile_groups ? page_groups : tile_groups);
    // elements of half a row, the rows of a group, keys and values, halves, groups
    const uint64_t dims[5] = {row / halves / (e4m3 ? 1 : 2), 16, 2, halves, groups};
    const uint64_t strides[4] = {row, groups * 16 * row, row / halves, 16 * row};
    for (int i = 0; i < 2; ++i) {
        const uint32_t box[5] = {static_cast<uint32_t>(dims[0]), 16, 2, halves, i == 0 ? static_cast<uint32_t>(maps->groups) : 1u};
        const int rc = encode_5d(i == 0 ? &maps->box : &maps->group,
                                 e4m3 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16,
                                 kv.pages + 2 * groups * 16 * row * layer, dims, strides, box);
        if (rc != 0) return rc;
    }
    return 0;
}

cudaError_t launch_attention_decode(const CacheMaps& maps, const KvView& kv, const DecodeParams& p, int sm_count,
                                    cudaStream_t stream) {
    DecodeArgs a{kv, p, columns_of(p.H / kv.kv_heads), 0, 0, 0};
    const int grid = sm_count * kCtasPerSm;
    const bool e4m3 = kv.exponents != nullptr;
    // (measured with 3 / 5 / 8 / 12 / 16 / 20.  bf16: 64 pairs 288 / 290 / 291 / 291 us, 200 short
    // rows 68 / 61 / 55 / 57; e4m3: 168 / 163 / 157 / 155 / 155 / 158 and 91 / 80 / 71 / 61 / 58 / 58, 64
    // rows of 8 key heads and 12 queries each 34.4 / 33.6 / 33.6 / 33.8 / 34.7 / 35.4)
    a.item_weight = e4m3 ? 12 : 8;
    a.snap = a.item_weight + (e4m3 ? 12 : 10);
    a.grid_reciprocal = ~uint64_t{0} / grid + 1;
    if (p.H == kv.kv_heads) return e4m3 ? launch<true, true>(maps, a, grid, stream) : launch<false, true>(maps, a, grid, stream);
    return e4m3 ? launch<true, false>(maps, a, grid, stream) : launch<false, false>(maps, a, grid, stream);
}

}  // namespace w4a16
