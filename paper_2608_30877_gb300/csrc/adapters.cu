// Low-rank adapters of many sequences beside a shared projection:
//   out = base + t B_a^T,  t = scale_a (x A_a^T),  a the adapter of the row's sequence.
//
// Two kernels.  The first reads x and gives t.  Long sequences: 128 tokens of x and the tile's adapters by
// TMA into a ring of stages, tcgen05 MMAs (tokens as rows, an adapter's rank as columns) into tensor memory.
// Short ones: warp-level MMAs with the adapter's rows as the 16-row operand and eight tokens as columns.
// K is split over the CTAs of a cluster, whose fp32 sums are added up in order through distributed shared
// memory; t goes to the workspace with 12 significant bits in 16 (pack_t), which the second takes as two bf16
// parts, a product with B each: what is left of t's rounding is 2^-12 of an update whose sum with base a bf16 store
// rounds to 2^-8.  The second streams base and
// out, with tokens as rows and 32 features as columns of its MMAs, arranged so that a thread has eight
// neighbours: the accumulators begin as base and are stored as out, 16 bytes a thread.
// Rows of a tile that share an adapter are done together.
//
// Bound by HBM: the rank gives a product 2 R FLOPs a byte of x.  39004 tokens, 12288 x 12288, eight adapters of rank
// 16: 136 us (x at 6.4 TB/s) and 313 (base and out at 6.1), 457 together.  Before: mma.sync on x through registers
// 240 us, through shared memory by 16-byte copies 195; the second kernel with an address computed for every load
// 340.  1363 tokens on 49152 x 12288, rank 64: 40 + 32 us cold, 70 together (33 at the copy bandwidth): one turn of 176 CTAs,
// and an adapter's rows that come from L2 for every tile, as many bytes as x.  64 requests of one token with 48 adapters,
// 12288 x 36864: 21 us (11.3): each kernel starts with the adapters' numbers, a list of them, and only then loads, and the
// second waits for the first before that.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "kv.h"
#include "layer.h"
#include "ptx.cuh"
#include "sequences.cuh"

namespace w4a16 {

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kNone = -1;     // a row without an adapter
constexpr int kOutside = -2;  // past the last row

__device__ __forceinline__ float bf16_low(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float bf16_high(uint32_t v) { return __uint_as_float(v & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&p);
}

__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// t in the workspace: eight ranks of a token in 16 bytes.  E is the exponent field of the largest; each has its sign, 14
// bits of |t| / 2^(E - 127) < 2 as a small float (three of exponent, eleven of mantissa: 2^-12 of the value down to 2^-6
// of the largest, 2^-18 of that below) and, lowest, its bit of E.  With E 255, an infinity or a NaN among the eight, they
// are bf16 without the last bit.
// A lane has one of the eight, those of its aligned group of lanes; all lanes take part.
__device__ __forceinline__ uint32_t pack_t(float v) {
    uint32_t top = __float_as_uint(v) & 0x7FFFFFFFu;
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    const uint32_t E = top >> 23;
    if (E == 255u) return __float_as_uint(v) >> 16 | (v != v ? 0x41u : 1u);
    const float unit = __uint_as_float(E == 254u ? 0x00400000u : (254u - E) << 23);  // 2^(127 - E)
    const uint32_t g = __float_as_uint(v * unit * 0x1p-120f), m = g & 0x7FFFFFFFu;  // (1 has exponent field 7)
    return g >> 31 << 15 | min((m + 0x7FFu + (m >> 12 & 1u)) >> 12, 0x3FFFu) << 1 | (E >> (threadIdx.x & 7) & 1u);
}

// Two of those eight as two bf16 each, whose sum they are: the upper eight bits (`first`) and the others.  The second part
// of a number other than 0 is not 0 either (2^-126 at least), so that its product with an infinity is one.  A lane has
// the two of its number in its aligned group of four lanes; all lanes take part.
__device__ __forceinline__ void unpack_t(uint32_t packed, uint32_t* first, uint32_t* second) {
    uint32_t E = ((packed & 1u) | (packed >> 15 & 2u)) << (2 * (threadIdx.x & 3));
    E |= __shfl_xor_sync(0xffffffffu, E, 1);
    E |= __shfl_xor_sync(0xffffffffu, E, 2);
    const float unit = __uint_as_float(E == 0 ? 0x00400000u : E << 23);  // 2^(E - 127)
    uint32_t a[2], b[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t c = packed >> (16 * h) & 0xFFFEu;
        uint32_t v = c << 16;
        float low = 0.0f;
        if (E != 255u) {
            const float x = __uint_as_float((c & 0x8000u) << 16 | (c & 0x7FFFu) << 11) * 0x1p120f * unit;
            v = __float_as_uint(x);
            low = x - __uint_as_float(v & 0xFFFF0000u);
        }
        a[h] = v >> 16;
        b[h] = low != 0.0f || v << 1 == 0u ? __float_as_uint(low) >> 16 : 0x80u | (a[h] & 0x8000u);
    }
    *first = a[0] | a[1] << 16;
    *second = b[0] | b[1] << 16;
}

// The rows of a tile: each one's adapter, the list of those that occur, and each row's place in it (-1: no
// adapter).
template <int ROWS>
struct Tile {
    int id[ROWS];
    int slot[ROWS];
    int list[ROWS];
    int count;
};

// The last of n entries that is <= m, by one warp (32 probes a round); -1 if there is none.
__device__ __forceinline__ int last_start(const int32_t* starts, int n, int64_t m) {
    const int lane = threadIdx.x & 31;
    int lo = 0;
    while (true) {
        const int step = (n + 31) / 32;
        const uint32_t before = __ballot_sync(0xffffffffu, lane * step < n && starts[lo + lane * step] <= m);
        const int c = __popc(before);
        if (c == 0) return -1;
        lo += (c - 1) * step;
        n = min(step, n - (c - 1) * step);
        if (step == 1) return lo;
    }
}

// All threads; ends behind a barrier.  The tile's first sequence is searched by one warp, the rows' in
// the starts behind it.
template <int ROWS>
__device__ __forceinline__ void find_adapters(Tile<ROWS>& tile, const AdapterParams& p, int64_t m0, bool check) {
    constexpr int kStarts = 96;
    __shared__ int32_t starts[kStarts];
    __shared__ int first_sequence;
    const int t = static_cast<int>(threadIdx.x), lane = t & 31;
    if (p.seq_start != nullptr) {
        if (t < 32) {
            const int s = max(last_start(p.seq_start, p.nseq + 1, m0), 0);
            if (lane == 0) first_sequence = s;
            for (int i = lane; i < kStarts; i += 32)
                starts[i] = p.seq_start[min(static_cast<int64_t>(s) + i, static_cast<int64_t>(p.nseq))];
        }
        __syncthreads();
    }
    if (t < ROWS) {
        const int64_t m = m0 + t;
        int id = kOutside;
        if (m < p.M) {
            int begin = 0, end = p.M, s = static_cast<int>(m);
            id = kNone;
            if (p.seq_start != nullptr) {
                int lo = 0, hi = kStarts - 1;
                while (lo < hi) {
                    const int mid = (lo + hi + 1) >> 1;
                    if (starts[mid] <= m) lo = mid; else hi = mid - 1;
                }
                s = first_sequence + lo;
                if (lo == kStarts - 1) {  // (many empty sequences)
                    s = sequence_of(p.seq_start, p.nseq, static_cast<int>(m), &begin, &end);
                } else {
                    begin = starts[lo];
                    end = starts[lo + 1];
                    if (s >= p.nseq || begin > m || m >= end) s = -1;
                }
            }
            if (s >= 0 && begin >= 0 && end <= p.M) {
                id = p.ids[s];
                if (id < -1 || id >= p.pool) {
                    if (check) record_status(p.status, 1 /* W4A16_ERR_INVALID_ARG */);
                    id = kNone;
                }
            }
        }
        tile.id[t] = id;
    }
    __syncthreads();
    if (t < 32) {  // the first row of each adapter, in order
        int n = 0;
#pragma unroll
        for (int i0 = 0; i0 < ROWS; i0 += 32) {
            const int id = i0 + lane < ROWS ? tile.id[i0 + lane] : kOutside;
            const uint32_t same = __match_any_sync(0xffffffffu, id);  // (every lane takes part)
            bool first = id >= 0 && (same & ((1u << lane) - 1u)) == 0;
            for (int j = 0; j < n; ++j) first = first && tile.list[j] != id;
            const uint32_t mask = __ballot_sync(0xffffffffu, first);
            __syncwarp();
            if (first) tile.list[n + __popc(mask & ((1u << lane) - 1u))] = id;
            __syncwarp();
            n += __popc(mask);
        }
        if (lane == 0) tile.count = n;
    }
    __syncthreads();
    if (t < ROWS) {
        int slot = -1;
        if (tile.id[t] >= 0)
            for (slot = 0; slot < tile.count - 1 && tile.list[slot] != tile.id[t]; ++slot) {}  // (it is in the list)
        tile.slot[t] = slot;
    }
    __syncthreads();
}

__device__ __forceinline__ uint4 load16(const uint16_t* p) { return __ldg(reinterpret_cast<const uint4*>(p)); }

// 32 k of 16 MT rows of an adapter with eight tokens: a lane has 16 bytes of its rows g and g + 8 of
// each 16 and of its token g, of which each MMA takes half; the order of k is the same on both sides.
template <int MT>
__device__ __forceinline__ void mma_step(float (&acc)[MT][4], const uint4 (&a)[MT][2], const uint4& x) {
#pragma unroll
    for (int i = 0; i < MT; ++i) mma_bf16(acc[i], a[i][0].x, a[i][1].x, a[i][0].y, a[i][1].y, x.x, x.y);
#pragma unroll
    for (int i = 0; i < MT; ++i) mma_bf16(acc[i], a[i][0].z, a[i][1].z, a[i][0].w, a[i][1].w, x.z, x.w);
}

// This CTA's slice of the steps that K takes.
struct Slice {
    int from, to;
    __device__ __forceinline__ explicit Slice(int64_t steps) {
        from = static_cast<int>(steps * blockIdx.y / gridDim.y);
        to = static_cast<int>(steps * (blockIdx.y + 1) / gridDim.y);
    }
};

__device__ __forceinline__ float load_cluster(uint32_t at) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
    return v;
}

// PARTS sums [ROWS][16 MT + 4] added up, in order, then those of the cluster's CTAs (gridDim.y of them), for
// the tokens of the adapters first .. last - 1 of the tile's list.  All threads; the sums may be overwritten
// after it.
template <int THREADS, int PARTS, int ROWS, int MT>
__device__ __forceinline__ void store_t(float* sums, const Tile<ROWS>& tile, const AdapterParams& p, int64_t m0, int first,
                                        int last) {
    constexpr int kPitch = 16 * MT + 4, kAll = ROWS * 16 * MT;
    const int ctas = static_cast<int>(gridDim.y);
    __syncthreads();
    if constexpr (PARTS > 1)
        for (int i = threadIdx.x; i < kAll; i += THREADS) {
            float* const at = sums + i / (16 * MT) * kPitch + i % (16 * MT);
            float sum = at[0];
#pragma unroll
            for (int w = 1; w < PARTS; ++w) sum += at[w * ROWS * kPitch];
            at[0] = sum;
        }
    if (ctas > 1) cluster_sync(); else if (PARTS > 1) __syncthreads();
    // each CTA adds up a part of the tokens
    static_assert(THREADS % 32 == 0 && kAll % 32 == 0, "whole warps");
    uint16_t* const out = p.t + m0 * p.R;
    for (int i = blockIdx.y * THREADS + threadIdx.x; i < kAll; i += ctas * THREADS) {
        const int token = i / (16 * MT), r = i % (16 * MT), slot = tile.slot[token];
        const bool mine = slot >= first && slot < last && r < p.R;
        float sum = 0.0f;
        if (mine) {
            const float* const at = sums + token * kPitch + r;
            if (ctas > 1) {
                const uint32_t local = smem_u32(at);
                for (int c = 0; c < ctas; ++c) sum += load_cluster(mapa_shared(local, c));
            } else {
                sum = at[0];
            }
            sum *= p.scale[tile.id[token]];
        }
        const uint32_t code = pack_t(sum);
        if (mine && dbg_check(m0 + token < p.M, p.status)) out[static_cast<int64_t>(token) * p.R + r] = static_cast<uint16_t>(code);
    }
    if (ctas > 1) cluster_sync(); else __syncthreads();
}

// D[tmem] (+)= A[smem] * B[smem]^T, kind::f16 (bf16 inputs, fp32 accumulator).
__device__ __forceinline__ void tc_mma_ss(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc,
                                          uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}

// One box of 64 columns of rows (of five dimensions, of which three have one entry).
__device__ __forceinline__ void load_rows(uint32_t to, const CUtensorMap* map, uint32_t bar, int32_t column, int32_t row) {
    asm volatile(
        "cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%3, %4, %2, %2, %2}], [%5];" ::"r"(to),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(column), "r"(row), "r"(bar)
        : "memory");
}

// t of 128 tokens (blockIdx.x) over a slice of K (blockIdx.y), for up to kGroup of the tile's adapters at
// once.  A stage of the ring: 64 k of the tokens, and of each adapter's rank (rounded up to 16: what the
// last rows hold is another adapter's, and not looked at).  Warps 0 to 3 take the sums out of tensor
// memory, one thread of warp 4 copies, one of warp 5 issues the MMAs.
constexpr int kTcRows = 128, kTcThreads = 192;
template <int MT>
struct TcLayout {
    static constexpr int kRank = 16 * MT, kGroup = MT <= 2 ? 4 : 2;
    static constexpr int kTokens = kTcRows * 128, kAdapter = kRank * 128;  // bytes
    static constexpr int kStage = kTokens + kGroup * kAdapter, kStages = MT == 1 ? 4 : 3;
    static constexpr int kColumns = kGroup * kRank <= 64 ? 64 : 128;       // of tensor memory
    static constexpr int kSums = kTcRows * (kRank + 4) * 4;
    static constexpr int kSmem = kStages * kStage + 1024;                  // (the ring begins on 1024 bytes)
    static_assert(kSums <= kStages * kStage, "the sums take the ring's place");
};

template <int MT>
__global__ void __launch_bounds__(kTcThreads, 2)
    adapters_down_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_a,
                         const AdapterParams p) {
    using L = TcLayout<MT>;
    __shared__ Tile<kTcRows> tile;
    __shared__ __align__(8) uint64_t full[L::kStages], empty[L::kStages], done, drain;
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag;
    extern __shared__ uint8_t dynamic[];
    const uint32_t ring = (smem_u32(dynamic) + 1023u) & ~1023u;
    float* const sums = reinterpret_cast<float*>(dynamic + (ring - smem_u32(dynamic)));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t m0 = static_cast<int64_t>(blockIdx.x) * kTcRows;
    if (threadIdx.x == 0) {
        for (int i = 0; i < L::kStages; ++i) {
            mbar_init(smem_u32(&full[i]), 1);
            mbar_init(smem_u32(&empty[i]), 1);
        }
        mbar_init(smem_u32(&done), 1);
        mbar_init(smem_u32(&drain), 1);
        abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == 5) {
        tmem_alloc(smem_u32(&tmem_slot), L::kColumns);
        tmem_relinquish();
    }
    grid_wait();
    find_adapters<kTcRows>(tile, p, m0, blockIdx.y == 0);
    if (p.seq_start != nullptr && blockIdx.y == 0) check_starts(p.seq_start, p.nseq, p.M, p.status);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    const Slice k(p.K / 64);
    uint32_t it = 0;    // stages so far
    bool alive = true;  // no wait of this CTA ran out: else only the cluster's barriers are kept
    for (int l = 0, turn = 0; l < tile.count; l += L::kGroup, ++turn) {
        const int n = min(L::kGroup, tile.count - l);
        bool ok = true, drained = false;  // drained: the MMAs' last commit is to `drain`
        if (alive && warp == 4) {
            if (lane == 0) {
                for (int s = k.from; s < k.to; ++s, ++it) {
                    const uint32_t stage = it % L::kStages, at = ring + stage * L::kStage, bar = smem_u32(&full[stage]);
                    if (it >= L::kStages && !wait_one(smem_u32(&empty[stage]), (it / L::kStages - 1) & 1u, &abort_flag,
                                                      p.status, p.wait_ns)) {
                        ok = false;
                        break;
                    }
                    mbar_arrive_expect_tx(bar, L::kTokens + n * L::kAdapter);
                    const uint32_t end = ring + L::kStages * L::kStage;
                    if (dbg_check(tma_box_ok(at, L::kTokens, 1024, ring, end, s * 64, 2), p.status))
                        load_rows(at, &map_x, bar, s * 64, static_cast<int32_t>(m0));
                    for (int i = 0; i < n; ++i) {
                        const uint32_t to = at + L::kTokens + i * L::kAdapter;
                        if (dbg_check(tma_box_ok(to, L::kAdapter, 1024, ring, end, s * 64, 2), p.status))
                            load_rows(to, &map_a, bar, s * 64, tile.list[l + i] * p.R);
                    }
                    if (it == 0 && !short_limit_ok(bar, 0, &abort_flag, p.status, p.wait_ns)) {
                        ++it;
                        ok = false;
                        break;
                    }
                }
            }
            __syncwarp();
            it = __shfl_sync(0xffffffffu, it, 0);
        } else if (alive && warp == 5) {
            constexpr uint32_t kIdesc = idesc_bf16_f32(kTcRows, L::kRank);
            for (int s = k.from; s < k.to; ++s, ++it) {
                const uint32_t stage = it % L::kStages, at = ring + stage * L::kStage;
                if (!wait_warp(smem_u32(&full[stage]), (it / L::kStages) & 1u, &abort_flag, p.status, p.wait_ns)) {
                    ok = false;
                    break;
                }
                tc_fence_after();
                if (elect_one()) {
                    const uint64_t x = sdesc_kmajor_sw128(at);
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk)  // 16 k: 32 bytes
                        for (int i = 0; i < n; ++i)
                            tc_mma_ss(tmem + i * L::kRank, x + 2 * kk,
                                      sdesc_kmajor_sw128(at + L::kTokens + i * L::kAdapter) + 2 * kk, kIdesc,
                                      s > k.from || kk > 0);
                    tc_commit(smem_u32(&empty[stage]));
                }
                __syncwarp();
            }
            if (elect_one()) tc_commit(smem_u32(ok ? &done : &drain));
            __syncwarp();
            drained = !ok;
        } else if (alive && warp < 4) {
            ok = wait_warp<false, 64>(smem_u32(&done), turn & 1, &abort_flag, p.status, p.wait_ns);
            if (ok) {
                tc_fence_after();
                const int token = warp * 32 + lane, mine = tile.slot[token] - l;
                for (int i = 0; i < n; ++i)
#pragma unroll
                    for (int c = 0; c < MT; ++c) {
                        uint32_t v[16];
                        tmem_ld_32x32b_x16(tmem + (static_cast<uint32_t>(warp * 32) << 16) + i * L::kRank + c * 16, v);
                        tmem_ld_wait_x16(v);
                        if (mine == i) {
                            float4* const to = reinterpret_cast<float4*>(sums + token * (L::kRank + 4) + c * 16);
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                to[e] = make_float4(__uint_as_float(v[4 * e]), __uint_as_float(v[4 * e + 1]),
                                                    __uint_as_float(v[4 * e + 2]), __uint_as_float(v[4 * e + 3]));
                        }
                    }
                tc_fence_before();
            }
        }
        // A CTA in which any role gave up lets all that it has in flight end, whatever the others' own waits said (a
        // producer with a stage for every copy waits for none, and MMAs may all have been issued): the last copy into each
        // stage, and the commit behind the MMAs.
        if (__syncthreads_or(alive && !ok) && alive) {
            alive = false;
            if (warp == 4 && lane == 0)
                for (uint32_t i = it > L::kStages ? it - L::kStages : 0; i < it; ++i)
                    settle(smem_u32(&full[i % L::kStages]), (i / L::kStages) & 1u);
            if (warp == 5) settle(smem_u32(drained ? &drain : &done), drained ? 0 : turn & 1);
            __syncthreads();
        }
        store_t<kTcThreads, 1, kTcRows, MT>(sums, tile, p, m0, l, l + n);
        // (the next copies into the ring come behind what was read and written here)
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        tc_fence_before();
        __syncthreads();
        tc_fence_after();
    }
    // (not before: the second kernel's CTAs would come to wait beside these, on SMs whose shared memory is laid out
    // for the ring, and run there by a few an SM: 39004 rows 654 us, 467 so)
    grid_launch_dependents();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 5) tmem_dealloc(tmem, L::kColumns);
}

// The same for short sequences: 8 tokens (blockIdx.x), one of the tile's adapters (blockIdx.z), a slice of
// K that its warps have under way at once.
template <int MT>
__global__ void __launch_bounds__(kThreads) adapters_down_few_kernel(const AdapterParams p) {
    constexpr int kRows = 8, U = MT == 1 ? 4 : 2;
    __shared__ Tile<kRows> tile;
    constexpr int kPitch = 16 * MT + 4;
    __shared__ float sums[kWarps * kRows * kPitch];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, q = lane & 3;
    const int64_t m0 = static_cast<int64_t>(blockIdx.x) * kRows;
    grid_launch_dependents();
    grid_wait();
    find_adapters<kRows>(tile, p, m0, blockIdx.y == 0 && blockIdx.z == 0);
    if (p.seq_start != nullptr && blockIdx.y == 0 && blockIdx.z == 0) check_starts(p.seq_start, p.nseq, p.M, p.status);
    const Slice k(p.K / 32);
    for (int l = blockIdx.z; l < tile.count; l += gridDim.z) {
        const int a = tile.list[l];
        const bool mine = tile.id[g] == a;
        const uint16_t* const x = p.x + (m0 + g) * p.K + 8 * q;
        const uint16_t* const w = p.a + (static_cast<int64_t>(a) * p.R + g) * p.K + 8 * q;
        float acc[MT][4] = {};
        for (int s = k.from + warp; s < k.to; s += kWarps * U) {
            uint4 xv[U], av[U][MT][2];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const bool in = s + u * kWarps < k.to;
                const int at = (s + u * kWarps) * 32;
                xv[u] = make_uint4(0, 0, 0, 0);
                if (in && mine) xv[u] = load16(x + at);
#pragma unroll
                for (int i = 0; i < 2 * MT; ++i) {
                    av[u][i / 2][i % 2] = make_uint4(0, 0, 0, 0);
                    if (in && i * 8 + g < p.R) av[u][i / 2][i % 2] = load16(w + static_cast<int64_t>(i * 8) * p.K + at);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) mma_step<MT>(acc, av[u], xv[u]);
        }
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                sums[(warp * kRows + 2 * q + (e & 1)) * kPitch + i * 16 + g + (e & 2) * 4] = acc[i][e];
        store_t<kThreads, kWarps, kRows, MT>(sums, tile, p, m0, l, l + 1);
    }
}

// Rank in the second product: 16, or CH times 32 (CH 0: 16).  A lane has as many k of its rows in one
// piece as two MMAs take (one for 16), in the same order on both sides.
template <int CH>
struct UpFragments {
    static constexpr int kSteps = CH == 0 ? 1 : 2 * CH;  // MMAs
    uint32_t w[kSteps][2];

    // q: the lane's place among the four of a row
    template <bool EXACT>
    __device__ __forceinline__ void load_b(const uint16_t* row, int q, int R) {
        if constexpr (CH == 0) {
            uint2 v = make_uint2(0, 0);
            if (EXACT || 4 * q < R) v = __ldg(reinterpret_cast<const uint2*>(row + 4 * q));
            w[0][0] = v.x, w[0][1] = v.y;
        } else {
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                uint4 v = make_uint4(0, 0, 0, 0);
                if (EXACT || 32 * c + 8 * q < R) v = load16(row + 32 * c + 8 * q);
                w[2 * c][0] = v.x, w[2 * c][1] = v.y, w[2 * c + 1][0] = v.z, w[2 * c + 1][1] = v.w;
            }
        }
    }
};

// 16 rows and 16 k of t's parts in shared memory, as an MMA takes them: lanes 8 i .. 8 i + 7 have the rows' addresses of
// piece i.
__device__ __forceinline__ void load_t(uint32_t (&w)[4], const uint32_t* row) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
                 : "r"(smem_u32(row))
                 : "memory");
}

// out of a tile of tokens (blockIdx.x) and `chunk` blocks of 32 features (blockIdx.y), for the tile's
// adapters blockIdx.z, + gridDim.z, ...; a warp has FB blocks under way.  MB: 16s of tokens, with an MMA for each
// part of t; 0: eight, the upper half of one for its first part, the lower for the second.  EXACT: the rank is 16
// or 32 CH.  WHOLE: rows of 16-byte units.
template <int CH, int MB, int FB, bool EXACT, bool WHOLE>
__global__ void __launch_bounds__(kThreads, !WHOLE ? 1 : 2)
    adapters_up_kernel(const AdapterParams p, const int chunk) {
    constexpr int kRows = MB == 0 ? 8 : 16 * MB, kHalves = MB == 0 ? 1 : 2 * MB;  // rows of a lane
    constexpr int kWords = CH == 0 ? 8 : 16 * CH, kPitch = kWords + 4;            // (pairs of bf16)
    __shared__ Tile<kRows> tile;
    __shared__ __align__(16) uint32_t t[2][kRows][kPitch];  // t's two parts
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, q = lane & 3;
    const int64_t m0 = static_cast<int64_t>(blockIdx.x) * kRows;
    grid_launch_dependents();
    grid_wait();
    find_adapters<kRows>(tile, p, m0, false);
    static_assert(kRows * kWords % 32 == 0, "whole warps");
    for (int i = threadIdx.x; i < kRows * kWords; i += kThreads) {
        const int row = i / kWords, word = i % kWords;
        const bool there = tile.id[row] >= 0 && 2 * word < p.R;
        // (in the order in which the products take them: a lane's pieces of B are k in a row of several MMAs)
        const int at = CH == 0 ? word % 2 * 4 + word / 2 : word / 16 * 16 + word % 4 * 4 + word / 4 % 4;
        unpack_t(there ? *reinterpret_cast<const uint32_t*>(p.t + (m0 + row) * p.R + 2 * word) : 0u, &t[0][row][at],
                 &t[1][row][at]);
    }
    __syncthreads();
    const int first = static_cast<int>(blockIdx.y) * chunk, last = min(first + chunk, (p.N + 31) / 32);
    const int columns = min(p.N, last * 32);
    const int R = EXACT ? (CH == 0 ? 16 : 32 * CH) : p.R;
    // t: in registers, but for the larger ranks on many tokens (8000 rows of rank 32 303 us, 242 from shared memory)
    constexpr int kSteps = UpFragments<CH>::kSteps, kTiles = MB == 0 ? 1 : MB, kParts = MB == 0 ? 1 : 2;
    constexpr bool kHeld = CH < 1 || MB == 0;
    const uint32_t* const t_lane =
        MB == 0 ? &t[lane >> 3 & 1][lane & 7][lane >> 4 << 2] : &t[0][lane & 15][lane >> 4 << 2];
    auto load_step = [&](uint32_t (&w)[4], int m, int part, int s) { load_t(w, t_lane + (part * kRows + m * 16) * kPitch + 8 * s); };
    uint32_t tf[kHeld ? kTiles : 1][kParts][kSteps][4];
    if constexpr (kHeld) {
#pragma unroll
        for (int m = 0; m < kTiles; ++m)
#pragma unroll
            for (int part = 0; part < kParts; ++part)
#pragma unroll
                for (int s = 0; s < kSteps; ++s) load_step(tf[m][part][s], m, part, s);
    }
    // (rows without an adapter come last: they are copied)
    const int passes = tile.count + (p.out != p.base);
    for (int l = blockIdx.z; l < passes; l += gridDim.z) {
        const int a = l < tile.count ? tile.list[l] : kNone;
        uint32_t mine = 0;  // of this lane's rows g, g + 8, ...
#pragma unroll
        for (int i = 0; i < kHalves; ++i) mine |= static_cast<uint32_t>(tile.id[i * 8 + g] == a) << i;
        const uint32_t any = __reduce_or_sync(0xffffffffu, mine);
        if (any == 0) continue;
        // (rows that are not done here read one that is there)
        const uint16_t* from[kHalves];
#pragma unroll
        for (int i = 0; i < kHalves; ++i) from[i] = p.base + (m0 + (mine >> i & 1u ? i * 8 + g : 0)) * p.N;
        const int64_t to_out = p.out - p.base;
        // column g of block j is feature (g / 2) 8 + 2 j + g % 2: a thread's two columns of each block
        // are then its eight neighbours
        const uint16_t* const b_rows = p.b + static_cast<int64_t>(a < 0 ? 0 : a) * p.N * R;
        const int feature = (g >> 1) * 8 + (g & 1);
        // blocks from f on: FB with every column there, or one that is checked
        auto batch = [&](int f, auto inside) __attribute__((always_inline)) {
            constexpr bool kInside = decltype(inside)::value;
            constexpr int NB = kInside ? FB : 1;
            uint4 c[NB][kHalves];
            const int n0 = f * 32 + 8 * q;
#pragma unroll
            for (int i = 0; i < kHalves; ++i)
#pragma unroll
                for (int u = 0; u < NB; ++u) {
                    const int n = n0 + u * 32;
                    if constexpr (WHOLE) {
                        c[u][i] = *reinterpret_cast<const uint4*>(from[i] + (kInside ? n : min(n, p.N - 8)));
                    } else {
                        uint32_t w[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) w[e] = from[i][kInside ? n + e : min(n + e, p.N - 1)];
                        c[u][i] = make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
                    }
                }
            UpFragments<CH> b[NB][4];
            if (a >= 0) {
                const uint16_t* const bf = b_rows + static_cast<int64_t>(f * 32 + feature) * R;
#pragma unroll
                for (int u = 0; u < NB; ++u)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int d = u * 32 + 2 * j;
                        b[u][j].template load_b<EXACT>(
                            kInside ? bf + d * R : b_rows + static_cast<int64_t>(min(f * 32 + feature + d, p.N - 1)) * R, q, R);
                    }
            }
#pragma unroll
            for (int m = 0; m < kTiles; ++m) {
                if (MB > 1 && !(any >> (2 * m) & 3u)) continue;
#pragma unroll
                for (int u = 0; u < NB; ++u) {
                    float acc[4][4];
                    const uint4& low = c[u][2 * m];
                    const uint4& high = c[u][MB == 0 ? 0 : 2 * m + 1];
                    const uint32_t lo[4] = {low.x, low.y, low.z, low.w}, hi[4] = {high.x, high.y, high.z, high.w};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        acc[j][0] = bf16_low(lo[j]), acc[j][1] = bf16_high(lo[j]);
                        acc[j][2] = MB == 0 ? 0.0f : bf16_low(hi[j]), acc[j][3] = MB == 0 ? 0.0f : bf16_high(hi[j]);
                    }
                    if (a >= 0) {
#pragma unroll
                        for (int part = 0; part < kParts; ++part)
#pragma unroll
                            for (int s = 0; s < kSteps; ++s) {
                                uint32_t w[4];
                                if constexpr (!kHeld) load_step(w, m, part, s);
                                const uint32_t (&x)[4] = kHeld ? tf[kHeld ? m : 0][part][s] : w;
#pragma unroll
                                for (int j = 0; j < 4; ++j)
                                    mma_bf16(acc[j], x[0], x[1], x[2], x[3], b[u][j].w[s][0], b[u][j].w[s][1]);
                            }
                        if constexpr (MB == 0) {
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                acc[j][0] += acc[j][2];
                                acc[j][1] += acc[j][3];
                            }
                        }
                    }
                    const int n = n0 + u * 32;
#pragma unroll
                    for (int h = 0; h < (MB == 0 ? 1 : 2); ++h) {
                        if (!(mine >> (2 * m + h) & 1u)) continue;
                        const uint32_t v[4] = {pack_bf16(acc[0][2 * h], acc[0][2 * h + 1]),
                                               pack_bf16(acc[1][2 * h], acc[1][2 * h + 1]),
                                               pack_bf16(acc[2][2 * h], acc[2][2 * h + 1]),
                                               pack_bf16(acc[3][2 * h], acc[3][2 * h + 1])};
                        uint16_t* const to = const_cast<uint16_t*>(from[2 * m + h]) + to_out + n;
                        const int64_t end = to - p.out + (WHOLE ? 8 : 1), all = static_cast<int64_t>(p.M) * p.N;
                        if constexpr (WHOLE) {
                            if ((kInside || n < columns) && dbg_check(to >= p.out && end <= all, p.status))
                                *reinterpret_cast<uint4*>(to) = make_uint4(v[0], v[1], v[2], v[3]);
                        } else {
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                if ((kInside || n + e < columns) && dbg_check(to >= p.out && end + e <= all, p.status))
                                    to[e] = static_cast<uint16_t>(e & 1 ? v[e / 2] >> 16 : v[e / 2]);
                        }
                    }
                }
            }
        };
        for (int f = first + FB * warp; f < last; f += FB * kWarps) {
            if ((f + FB) * 32 <= columns) {
                batch(f, std::true_type{});
            } else {
#pragma unroll 1
                for (int u = f; u < min(f + FB, last); ++u) batch(u, std::false_type{});
            }
        }
    }
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Whether tiles of 8 tokens, an adapter of the tile to a CTA, read no more than the larger tiles, which take an
// adapter once for more tokens but start fewer CTAs.  Which adapters occur is on the device: as many of a tile are
// counted as it has sequences, and as there are.  (us with small tiles / large ones in both kernels, 12288 x 36864 of
// rank 16: 8 rows of 8 adapters 9.8 / 27, 64 of 48 24 / 129, 1000 of 40 sequences 93 / 69; 12288 x 12288 of rank 64: 200 rows
// of 2 sequences 71 / 24, 512 of one token with 8 adapters 173 / 86.  Where the bytes are few the rule misses: 256 rows of one
// token with 8 adapters of rank 16, 4096 x 4096, 17 / 25, of which it takes the large ones.)
int64_t adapters_of(const AdapterParams& p, int64_t rows) {
    return std::min<int64_t>(p.pool, std::min(rows, ceil_div(std::min<int64_t>(rows, p.M) * p.nseq, p.M)));
}
bool few_down(const AdapterParams& p) {  // (in rows of K)
    const int64_t group = p.R <= 32 ? 4 : 2, adapters = adapters_of(p, kTcRows);
    const int64_t passes = ceil_div(adapters, group);
    return ceil_div(p.M, 8) * adapters_of(p, 8) * p.R + p.M <=
           ceil_div(p.M, kTcRows) * (adapters * p.R + passes * std::min<int64_t>(kTcRows, p.M));
}
bool few_up(const AdapterParams& p) {
    return ceil_div(p.M, 8) * adapters_of(p, 8) <= ceil_div(p.M, 32) * adapters_of(p, 32);
}

// CTAs of a cluster that share K: a power of two up to 16.  Few tokens of an adapter each: while there is K for
// every warp and SMs would be idle (8 at most: 28.7 against 32.4 us with 64 requests).  Tiles of 128 tokens: by the
// turns that 2 CTAs an SM take, each of its K and some start and end (in steps of 64 k).
int cluster_of(const AdapterParams& p, bool few, int sm_count) {
    int s = 1;
    if (few) {
        const int64_t ctas = ceil_div(p.M, 8) * (p.M < 8 ? p.M : 8);
        while (s < 8 && s * ctas < 4 * sm_count && 2 * s * kWarps * 32 <= p.K) s *= 2;
        return s;
    }
    const int64_t tiles = ceil_div(p.M, kTcRows), steps = p.K / 64;
    int64_t least = -1;
    for (int c = 1; c <= 16 && c <= steps; c *= 2) {
        const int64_t cost = ceil_div(tiles * c, 2 * sm_count) * (ceil_div(steps, c) + 8);
        if (least < 0 || cost < least) {
            least = cost;
            s = c;
        }
    }
    return s;
}

template <typename... P, typename... A>
cudaError_t launch_cluster(void (*kernel)(P...), dim3 grid, int block, int smem, cudaStream_t stream, const A&... args) {
    cudaError_t e = cudaSuccess;
    if (smem > 0) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e == cudaSuccess && grid.y > 8) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = attr[1].val.clusterDim.z = 1;
    attr[1].val.clusterDim.y = grid.y;
    cfg.attrs = attr;
    cfg.numAttrs = grid.y > 1 ? 2 : 1;
    e = cudaLaunchKernelEx(&cfg, kernel, P(args)...);
    return e != cudaSuccess ? e : cudaGetLastError();
}

// A tensor map of bf16 rows, in boxes of 64 columns (128-byte swizzle).
int encode_rows(CUtensorMap* map, const void* base, int64_t columns, int64_t rows, int box_rows) {
    const uint64_t dims[5] = {static_cast<uint64_t>(columns), static_cast<uint64_t>(rows), 1, 1, 1};
    const uint64_t stride = static_cast<uint64_t>(columns) * 2, strides[4] = {stride, stride, stride, stride};
    const uint32_t box[5] = {64, static_cast<uint32_t>(box_rows), 1, 1, 1};
    return encode_5d(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, base, dims, strides, box);
}

template <int MT>
cudaError_t launch_down(const AdapterParams& p, bool few, int sm_count, cudaStream_t stream) {
    const int ctas = cluster_of(p, few, sm_count);
    if (few)
        return launch_cluster(adapters_down_few_kernel<MT>, dim3((p.M + 7) / 8, ctas, p.M < 8 ? p.M : 8), kThreads, 0,
                              stream, p);
    alignas(64) CUtensorMap x, a;
    if (encode_rows(&x, p.x, p.K, p.M, kTcRows) != 0 ||
        encode_rows(&a, p.a, p.K, static_cast<int64_t>(p.pool) * p.R, TcLayout<MT>::kRank) != 0)
        return cudaErrorInvalidValue;
    return launch_cluster(adapters_down_kernel<MT>, dim3((p.M + kTcRows - 1) / kTcRows, ctas), kTcThreads,
                          TcLayout<MT>::kSmem, stream, x, a, p);
}

template <int CH, bool EXACT, bool WHOLE>
cudaError_t launch_up(const AdapterParams& p, bool few, int sm_count, cudaStream_t stream) {
    // blocks that a warp has under way
    constexpr int kFew = !WHOLE || CH == 2 ? 1 : 4, kMany = !WHOLE || CH == 2 ? 1 : 2;
    const int rows = few ? 8 : 32, z = few ? (p.M < 8 ? p.M : 8) : 1, unit = kWarps * (few ? kFew : kMany);
    const int64_t tiles = ceil_div(p.M, rows) * z, units = ceil_div(ceil_div(p.N, 32), unit);
    // Few tokens: the CTAs that are resident, at most, as each starts with four loads in a row.  Many: several
    // turns of them, but four units each at least, unless that leaves SMs idle.
    const int64_t sms = sm_count;
    int64_t y = few ? 2 * sms / tiles
                    : std::max(std::min(ceil_div(16 * sms, tiles), units / 4), std::min(units, ceil_div(2 * sms, tiles)));
    if (y < 1) y = 1;
    const int64_t chunk = ceil_div(units, y);
    const dim3 grid(static_cast<unsigned>(ceil_div(p.M, rows)), static_cast<unsigned>(ceil_div(units, chunk)), z);
    auto kernel = few ? adapters_up_kernel<CH, 0, kFew, EXACT, WHOLE> : adapters_up_kernel<CH, 2, kMany, EXACT, WHOLE>;
    return launch_overlapped(kernel, grid, kThreads, 0, stream, p, static_cast<int>(chunk * unit));
}

template <int CH>
cudaError_t launch_up(const AdapterParams& p, bool few, int sm_count, cudaStream_t stream) {
    // (other ranks, and rows that are not whole 16-byte units, take checks on every load)
    if (p.N % 8 != 0) return launch_up<CH, false, false>(p, few, sm_count, stream);
    return p.R == (CH == 0 ? 16 : 32 * CH) ? launch_up<CH, true, true>(p, few, sm_count, stream)
                                           : launch_up<CH, false, true>(p, few, sm_count, stream);
}

}  // namespace

int64_t adapters_workspace_bytes(int64_t M, int64_t R) { return M * R * static_cast<int64_t>(sizeof(uint16_t)); }

cudaError_t launch_adapters(const AdapterParams& p, int sm_count, cudaStream_t stream) {
    const bool few = few_down(p), few_rows = few_up(p);
    const cudaError_t e = p.R <= 16   ? launch_down<1>(p, few, sm_count, stream)
                          : p.R <= 32 ? launch_down<2>(p, few, sm_count, stream)
                          : p.R <= 48 ? launch_down<3>(p, few, sm_count, stream)
                                      : launch_down<4>(p, few, sm_count, stream);
    if (e != cudaSuccess) return e;
    return p.R <= 16   ? launch_up<0>(p, few_rows, sm_count, stream)
           : p.R <= 32 ? launch_up<1>(p, few_rows, sm_count, stream)
                       : launch_up<2>(p, few_rows, sm_count, stream);
}

}  // namespace w4a16
