// Low-rank adapters of many sequences beside a shared projection:
//   out = base + t B_a^T,  t = scale_a (x A_a^T),  a the adapter of the row's sequence.
//
// Two kernels.  The first reads x and gives t: warp-level MMAs with the adapter's rows as the 16-row
// operand and eight tokens as columns, K split over warps and over the CTAs of a cluster, whose fp32
// sums are added up in order through distributed shared memory; t is rounded to bf16 (2^-8 of each, of an
// update beside a sum that a bf16 store rounds as much) into the workspace.  The second streams base and
// out, with tokens as rows and 32 features as columns of its MMAs, arranged so that a thread has eight
// neighbours: the accumulators begin as base and are stored as out, 16 bytes a thread.
// Rows of a tile that share an adapter are done together; x is zero in the others' columns.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
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
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// The rows of a tile: each one's adapter, and the list of those that occur.
template <int ROWS>
struct Tile {
    int id[ROWS];
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
}

__device__ __forceinline__ uint4 load16(const uint16_t* p) { return __ldg(reinterpret_cast<const uint4*>(p)); }

__device__ __forceinline__ void copy_async16(uint32_t to, const void* from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void store_shared_zero16(uint32_t at) {
    asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(at), "r"(0) : "memory");
}
__device__ __forceinline__ void copy_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_async_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ uint4 load_shared16(uint32_t at) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}

// 32 k of 16 MT rows of an adapter with eight tokens: a lane has 16 bytes of its rows g and g + 8 of
// each 16 and of its token g, of which each MMA takes half; the order of k is the same on both sides.
template <int MT>
__device__ __forceinline__ void mma_step(float (&acc)[MT][4], const uint4 (&a)[MT][2], const uint4& x) {
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        mma_bf16(acc[i], a[i][0].x, a[i][1].x, a[i][0].y, a[i][1].y, x.x, x.y);
        mma_bf16(acc[i], a[i][0].z, a[i][1].z, a[i][0].w, a[i][1].w, x.z, x.w);
    }
}

// A slice of K for a split: steps of 32.
struct Slice {
    int from, to;
    __device__ __forceinline__ explicit Slice(int K) {
        const int64_t steps = K / 32;
        from = static_cast<int>(steps * blockIdx.y / gridDim.y);
        to = static_cast<int>(steps * (blockIdx.y + 1) / gridDim.y);
    }
};

__device__ __forceinline__ float load_cluster(uint32_t at) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
    return v;
}

// The warps' sums [WARPS][ROWS][16 MT + 4] added up, in order, then those of the cluster's CTAs (gridDim.y
// of them), for the tokens with the adapter.  All threads; the sums may be overwritten after it.
template <int WARPS, int ROWS, int MT>
__device__ __forceinline__ void store_t(float* sums, const Tile<ROWS>& tile, const AdapterParams& p, int64_t m0, int a) {
    constexpr int kPitch = 16 * MT + 4, kAll = ROWS * 16 * MT;
    const int ctas = static_cast<int>(gridDim.y);
    __syncthreads();
    for (int i = threadIdx.x; i < kAll; i += WARPS * 32) {
        float* const at = sums + i / (16 * MT) * kPitch + i % (16 * MT);
        float sum = at[0];
#pragma unroll
        for (int w = 1; w < WARPS; ++w) sum += at[w * ROWS * kPitch];
        at[0] = sum;
    }
    if (ctas > 1) cluster_sync(); else __syncthreads();
    // each CTA adds up a part of the tokens
    const float scale = p.scale[a];
    uint16_t* const out = p.t + m0 * p.R;
    for (int i = blockIdx.y * (WARPS * 32) + threadIdx.x; i < kAll; i += ctas * WARPS * 32) {
        const int token = i / (16 * MT), r = i % (16 * MT);
        if (tile.id[token] != a || r >= p.R) continue;
        const float* const at = sums + token * kPitch + r;
        float sum = 0.0f;
        if (ctas > 1) {
            const uint32_t local = smem_u32(at);
            for (int c = 0; c < ctas; ++c) sum += load_cluster(mapa_shared(local, c));
        } else {
            sum = at[0];
        }
        out[static_cast<int64_t>(token) * p.R + r] = __bfloat16_as_ushort(__float2bfloat16_rn(sum * scale));
    }
    if (ctas > 1) cluster_sync(); else __syncthreads();
}

// t of 64 tokens (blockIdx.x) over a slice of K (blockIdx.y), for each of the tile's adapters; K between
// the warps.  What a lane needs of x and of the adapter it copies itself, kStages steps ahead, into its
// own places of shared memory: no barrier, and 96 KB an SM under way.
constexpr int kDownWarps = 4;
template <int MT>
constexpr int kStages = MT == 4 ? 3 : 4;

template <int MT>
__global__ void __launch_bounds__(kDownWarps * 32, 2) adapters_down_kernel(const AdapterParams p) {
    constexpr int kRows = 64, NB = kRows / 8, ST = kStages<MT>, kPieces = NB + 2 * MT;
    __shared__ Tile<kRows> tile;
    extern __shared__ __align__(16) uint8_t ring[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, q = lane & 3;
    const int64_t m0 = static_cast<int64_t>(blockIdx.x) * kRows;
    grid_launch_dependents();
    grid_wait();
    find_adapters<kRows>(tile, p, m0, blockIdx.y == 0);
    if (p.seq_start != nullptr && blockIdx.y == 0) check_starts(p.seq_start, p.nseq, p.M, p.status);
    const Slice k(p.K);
    const uint32_t mine_at = smem_u32(ring) + (warp * ST * kPieces * 32 + lane) * 16;
    for (int l = 0; l < tile.count; ++l) {
        const int a = tile.list[l];
        uint32_t mine = 0;  // blocks in which this lane's token has the adapter
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) mine |= static_cast<uint32_t>(tile.id[nb * 8 + g] == a) << nb;
        const uint32_t any = __reduce_or_sync(0xffffffffu, mine);
        // the places of rows that are not copied hold zeros
        for (int stage = 0; stage < ST; ++stage)
#pragma unroll
            for (int i = 0; i < kPieces; ++i)
                if (i < NB ? !(mine >> i & 1u) : (i - NB) * 8 + g >= p.R)
                    store_shared_zero16(mine_at + (stage * kPieces + i) * 512);
        const uint8_t* const x = reinterpret_cast<const uint8_t*>(p.x + (m0 + g) * p.K + 8 * q);
        const uint8_t* const w =
            reinterpret_cast<const uint8_t*>(p.a + (static_cast<int64_t>(a) * p.R + g) * p.K + 8 * q);
        const uint32_t rows8 = 16u * static_cast<uint32_t>(p.K);  // bytes of eight rows (K < 2^25)
        auto fetch = [&](int stage, int s) {
            if (s < k.to) {
                const uint32_t at = mine_at + stage * (kPieces * 512);
                const uint8_t* const xs = x + static_cast<int64_t>(s) * 64;
                const uint8_t* const ws = w + static_cast<int64_t>(s) * 64;
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
                    if (mine >> nb & 1u) copy_async16(at + nb * 512, xs + rows8 * nb);
#pragma unroll
                for (int i = 0; i < 2 * MT; ++i)
                    if (i * 8 + g < p.R) copy_async16(at + (NB + i) * 512, ws + rows8 * i);
            }
            copy_async_commit();
        };
        float acc[NB][MT][4] = {};
        int s = k.from + warp;
#pragma unroll
        for (int i = 0; i < ST - 1; ++i) fetch(i, s + i * kDownWarps);
        for (int stage = 0; s < k.to; s += kDownWarps) {
            copy_async_wait<ST - 2>();
            const uint32_t at = mine_at + stage * (kPieces * 512);
            uint4 av[MT][2];
#pragma unroll
            for (int i = 0; i < 2 * MT; ++i) av[i / 2][i % 2] = load_shared16(at + (NB + i) * 512);
            // (its place was read a turn ago)
            fetch(stage == 0 ? ST - 1 : stage - 1, s + (ST - 1) * kDownWarps);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
                if (any >> nb & 1u) mma_step<MT>(acc[nb], av, load_shared16(at + nb * 512));
            stage = stage == ST - 1 ? 0 : stage + 1;
        }
        copy_async_wait<0>();
        __syncthreads();
        float* const sums = reinterpret_cast<float*>(ring);
        constexpr int kPitch = 16 * MT + 4;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    sums[(warp * kRows + nb * 8 + 2 * q + (e & 1)) * kPitch + i * 16 + g + (e & 2) * 4] = acc[nb][i][e];
        store_t<kDownWarps, kRows, MT>(sums, tile, p, m0, a);
    }
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
    const Slice k(p.K);
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
        store_t<kWarps, kRows, MT>(sums, tile, p, m0, a);
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
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int s = 0; s < kSteps; ++s) w[s][0] = w[s][1] = 0;
    }
    __device__ __forceinline__ void load_t(const uint32_t* row, int q) {
        if constexpr (CH == 0) {
            const uint2 v = *reinterpret_cast<const uint2*>(row + 2 * q);
            w[0][0] = v.x, w[0][1] = v.y;
        } else {
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const uint4 v = *reinterpret_cast<const uint4*>(row + 16 * c + 4 * q);
                w[2 * c][0] = v.x, w[2 * c][1] = v.y, w[2 * c + 1][0] = v.z, w[2 * c + 1][1] = v.w;
            }
        }
    }
};

// out of a tile of tokens (blockIdx.x) and `chunk` blocks of 32 features (blockIdx.y), for the tile's
// adapters blockIdx.z, + gridDim.z, ...; a warp has FB blocks under way.  MB: 16s of tokens; 0: eight, in
// the upper half of one.  EXACT: the rank is 16 or 32 CH.  WHOLE: rows of 16-byte units.
template <int CH, int MB, int FB, bool EXACT, bool WHOLE>
__global__ void __launch_bounds__(kThreads, !WHOLE || CH == 2 ? 1 : CH == 0 && MB == 0 ? 3 : 2)
    adapters_up_kernel(const AdapterParams p, const int chunk) {
    constexpr int kRows = MB == 0 ? 8 : 16 * MB, kHalves = MB == 0 ? 1 : 2 * MB;  // rows of a lane
    constexpr int kWords = CH == 0 ? 8 : 16 * CH, kPitch = kWords + 4;            // (pairs of bf16)
    __shared__ Tile<kRows> tile;
    __shared__ __align__(16) uint32_t t[kRows][kPitch];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, q = lane & 3;
    const int64_t m0 = static_cast<int64_t>(blockIdx.x) * kRows;
    grid_launch_dependents();
    grid_wait();
    find_adapters<kRows>(tile, p, m0, false);
    for (int i = threadIdx.x; i < kRows * kWords; i += kThreads) {
        const int row = i / kWords, word = i % kWords;
        t[row][word] = tile.id[row] >= 0 && 2 * word < p.R
                           ? *reinterpret_cast<const uint32_t*>(p.t + (m0 + row) * p.R + 2 * word) : 0u;
    }
    __syncthreads();
    const int first = static_cast<int>(blockIdx.y) * chunk, last = min(first + chunk, (p.N + 31) / 32);
    const int columns = min(p.N, last * 32);
    const int R = EXACT ? (CH == 0 ? 16 : 32 * CH) : p.R;
    UpFragments<CH> tf[kHalves];  // of the lane's rows
#pragma unroll
    for (int i = 0; i < kHalves; ++i) tf[i].load_t(t[i * 8 + g], q);
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
        // `blocks` blocks from f on: FB with every column there, or one that is checked
        auto batch = [&](int f, auto blocks) __attribute__((always_inline)) {
            constexpr int NB = decltype(blocks)::value;
            constexpr bool kInside = NB == FB && FB > 1;
            uint4 c[NB][kHalves];
            const int n0 = f * 32 + 8 * q;
#pragma unroll
            for (int i = 0; i < kHalves; ++i)
#pragma unroll
                for (int u = 0; u < NB; ++u) {
                    const int n = n0 + u * 32;
                    if constexpr (WHOLE) {
                        c[u][i] = __ldcs(reinterpret_cast<const uint4*>(from[i] + (kInside ? n : min(n, p.N - 8))));
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
            for (int m = 0; m < (MB == 0 ? 1 : MB); ++m) {
                if (MB > 1 && !(any >> (2 * m) & 3u)) continue;
                UpFragments<CH> tb;
                if (MB == 0) tb.zero(); else tb = tf[MB == 0 ? 0 : 2 * m + 1];
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
                        for (int s = 0; s < UpFragments<CH>::kSteps; ++s)
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                mma_bf16(acc[j], tf[2 * m].w[s][0], tb.w[s][0], tf[2 * m].w[s][1], tb.w[s][1],
                                         b[u][j].w[s][0], b[u][j].w[s][1]);
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
                        if constexpr (WHOLE) {
                            if (kInside || n < columns) *reinterpret_cast<uint4*>(to) = make_uint4(v[0], v[1], v[2], v[3]);
                        } else {
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                if (kInside || n + e < columns)
                                    to[e] = static_cast<uint16_t>(e & 1 ? v[e / 2] >> 16 : v[e / 2]);
                        }
                    }
                }
            }
        };
        for (int f = first + FB * warp; f < last; f += FB * kWarps) {
            if (FB > 1 && (f + FB) * 32 <= columns) {
                batch(f, std::integral_constant<int, FB>{});
            } else {
#pragma unroll 1
                for (int u = f; u < min(f + FB, last); ++u) batch(u, std::integral_constant<int, 1>{});
            }
        }
    }
}

// Short sequences: tiles of 8 tokens, an adapter of the tile to a CTA.
bool short_sequences(int64_t M, int64_t nseq) { return M < 16 * nseq; }

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// CTAs of a cluster that share K: a power of two up to 16 (8 where adapters are few tokens each: 28.7 against 32.4 us
// with 64 requests), while that leaves each of them something and SMs
// would be idle otherwise.
int cluster_of(const AdapterParams& p, bool few, int sm_count) {
    const int64_t ctas = few ? ceil_div(p.M, 8) * (p.M < 8 ? p.M : 8) : ceil_div(p.M, 64);
    const int64_t least = few ? kWarps * 32 : kDownWarps * 128;  // of K
    int s = 1;
    while (s < (few ? 8 : 16) && s * ctas < 4 * sm_count && 2 * s * least <= p.K) s *= 2;
    return s;
}

template <typename Kernel>
cudaError_t launch_cluster(Kernel kernel, dim3 grid, int block, int smem, cudaStream_t stream, const AdapterParams& p) {
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
    e = cudaLaunchKernelEx(&cfg, kernel, p);
    return e != cudaSuccess ? e : cudaGetLastError();
}

template <int MT>
cudaError_t launch_down(const AdapterParams& p, bool few, int sm_count, cudaStream_t stream) {
    const int ctas = cluster_of(p, few, sm_count);
    if (few)
        return launch_cluster(adapters_down_few_kernel<MT>, dim3((p.M + 7) / 8, ctas, p.M < 8 ? p.M : 8), kThreads, 0,
                              stream, p);
    constexpr int kRing = kDownWarps * kStages<MT> * (8 + 2 * MT) * 512;
    constexpr int kSums = kDownWarps * 64 * (16 * MT + 4) * 4;
    return launch_cluster(adapters_down_kernel<MT>, dim3((p.M + 63) / 64, ctas), kDownWarps * 32,
                          kRing > kSums ? kRing : kSums, stream, p);
}

template <int CH, bool EXACT, bool WHOLE>
cudaError_t launch_up(const AdapterParams& p, bool few, int sm_count, cudaStream_t stream) {
    constexpr int FB = CH == 2 ? 2 : 4;  // few rows
    const int rows = few ? 8 : 32, z = few ? (p.M < 8 ? p.M : 8) : 1;
    const int64_t tiles = ceil_div(p.M, rows) * z, blocks = ceil_div(p.N, 32);
    // as many features to a CTA as leave every SM several CTAs
    int64_t y = ceil_div((few ? 4 : 16) * static_cast<int64_t>(sm_count), tiles);
    const int64_t unit = kWarps * (!WHOLE ? 1 : few ? FB : 2);  // blocks that a CTA has under way
    const int64_t chunk = ceil_div(ceil_div(blocks, y), unit) * unit;
    y = ceil_div(blocks, chunk);
    const dim3 grid(static_cast<unsigned>(ceil_div(p.M, rows)), static_cast<unsigned>(y), z);
    auto kernel = few ? adapters_up_kernel<CH, 0, WHOLE ? FB : 1, EXACT, WHOLE>
                      : adapters_up_kernel<CH, 2, WHOLE ? 2 : 1, EXACT, WHOLE>;
    return launch_overlapped(kernel, grid, kThreads, 0, stream, p, static_cast<int>(chunk));
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
    const bool few = short_sequences(p.M, p.nseq);
    const cudaError_t e = p.R <= 16   ? launch_down<1>(p, few, sm_count, stream)
                          : p.R <= 32 ? launch_down<2>(p, few, sm_count, stream)
                                      : launch_down<4>(p, few, sm_count, stream);
    if (e != cudaSuccess) return e;
    return p.R <= 16   ? launch_up<0>(p, few, sm_count, stream)
           : p.R <= 32 ? launch_up<1>(p, few, sm_count, stream)
                       : launch_up<2>(p, few, sm_count, stream);
}

}  // namespace w4a16
