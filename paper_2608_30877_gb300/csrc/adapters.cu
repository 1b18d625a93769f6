// Low-rank adapters of many sequences beside a shared projection:
//   out = base + t B_a^T,  t = scale_a (x A_a^T),  a the adapter of the row's sequence.
//
// Two kernels.  The first reads x and gives t: warp-level MMAs with the adapter's rows as the 16-row
// operand and eight tokens as columns, K split over warps and CTAs, each CTA's sums of fp32 to
// the workspace.  The second adds these up, in order, rounds t to bf16 (2^-9 of a product of which
// only the update is made, beside a bf16 store of the sum) and streams base and out, with 16
// tokens as rows and 32 features as columns, arranged so that a thread has eight neighbours: the
// accumulators begin as base and are stored as out, 16 bytes a thread.
// Rows of a tile that share an adapter are done together; t is zero in the others' columns.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <cstdint>

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

// All threads; ends behind a barrier.
template <int ROWS>
__device__ __forceinline__ void find_adapters(Tile<ROWS>& tile, const AdapterParams& p, int64_t m0, bool check) {
    if (threadIdx.x < ROWS) {
        const int64_t m = m0 + threadIdx.x;
        int id = kOutside;
        if (m < p.M) {
            int begin = 0, end = p.M, s = static_cast<int>(m);
            id = kNone;
            if (p.seq_start != nullptr) s = sequence_of(p.seq_start, p.nseq, s, &begin, &end);
            if (s >= 0 && begin >= 0 && end <= p.M) {
                id = p.ids[s];
                if (id < -1 || id >= p.pool) {
                    if (check) record_status(p.status, 1 /* W4A16_ERR_INVALID_ARG */);
                    id = kNone;
                }
            }
        }
        tile.id[threadIdx.x] = id;
    }
    if (threadIdx.x == 0) tile.count = 0;
    __syncthreads();
    if (threadIdx.x < 32) {  // the first row of each adapter, in order
        int n = 0;
#pragma unroll
        for (int i0 = 0; i0 < ROWS; i0 += 32) {
            const int i = i0 + static_cast<int>(threadIdx.x);
            bool first = i < ROWS && tile.id[i < ROWS ? i : 0] >= 0;
            if (first)
                for (int j = 0; j < i; ++j) first = first && tile.id[j] != tile.id[i];
            const uint32_t mask = __ballot_sync(0xffffffffu, first);
            if (first) tile.list[n + __popc(mask & ((1u << threadIdx.x) - 1u))] = tile.id[i];
            n += __popc(mask);
        }
        if (threadIdx.x == 0) tile.count = n;
    }
    __syncthreads();
}

__device__ __forceinline__ uint4 load16(const uint16_t* p) { return __ldg(reinterpret_cast<const uint4*>(p)); }

// t of 8 NB tokens (blockIdx.x) over a slice of K (blockIdx.y), for the tile's adapters blockIdx.z,
// + gridDim.z, ...  The warps: RG times 16 MT rows of the adapter, and K between the others.
template <int MT, int RG, int NB>
__global__ void __launch_bounds__(kThreads, 2) adapters_down_kernel(const AdapterParams p) {
    constexpr int kRows = 8 * NB, KG = kWarps / RG, kR = 16 * MT * RG;
    constexpr int U = NB == 1 ? 4 : 1;  // steps of 32 k under way
    __shared__ Tile<kRows> tile;
    extern __shared__ __align__(16) float sums[];  // [KG / 2][kRows][kR + 4]
    constexpr int kPitch = kR + 4;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, q = lane & 3;
    const int rg = warp % RG, kg = warp / RG;
    const int64_t m0 = static_cast<int64_t>(blockIdx.x) * kRows;
    grid_launch_dependents();
    grid_wait();
    find_adapters<kRows>(tile, p, m0, blockIdx.y == 0 && blockIdx.z == 0);
    if (p.seq_start != nullptr && blockIdx.y == 0 && blockIdx.z == 0) check_starts(p.seq_start, p.nseq, p.M, p.status);
    const int steps = p.K / 32;
    const int from = static_cast<int>(static_cast<int64_t>(steps) * blockIdx.y / gridDim.y);
    const int to = static_cast<int>(static_cast<int64_t>(steps) * (blockIdx.y + 1) / gridDim.y);
    for (int l = blockIdx.z; l < tile.count; l += gridDim.z) {
        const int a = tile.list[l];
        const uint16_t* const w = p.a + static_cast<int64_t>(a) * p.R * p.K + 8 * q;
        uint32_t mine = 0;  // blocks in which this lane's token has the adapter
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) mine |= static_cast<uint32_t>(tile.id[nb * 8 + g] == a) << nb;
        const uint32_t any = __reduce_or_sync(0xffffffffu, mine);
        float acc[MT][NB][4];
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][nb][e] = 0.0f;
        for (int s = from + kg; s < to; s += KG * U) {
            uint4 xv[U][NB], av[U][MT][2];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int k = (s + u * KG) * 32;
                const bool in = s + u * KG < to;
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    xv[u][nb] = make_uint4(0, 0, 0, 0);
                    if (in && (mine >> nb & 1u)) xv[u][nb] = load16(p.x + (m0 + nb * 8 + g) * p.K + k + 8 * q);
                }
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int r = (rg * MT + i) * 16 + h * 8 + g;
                        av[u][i][h] = make_uint4(0, 0, 0, 0);
                        if (in && r < p.R) av[u][i][h] = load16(w + static_cast<int64_t>(r) * p.K + k);
                    }
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    if (NB > 1 && !(any >> nb & 1u)) continue;
#pragma unroll
                    for (int i = 0; i < MT; ++i) {
                        mma_bf16(acc[i][nb], av[u][i][0].x, av[u][i][1].x, av[u][i][0].y, av[u][i][1].y, xv[u][nb].x,
                                 xv[u][nb].y);
                        mma_bf16(acc[i][nb], av[u][i][0].z, av[u][i][1].z, av[u][i][0].w, av[u][i][1].w, xv[u][nb].z,
                                 xv[u][nb].w);
                    }
                }
        }
        // the upper half of the warps that split K hands its sums to the lower one, and so on
#pragma unroll
        for (int half = KG / 2; half > 0; half /= 2) {
            if (kg >= half && kg < 2 * half) {
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            sums[((kg - half) * kRows + nb * 8 + 2 * q + (e & 1)) * kPitch + (rg * MT + i) * 16 + g + (e & 2) * 4] =
                                acc[i][nb][e];
            }
            __syncthreads();
            if (kg < half) {
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            acc[i][nb][e] +=
                                sums[(kg * kRows + nb * 8 + 2 * q + (e & 1)) * kPitch + (rg * MT + i) * 16 + g + (e & 2) * 4];
            }
            __syncthreads();
        }
        if (kg == 0) {
            const float scale = p.scale[a];
            float* const out = p.parts + (static_cast<int64_t>(blockIdx.y) * p.M + m0) * p.R;
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int token = nb * 8 + 2 * q + (e & 1), r = (rg * MT + i) * 16 + g + (e & 2) * 4;
                        if (tile.id[token] == a && r < p.R) out[static_cast<int64_t>(token) * p.R + r] = acc[i][nb][e] * scale;
                    }
        }
    }
}

// Eight neighbouring columns of a row, from column n on; WHOLE: rows of 16-byte units.
template <bool WHOLE>
__device__ __forceinline__ uint4 load_columns(const uint16_t* row, int n, int N) {
    if constexpr (WHOLE) {
        return n < N ? __ldcs(reinterpret_cast<const uint4*>(row + n)) : make_uint4(0, 0, 0, 0);
    } else {
        uint32_t w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = n + e < N ? row[n + e] : 0u;
        return make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
    }
}
template <bool WHOLE>
__device__ __forceinline__ void store_columns(uint16_t* row, int n, int N, uint4 v) {
    if constexpr (WHOLE) {
        if (n < N) *reinterpret_cast<uint4*>(row + n) = v;
    } else {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (n + e < N) row[n + e] = static_cast<uint16_t>(e & 1 ? w[e / 2] >> 16 : w[e / 2]);
    }
}

// out of 16 MB tokens (blockIdx.x) and `blocks` blocks of 32 features (blockIdx.y), for the tile's
// adapters blockIdx.z, + gridDim.z, ...; KS: steps of 16 of the rank.
template <int KS, int MB, bool WHOLE>
__global__ void __launch_bounds__(kThreads) adapters_up_kernel(const AdapterParams p, const int splits, const int blocks) {
    constexpr int kRows = 16 * MB, kPitch = KS * 8 + 4;  // (in pairs of bf16)
    __shared__ Tile<kRows> tile;
    __shared__ __align__(16) uint32_t t[kRows][kPitch];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, q = lane & 3;
    const int64_t m0 = static_cast<int64_t>(blockIdx.x) * kRows;
    grid_launch_dependents();
    grid_wait();
    find_adapters<kRows>(tile, p, m0, false);
    for (int i = threadIdx.x; i < kRows * KS * 8; i += kThreads) {
        const int row = i / (KS * 8), r = 2 * (i - row * (KS * 8));
        float2 sum = make_float2(0.0f, 0.0f);
        if (tile.id[row] >= 0 && r < p.R) {
            const float* part = p.parts + (m0 + row) * p.R + r;
            for (int s = 0; s < splits; ++s) {
                const float2 v = *reinterpret_cast<const float2*>(part + static_cast<int64_t>(s) * p.M * p.R);
                sum.x += v.x;
                sum.y += v.y;
            }
        }
        t[row][r / 2] = pack_bf16(sum.x, sum.y);
    }
    __syncthreads();
    const int first = static_cast<int>(blockIdx.y) * blocks, last = min(first + blocks, (p.N + 31) / 32);
    // (rows without an adapter come last: they are copied)
    const int passes = tile.count + (p.out != p.base);
    for (int l = blockIdx.z; l < passes; l += gridDim.z) {
        const int a = l < tile.count ? tile.list[l] : kNone;
        uint32_t mine = 0;  // of this lane's rows g and g + 8 of each 16
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
            mine |= static_cast<uint32_t>(tile.id[mb * 16 + g] == a) << (2 * mb);
            mine |= static_cast<uint32_t>(tile.id[mb * 16 + g + 8] == a) << (2 * mb + 1);
        }
        const uint32_t any = __reduce_or_sync(0xffffffffu, mine);
        if (any == 0) continue;
        for (int f = first + warp; f < last; f += kWarps) {
            const int n = f * 32 + 8 * q;
            uint4 c[MB][2];
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    c[mb][h] = make_uint4(0, 0, 0, 0);
                    if (mine >> (2 * mb + h) & 1u)
                        c[mb][h] = load_columns<WHOLE>(p.base + (m0 + mb * 16 + h * 8 + g) * p.N, n, p.N);
                }
            uint2 b[KS][4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                // column g of block j is feature (g / 2) 8 + 2 j + g % 2: a thread's two columns of each
                // block are then its eight neighbours
                const int feature = f * 32 + (g >> 1) * 8 + 2 * j + (g & 1);
                const uint16_t* const w = p.b + (static_cast<int64_t>(a < 0 ? 0 : a) * p.N + feature) * p.R + 4 * q;
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    b[k][j] = make_uint2(0, 0);
                    if (a >= 0 && feature < p.N && 16 * k + 4 * q < p.R)
                        b[k][j] = __ldg(reinterpret_cast<const uint2*>(w + 16 * k));
                }
            }
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) {
                if (!(any >> (2 * mb) & 3u)) continue;
                float acc[4][4];
                const uint32_t lo[4] = {c[mb][0].x, c[mb][0].y, c[mb][0].z, c[mb][0].w};
                const uint32_t hi[4] = {c[mb][1].x, c[mb][1].y, c[mb][1].z, c[mb][1].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    acc[j][0] = bf16_low(lo[j]), acc[j][1] = bf16_high(lo[j]);
                    acc[j][2] = bf16_low(hi[j]), acc[j][3] = bf16_high(hi[j]);
                }
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    const uint2 ta = *reinterpret_cast<const uint2*>(&t[mb * 16 + g][k * 8 + 2 * q]);
                    const uint2 tb = *reinterpret_cast<const uint2*>(&t[mb * 16 + g + 8][k * 8 + 2 * q]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) mma_bf16(acc[j], ta.x, tb.x, ta.y, tb.y, b[k][j].x, b[k][j].y);
                }
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    if (mine >> (2 * mb + h) & 1u)
                        store_columns<WHOLE>(p.out + (m0 + mb * 16 + h * 8 + g) * p.N, n, p.N,
                                             make_uint4(pack_bf16(acc[0][2 * h], acc[0][2 * h + 1]),
                                                        pack_bf16(acc[1][2 * h], acc[1][2 * h + 1]),
                                                        pack_bf16(acc[2][2 * h], acc[2][2 * h + 1]),
                                                        pack_bf16(acc[3][2 * h], acc[3][2 * h + 1])));
            }
        }
    }
}

// Short sequences: tiles of 8 tokens, an adapter of the tile to a CTA.
bool short_sequences(int64_t M, int64_t nseq) { return M < 16 * nseq; }

int splits_of(int64_t M, int64_t nseq, int64_t K, int sm_count) {
    const bool few = short_sequences(M, nseq);
    const int64_t ctas = few ? (M + 7) / 8 * (M < 8 ? M : 8) : (M + 63) / 64;
    int64_t s = ((few ? 4 : 16) * static_cast<int64_t>(sm_count) + ctas - 1) / ctas;
    const int64_t most = K / 256 < 32 ? K / 256 : 32;
    if (s > most) s = most;
    return s < 1 ? 1 : static_cast<int>(s);
}

template <int MT, int RG>
cudaError_t launch_down(const AdapterParams& p, bool few, int splits, cudaStream_t stream) {
    constexpr int KG = kWarps / RG;
    const int rows = few ? 8 : 64;
    const int smem = KG / 2 * rows * (16 * MT * RG + 4) * static_cast<int>(sizeof(float));
    const dim3 grid((p.M + rows - 1) / rows, splits, few ? (p.M < 8 ? p.M : 8) : 1);
    auto kernel = few ? adapters_down_kernel<MT, RG, 1> : adapters_down_kernel<MT, RG, 8>;
    if (smem > 48 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != cudaSuccess) return e;
    }
    return launch_overlapped(kernel, grid, kThreads, smem, stream, p);
}

template <int KS>
cudaError_t launch_up(const AdapterParams& p, bool few, int splits, cudaStream_t stream) {
    const bool whole = p.N % 8 == 0;
    const int rows = few ? 16 : 64;
    const int blocks = 32;  // 1024 features
    const dim3 grid((p.M + rows - 1) / rows, ((p.N + 31) / 32 + blocks - 1) / blocks, few ? (p.M < 16 ? p.M : 16) : 1);
    auto kernel = few ? (whole ? adapters_up_kernel<KS, 1, true> : adapters_up_kernel<KS, 1, false>)
                      : (whole ? adapters_up_kernel<KS, 4, true> : adapters_up_kernel<KS, 4, false>);
    return launch_overlapped(kernel, grid, kThreads, 0, stream, p, splits, blocks);
}

}  // namespace

int64_t adapters_workspace_bytes(int64_t M, int64_t nseq, int64_t K, int64_t R, int sm_count) {
    return splits_of(M, nseq, K, sm_count) * M * R * static_cast<int64_t>(sizeof(float));
}

cudaError_t launch_adapters(const AdapterParams& p, int sm_count, cudaStream_t stream) {
    const bool few = short_sequences(p.M, p.nseq);
    const int splits = splits_of(p.M, p.nseq, p.K, sm_count);
    const cudaError_t e = p.R <= 16   ? launch_down<1, 1>(p, few, splits, stream)
                          : p.R <= 32 ? launch_down<2, 1>(p, few, splits, stream)
                                      : launch_down<2, 2>(p, few, splits, stream);
    if (e != cudaSuccess) return e;
    return p.R <= 16   ? launch_up<1>(p, few, splits, stream)
           : p.R <= 32 ? launch_up<2>(p, few, splits, stream)
                       : launch_up<4>(p, few, splits, stream);
}

}  // namespace w4a16
