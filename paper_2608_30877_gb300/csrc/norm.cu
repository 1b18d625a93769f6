// The residual stream between two blocks of the decoder, in one pass over its rows:
//   h = scale r + gate post(b),   out = pre(h)
// with post and pre RMS norms v / sqrt(mean v^2 + eps) or layer norms (v - mean) / sqrt(var + eps),
// each times (offset + weight) plus a bias.
//
// A row's values stay in registers between the reductions and the store, so that each is read
// once and written once, and a variance is the mean of squares about a mean that is known (no
// difference of large sums).  Up to 1024 columns a warp has a row, else a CTA; a thread has up to
// kMost pieces of eight columns.  The norm is of h as computed, not as rounded for the store.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <cstdint>

#include "kv.h"
#include "layer.h"
#include "ptx.cuh"

namespace w4a16 {

namespace {

constexpr int kMaxWarps = 16;

__device__ __forceinline__ float bf16_low(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float bf16_high(uint32_t v) { return __uint_as_float(v & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&p);
}

// Rows are read once: they leave L1 to the weights, which every row reads.
__device__ __forceinline__ uint4 load_row16(const void* p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "l"(p)
                 : "memory");
    return v;
}

// A row lies in 16-byte units of the memory it is in: a thread has the units t, t + group, ... of
// eight columns each, of which the first and the last may lie partly in other rows where D is no
// multiple of 8 (ODD; all arrays of rows have the same units then, whatever their type).
template <bool ODD>
struct Row {
    int t, group, D, shift;  // shift: columns of the first unit that are the row before's

    __device__ __forceinline__ int first(int v) const { return (v * group + t) * 8 - (ODD ? shift : 0); }
    __device__ __forceinline__ bool whole(int c) const { return ODD ? c >= 0 && c + 8 <= D : c < D; }
    // Whether the row has column e of the unit at column c.
    __device__ __forceinline__ bool has(int c, int e) const {
        return ODD ? static_cast<unsigned>(c + e) < static_cast<unsigned>(D) : c < D;
    }
};

__device__ __forceinline__ void unpack8(uint4 u, float (&x)[8]) {
    x[0] = bf16_low(u.x), x[1] = bf16_high(u.x), x[2] = bf16_low(u.y), x[3] = bf16_high(u.y);
    x[4] = bf16_low(u.z), x[5] = bf16_high(u.z), x[6] = bf16_low(u.w), x[7] = bf16_high(u.w);
}

// Eight columns as they are in memory, from their load to their use.
template <typename R>
struct Raw;
template <>
struct Raw<uint16_t> {
    uint4 u;
    template <bool ODD>
    __device__ __forceinline__ void load(const uint16_t* row, int c, const Row<ODD>& r) {
        u = make_uint4(0, 0, 0, 0);
        if (r.whole(c)) {
            u = load_row16(row + c);
        } else if (ODD) {
            uint32_t w[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = r.has(c, e) ? row[c + e] : 0u;
            u = make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
        }
    }
    __device__ __forceinline__ void values(float (&x)[8]) const { unpack8(u, x); }
};
template <>
struct Raw<float> {
    uint4 a, b;
    template <bool ODD>
    __device__ __forceinline__ void load(const float* row, int c, const Row<ODD>& r) {
        a = b = make_uint4(0, 0, 0, 0);
        if (r.whole(c)) {
            a = load_row16(row + c);
            b = load_row16(row + c + 4);
        } else if (ODD) {
            uint32_t w[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = r.has(c, e) ? __float_as_uint(row[c + e]) : 0u;
            a = make_uint4(w[0], w[1], w[2], w[3]);
            b = make_uint4(w[4], w[5], w[6], w[7]);
        }
    }
    __device__ __forceinline__ void values(float (&x)[8]) const {
        x[0] = __uint_as_float(a.x), x[1] = __uint_as_float(a.y), x[2] = __uint_as_float(a.z);
        x[3] = __uint_as_float(a.w), x[4] = __uint_as_float(b.x), x[5] = __uint_as_float(b.y);
        x[6] = __uint_as_float(b.z), x[7] = __uint_as_float(b.w);
    }
};

// Vectors that every row reads, through L1.
template <bool ODD>
__device__ __forceinline__ void load_vector(const uint16_t* vec, int c, const Row<ODD>& r, float (&x)[8]) {
    if constexpr (!ODD) {
        unpack8(r.whole(c) ? __ldg(reinterpret_cast<const uint4*>(vec + c)) : make_uint4(0, 0, 0, 0), x);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = r.has(c, e) ? bf16_low(__ldg(vec + c + e)) : 0.0f;
    }
}

template <bool ODD>
__device__ __forceinline__ void store8(uint16_t* row, int c, const Row<ODD>& r, const float (&x)[8]) {
    if (r.whole(c)) {
        *reinterpret_cast<uint4*>(row + c) = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]),
                                                        pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
    } else if (ODD) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (r.has(c, e)) row[c + e] = __bfloat16_as_ushort(__float2bfloat16_rn(x[e]));
    }
}

template <bool ODD>
__device__ __forceinline__ void store8(float* row, int c, const Row<ODD>& r, const float (&x)[8]) {
    if (r.whole(c)) {
        *reinterpret_cast<float4*>(row + c) = make_float4(x[0], x[1], x[2], x[3]);
        *reinterpret_cast<float4*>(row + c + 4) = make_float4(x[4], x[5], x[6], x[7]);
    } else if (ODD) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (r.has(c, e)) row[c + e] = x[e];
    }
}

// Reductions over the threads of a row: lanes by exchange, warps through shared memory, in an order
// that is always the same.  `turn` alternates between two buffers: one barrier each.
struct Reducer {
    float (*parts)[kMaxWarps];
    int warps;  // of the row; 1: no shared memory
    int turn;

    template <bool MAX>
    __device__ __forceinline__ float reduce(float x) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            const float y = __shfl_xor_sync(0xffffffffu, x, o);
            x = MAX ? fmaxf(x, y) : x + y;
        }
        if (warps == 1) return x;
        float* const p = parts[turn & 1];
        ++turn;
        if ((threadIdx.x & 31) == 0) p[threadIdx.x >> 5] = x;
        __syncthreads();
        x = p[0];
        for (int w = 1; w < warps; ++w) x = MAX ? fmaxf(x, p[w]) : x + p[w];
        return x;
    }
};

// The mean (layer norm; else 0) and 1 / sqrt(mean square about it + eps) of a row.
template <int NV, bool ODD>
__device__ __forceinline__ void statistics(const float (&x)[NV][8], bool layer, const Row<ODD>& r, float inv_d, float eps,
                                           Reducer& red, float* mean, float* rstd) {
    float m = 0.0f;
    if (layer) {
        // (a sum of x / D: one of x could overflow)
        float sum = 0.0f;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (r.has(r.first(v), e)) sum = fmaf(x[v][e], inv_d, sum);
        m = red.reduce<false>(sum);
    }
    float ss = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (r.has(r.first(v), e)) {
                const float c = x[v][e] - m;
                ss = fmaf(c, c, ss);
            }
    const float total = red.reduce<false>(ss);
    *mean = m;
    *rstd = rsqrtf(fmaf(total, inv_d, eps));
    if (total < 1e38f) return;
    // Squares that overflow, of values that do not: divided by a power of two near the largest.  (The
    // branch is the same for all threads of the row.  An infinity or a NaN gives 0 or NaN, as the
    // formula has it.)
    float top = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (r.has(r.first(v), e)) top = fmaxf(top, fabsf(x[v][e] - m));
    top = red.reduce<true>(top);
    if (!(top < INFINITY) || total != total) return;
    const float s = __uint_as_float((253u << 23) - (__float_as_uint(top) & 0x7F800000u));  // 2^-exponent / 2
    ss = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (r.has(r.first(v), e)) {
                const float c = (x[v][e] - m) * s;
                ss = fmaf(c, c, ss);
            }
    *rstd = s * rsqrtf(red.reduce<false>(ss) * inv_d);  // (eps s^2 is far below half a step)
}

template <typename R, int NV, bool ODD>
__global__ void __launch_bounds__(NV > 8 ? 384 : 512) residual_norm_kernel(const NormParams p, const int group) {
    // (with more pieces than that the stream's values are read after the block's norm: registers)
    constexpr bool kAhead = NV <= 6;
    __shared__ float parts[2][kMaxWarps];
    const int64_t row = group == 32 ? static_cast<int64_t>(blockIdx.x) * (blockDim.x >> 5) + (threadIdx.x >> 5)
                                    : blockIdx.x;
    grid_launch_dependents();
    grid_wait();
    if (row >= p.M) return;  // (a whole warp; a CTA's row always exists)
    Reducer red{parts, group >> 5, 0};
    const int D = p.D;
    const int64_t at = row * D;
    const Row<ODD> r{static_cast<int>(group == 32 ? threadIdx.x & 31 : threadIdx.x), group, D,
                     static_cast<int>(at & 7)};
    const float inv_d = 1.0f / static_cast<float>(D);
    const R* const residual = static_cast<const R*>(p.residual) + at;
    float x[NV][8];
    if (p.block != nullptr) {
        Raw<R> stream[kAhead ? NV : 1];
        constexpr int kTogether = kAhead ? NV : 4;
        static_assert(NV % kTogether == 0, "a row's pieces in whole batches");
#pragma unroll
        for (int v0 = 0; v0 < NV; v0 += kTogether) {
            Raw<uint16_t> block[kTogether];
#pragma unroll
            for (int v = 0; v < kTogether; ++v) block[v].load(p.block + at, r.first(v0 + v), r);
            if constexpr (kAhead) {
#pragma unroll
                for (int v = 0; v < NV; ++v) stream[v].load(residual, r.first(v), r);
            }
#pragma unroll
            for (int v = 0; v < kTogether; ++v) block[v].values(x[v0 + v]);
        }
        if (p.post_weight != nullptr) {
            float mean, rstd;
            statistics<NV, ODD>(x, p.layer, r, inv_d, p.eps, red, &mean, &rstd);
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                float w[8];
                load_vector(p.post_weight, r.first(v), r, w);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[v][e] = (x[v][e] - mean) * rstd * (p.weight_offset + w[e]);
                if (p.post_bias != nullptr) {
                    load_vector(p.post_bias, r.first(v), r, w);
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[v][e] += w[e];
                }
            }
        }
        if (p.gate != nullptr) {
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                float w[8];
                if (p.gate_stride == 0) {
                    load_vector(p.gate, r.first(v), r, w);
                } else {
                    Raw<uint16_t> g;
                    g.load(p.gate + at, r.first(v), r);
                    g.values(w);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) x[v][e] *= w[e];
            }
        }
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            float w[8];
            if constexpr (!kAhead) stream[0].load(residual, r.first(v), r);
            stream[kAhead ? v : 0].values(w);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[v][e] = fmaf(p.residual_scale, w[e], x[v][e]);
        }
    } else {
        constexpr int kTogether = kAhead ? NV : 2;
#pragma unroll
        for (int v0 = 0; v0 < NV; v0 += kTogether) {
            Raw<R> stream[kTogether];
#pragma unroll
            for (int v = 0; v < kTogether; ++v) stream[v].load(residual, r.first(v0 + v), r);
#pragma unroll
            for (int v = 0; v < kTogether; ++v) {
                stream[v].values(x[v0 + v]);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[v0 + v][e] *= p.residual_scale;
            }
        }
    }
    if (p.residual_out != nullptr) {
        R* const to = static_cast<R*>(p.residual_out) + at;
#pragma unroll
        for (int v = 0; v < NV; ++v) store8(to, r.first(v), r, x[v]);
    }
    if (p.out == nullptr) return;
    float mean, rstd;
    statistics<NV, ODD>(x, p.layer, r, inv_d, p.eps, red, &mean, &rstd);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        float w[8], y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = (x[v][e] - mean) * rstd;
        if (p.weight != nullptr) {
            load_vector(p.weight, r.first(v), r, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] *= p.weight_offset + w[e];
        }
        if (p.bias != nullptr) {
            load_vector(p.bias, r.first(v), r, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] += w[e];
        }
        store8(p.out + at, r.first(v), r, y);
    }
}

template <typename R, bool ODD>
cudaError_t launch(const NormParams& p, cudaStream_t stream) {
    const int pieces = (p.D + (ODD ? 14 : 7)) / 8;  // units that a row may touch
    void (*kernel)(NormParams, int);
    int group = 32, threads = 256;
    if (pieces <= 128) {
        const int nv = (pieces + 31) / 32;
        kernel = nv == 1   ? residual_norm_kernel<R, 1, ODD>
                 : nv == 2 ? residual_norm_kernel<R, 2, ODD>
                 : nv == 3 ? residual_norm_kernel<R, 3, ODD>
                           : residual_norm_kernel<R, 4, ODD>;
    } else {
        const int least = (pieces + 511) / 512;
        const int nv = least <= 2 ? 2 : least <= 4 ? least : least <= 6 ? 6 : least <= 8 ? 8 : 16;
        if (ODD && nv > 6) return cudaErrorInvalidValue;  // (refused before: kNormMaxOdd)
        kernel = nv == 2   ? residual_norm_kernel<R, 2, ODD>
                 : nv == 3 ? residual_norm_kernel<R, 3, ODD>
                 : nv == 4 ? residual_norm_kernel<R, 4, ODD>
                 : nv == 6 ? residual_norm_kernel<R, 6, ODD>
                 : nv == 8 ? residual_norm_kernel<R, ODD ? 6 : 8, ODD>
                           : residual_norm_kernel<R, ODD ? 6 : 16, ODD>;
        group = threads = ((pieces + nv - 1) / nv + 31) / 32 * 32;
    }
    const int rows = threads / group;
    return launch_overlapped(kernel, (p.M - 1) / rows + 1, threads, 0, stream, p, group);
}

}  // namespace

cudaError_t launch_residual_norm(const NormParams& p, bool fp32, cudaStream_t stream) {
    const bool whole = p.D % 8 == 0;  // rows of 16-byte units (bases are 16-byte aligned)
    return fp32 ? (whole ? launch<float, false>(p, stream) : launch<float, true>(p, stream))
                : (whole ? launch<uint16_t, false>(p, stream) : launch<uint16_t, true>(p, stream));
}

}  // namespace w4a16
