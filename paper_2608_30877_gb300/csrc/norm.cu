// The residual stream between two blocks of the decoder, in one pass over its rows:
//   h = scale r + gate post(b),   out = pre(h)
// with post and pre RMS norms v / sqrt(mean v^2 + eps) or layer norms (v - mean) / sqrt(var + eps),
// each times (offset + weight) plus a bias.
//
// A row is read once and written once; between the reductions and the store its values stay on the SM, so that a
// variance is the mean of squares about a mean that is known (no difference of large sums).  The norm is of h as
// computed, not as rounded for the store.  Bound by HBM.  Where they stay:
//   registers, a warp to a row up to 1024 columns, else a CTA to a row: 39004 bf16 rows of 12288, RMS, 555 us (6.9 TB/s,
//     the copy bandwidth);
//   shared memory filled ahead by bulk copies, for what takes long between load and store (post norms, layer norms, an
//     fp32 stream): 4097 rows of 8200 with both layer norms, gate and biases on an fp32 stream 93 us (4.3 TB/s; 128
//     from registers), 20000 of 12288 with layer norms 95% of the copy bandwidth;
//   shared memory in fp32, a unit of eight columns at a time, for rows wider than 16384 and rows of odd width past a
//     warp's: 49152 columns 60%, 4099 columns 45% (the vectors' elements load one by one).
// One row is latency: 2.9 us on the device, the call's host side 13.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <cstdint>

#include "kv.h"
#include "layer.h"
#include "ptx.cuh"

namespace w4a16 {

namespace {

constexpr int kMaxWarps = 32;

__device__ __forceinline__ float bf16_low(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float bf16_high(uint32_t v) { return __uint_as_float(v & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&p);
}

// Two fp32 in one register pair, an instruction for both.
__device__ __forceinline__ uint64_t pair(float a, float b) {
    uint64_t p;
    asm("mov.b64 %0, {%1, %2};" : "=l"(p) : "f"(a), "f"(b));
    return p;
}
__device__ __forceinline__ float2 both(uint64_t p) {
    float2 v;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(v.x), "=f"(v.y) : "l"(p));
    return v;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
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
__device__ __forceinline__ uint4 load_vector(const uint16_t* vec, int c, const Row<ODD>& r) {
    if constexpr (!ODD) {
        return r.whole(c) ? __ldg(reinterpret_cast<const uint4*>(vec + c)) : make_uint4(0, 0, 0, 0);
    } else {
        uint32_t w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = r.has(c, e) ? __ldg(vec + c + e) : 0u;
        return make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
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

    __device__ __forceinline__ float sum(float x) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
        if (warps == 1) return x;
        float* const p = parts[turn & 1];
        ++turn;
        if ((threadIdx.x & 31) == 0) p[threadIdx.x >> 5] = x;
        __syncthreads();
        // (entries past the last warp's are 0)
        x = 0.0f;
        for (int w = 0; w < warps; w += 4) {
            const float4 v = *reinterpret_cast<const float4*>(p + w);
            x += (v.x + v.y) + (v.z + v.w);
        }
        return x;
    }
};

// The entries past a CTA's last warp; the first reduction's barrier is behind it.
__device__ __forceinline__ void clear(float (&parts)[2][kMaxWarps]) {
    const int t = threadIdx.x;
    if (t < 2 * kMaxWarps && t % kMaxWarps >= static_cast<int>(blockDim.x >> 5)) parts[t / kMaxWarps][t % kMaxWarps] = 0.0f;
}

// The mean (layer norm; else 0) and 1 / sqrt(mean square about it + eps) of a row.  pairs(absent, f): f(two values) for
// the thread's, in register pairs; a column that the row has not counts as `absent`.  scale(s): the thread's values
// times s, in their place.
//
// A mean that is off by a step is as much as the differences from it where a row's values are nearly equal.  The sum is of x
// itself (of x / D each term would be rounded), which is exact for values of few bits, as those of a bf16 stream are:
// rows of equal ones have no difference left.  (What is left for values of 24 bits: a mean that is off by a few steps. Correcting
// it by the differences' own sum took layer norms of 60000 bf16 rows of 4096 from 97% of the copy bandwidth to 85, beside the
// squares to 89, and only where the values lie within 2^-12 of the mean to 94, with RMS norms of gated rows from 98 to 82.)
template <bool PACKED, typename Pairs, typename Scale>
__device__ __forceinline__ void statistics(const Pairs& pairs, const Scale& scale, bool layer, float d, float inv_d,
                                           float eps, Reducer& red, float* mean, float* rstd) {
    const auto mean_of = [&]() {
        uint64_t sum = 0;
        pairs(0.0f, [&](uint64_t x) { sum = add2(sum, x); });
        const float all = red.sum(both(sum).x + both(sum).y), q = all * inv_d;
        return fmaf(fmaf(-q, d, all), inv_d, q);  // (all / d to the last bit)
    };
    float m = layer ? mean_of() : 0.0f;
    uint64_t ss = 0;
    if (PACKED || layer) {
        pairs(m, [&](uint64_t x) {
            const uint64_t c = add2(x, pair(-m, -m));
            ss = fma2(c, c, ss);
        });
    } else {
        float sum = 0.0f;
        pairs(0.0f, [&](uint64_t x) { sum = fmaf(both(x).x, both(x).x, fmaf(both(x).y, both(x).y, sum)); });
        ss = pair(sum, 0.0f);
    }
    float total = red.sum(both(ss).x + both(ss).y);
    *mean = m;
    *rstd = rsqrtf(fmaf(total, inv_d, eps));
    if (total < 1e38f) return;
    // Squares that overflow, of values that may not (and differences from the mean, and the mean's sum, of the largest
    // finite ones): the row is taken again times 2^-76, which leaves its norm as it is.  The root mean square was 2^55
    // at least, so that what counts stays a normal number and rstd below 2^22, as eps has it elsewhere; 49152 squares of
    // 2^(129 - 76) are far from overflow.  (The branch is the same for all threads of the row.  An infinity or a NaN gives
    // 0 or NaN, as the formula has it.)
    scale(0x1p-76f);
    m = layer ? mean_of() : 0.0f;
    ss = 0;
    pairs(m, [&](uint64_t x) {
        const uint64_t c = add2(x, pair(-m, -m));
        ss = fma2(c, c, ss);
    });
    total = red.sum(both(ss).x + both(ss).y);
    *mean = m;
    *rstd = rsqrtf(fmaf(total, inv_d, 1e-37f));  // (eps is far below half a step; not 1 / 0 where all are equal)
}

// f(two values) for a piece's pairs, with `absent` where the row has no column.
template <bool ODD, typename F>
__device__ __forceinline__ void piece_pairs(const float (&x)[8], int c, const Row<ODD>& r, float absent, const F& f) {
    if (ODD) {
#pragma unroll
        for (int e = 0; e < 8; e += 2) f(pair(r.has(c, e) ? x[e] : absent, r.has(c, e + 1) ? x[e + 1] : absent));
    } else if (r.whole(c)) {
#pragma unroll
        for (int e = 0; e < 8; e += 2) f(pair(x[e], x[e + 1]));
    } else {
        const uint64_t none = pair(absent, absent);
#pragma unroll
        for (int e = 0; e < 8; e += 2) f(none);
    }
}

template <bool PACKED, int NV, bool ODD>
__device__ __forceinline__ void statistics(float (&x)[NV][8], bool layer, const Row<ODD>& r, float inv_d, float eps,
                                           Reducer& red, float* mean, float* rstd) {
    statistics<PACKED>(
        [&](float absent, const auto& f) {
#pragma unroll
            for (int v = 0; v < NV; ++v) piece_pairs(x[v], r.first(v), r, absent, f);
        },
        [&](float s) {
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int e = 0; e < 8; ++e) x[v][e] *= s;
        },
        layer, static_cast<float>(r.D), inv_d, eps, red, mean, rstd);
}

// x = (x - mean) rstd (offset + weight) + bias; no weight: a factor of 1.  PACKED: in register pairs, which
// take more registers.
template <bool PACKED>
__device__ __forceinline__ void normalise8(float (&x)[8], float mean, float rstd, float offset, bool weighted, uint4 weight,
                                           bool biased, uint4 bias) {
    float w[8], b[8];
    unpack8(weight, w);
    unpack8(bias, b);
    if constexpr (PACKED) {
        const uint64_t minus = pair(-mean, -mean), scale = pair(rstd, rstd), more = pair(offset, offset);
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            const uint64_t c = add2(pair(x[e], x[e + 1]), minus);
            const uint64_t factor = weighted ? mul2(add2(pair(w[e], w[e + 1]), more), scale) : scale;
            const float2 y = both(biased ? fma2(c, factor, pair(b[e], b[e + 1])) : mul2(c, factor));
            x[e] = y.x;
            x[e + 1] = y.y;
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float c = x[e] - mean, factor = weighted ? (w[e] + offset) * rstd : rstd;
            x[e] = biased ? fmaf(c, factor, b[e]) : c * factor;
        }
    }
}

// The same for a row; the weights' loads together.
template <bool PACKED, int NV, bool ODD>
__device__ __forceinline__ void normalise(float (&x)[NV][8], const uint16_t* weight, const uint16_t* bias, const Row<ODD>& r,
                                          float mean, float rstd, float offset) {
    const uint4 none = make_uint4(0, 0, 0, 0);
    uint4 w[NV];
    if (PACKED && weight != nullptr && bias != nullptr) {
#pragma unroll
        for (int v = 0; v < NV; ++v) w[v] = load_vector(weight, r.first(v), r);
#pragma unroll
        for (int v = 0; v < NV; ++v)
            normalise8<PACKED>(x[v], mean, rstd, offset, true, w[v], true, load_vector(bias, r.first(v), r));
        return;
    }
    if (weight != nullptr) {
#pragma unroll
        for (int v = 0; v < NV; ++v) w[v] = load_vector(weight, r.first(v), r);
#pragma unroll
        for (int v = 0; v < NV; ++v) normalise8<PACKED>(x[v], mean, rstd, offset, true, w[v], false, none);
    } else {
#pragma unroll
        for (int v = 0; v < NV; ++v) normalise8<PACKED>(x[v], mean, rstd, offset, false, none, false, none);
    }
    if (bias != nullptr) {
#pragma unroll
        for (int v = 0; v < NV; ++v) w[v] = load_vector(bias, r.first(v), r);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            float b[8];
            unpack8(w[v], b);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[v][e] += b[e];
        }
    }
}

// The rest of a row whose block output is x (its scaled stream values without a block): `stream` and
// `gate` give a piece's values.
template <bool PACKED, typename R, int NV, bool ODD, typename Stream, typename Gate>
__device__ __forceinline__ void finish_row(const NormParams& p, const Row<ODD>& r, int64_t at, float inv_d, Reducer& red,
                                           float (&x)[NV][8], const Stream& stream, const Gate& gate) {
    const float offset = p.weight_offset;
    float mean, rstd;
    if (p.block != nullptr) {
        if (p.post_weight != nullptr) {
            statistics<PACKED>(x, p.layer, r, inv_d, p.eps, red, &mean, &rstd);
            normalise<PACKED>(x, p.post_weight, p.post_bias, r, mean, rstd, offset);
        }
        if (p.gate != nullptr) {
            if (p.gate_stride == 0) {
                uint4 raw[NV];
#pragma unroll
                for (int v = 0; v < NV; ++v) raw[v] = load_vector(p.gate, r.first(v), r);
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    float w[8];
                    unpack8(raw[v], w);
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[v][e] *= w[e];
                }
            } else {
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    float w[8];
                    gate(v, w);
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[v][e] *= w[e];
                }
            }
        }
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            float w[8];
            stream(v, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[v][e] = fmaf(p.residual_scale, w[e], x[v][e]);
        }
    }
    if (!dbg_check(at >= 0 && at + p.D <= static_cast<int64_t>(p.M) * p.D, p.status)) return;
    if (p.residual_out != nullptr) {
        R* const to = static_cast<R*>(p.residual_out) + at;
#pragma unroll
        for (int v = 0; v < NV; ++v) store8(to, r.first(v), r, x[v]);
    }
    if (p.out == nullptr) return;
    statistics<PACKED>(x, p.layer, r, inv_d, p.eps, red, &mean, &rstd);
    normalise<PACKED>(x, p.weight, p.bias, r, mean, rstd, offset);
#pragma unroll
    for (int v = 0; v < NV; ++v) store8(p.out + at, r.first(v), r, x[v]);
}

// A warp (up to 1024 columns) or a CTA to a row, which it holds in registers from the first load on.
template <typename R, int NV, bool ODD>
__global__ void __launch_bounds__(512, NV <= 3 && !ODD ? 2 : 1) residual_norm_kernel(const NormParams p, const int group) {
    __shared__ __align__(16) float parts[2][kMaxWarps];
    const int64_t row = group == 32 ? static_cast<int64_t>(blockIdx.x) * (blockDim.x >> 5) + (threadIdx.x >> 5)
                                    : blockIdx.x;
    grid_launch_dependents();
    grid_wait();
    if (row >= p.M) return;  // (a whole warp; a CTA's row always exists)
    Reducer red{parts, group >> 5, 0};
    clear(parts);
    const int64_t at = row * p.D;
    const Row<ODD> r{static_cast<int>(group == 32 ? threadIdx.x & 31 : threadIdx.x), group, p.D,
                     static_cast<int>(at & 7)};
    const float inv_d = 1.0f / static_cast<float>(p.D);
    const R* const residual = static_cast<const R*>(p.residual) + at;
    float x[NV][8];
    Raw<R> stream[NV];
    if (p.block != nullptr) {
        Raw<uint16_t> block[NV];
#pragma unroll
        for (int v = 0; v < NV; ++v) block[v].load(p.block + at, r.first(v), r);
#pragma unroll
        for (int v = 0; v < NV; ++v) stream[v].load(residual, r.first(v), r);
#pragma unroll
        for (int v = 0; v < NV; ++v) block[v].values(x[v]);
    } else {
#pragma unroll
        for (int v = 0; v < NV; ++v) stream[v].load(residual, r.first(v), r);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            stream[v].values(x[v]);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[v][e] *= p.residual_scale;
        }
    }
    finish_row<false, R, NV, ODD>(
        p, r, at, inv_d, red, x, [&](int v, float (&w)[8]) { stream[v].values(w); },
        [&](int v, float (&w)[8]) {
            Raw<uint16_t> g;
            g.load(p.gate + at, r.first(v), r);
            g.values(w);
        });
}

// Many rows of whole 16-byte units: as many CTAs as are resident, each with a ring of rows in shared
// memory that bulk copies fill while it is at a row before (the reductions leave the memory idle otherwise).  What is
// left is issue slots (44%) and the vectors, which the rings leave no room for in L1: five of them come from L2 for every
// row.  Register pairs (half the arithmetic instructions) took 99 us to 93.
constexpr int kRingThreads = 384;
constexpr int kRingRows = 4;               // at most
constexpr int kSmBytes = 224 * 1024;       // of an SM's shared memory, for all its rings
constexpr int kRingBytes = 114 * 1024;     // of one: two CTAs an SM at least

__device__ __forceinline__ void copy_row(uint32_t to, const void* from, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(to), "l"(from),
                 "r"(bytes), "r"(bar)
                 : "memory");
}

template <typename R>
__device__ __forceinline__ void ring_values(const uint8_t* row, int c, float (&w)[8]) {
    Raw<R> raw;
    const uint4* const at = reinterpret_cast<const uint4*>(row + c * sizeof(R));
    if constexpr (sizeof(R) == 2) {
        raw.u = at[0];
    } else {
        raw.a = at[0];
        raw.b = at[1];
    }
    raw.values(w);
}

template <typename R, int NV>
__global__ void __launch_bounds__(kRingThreads, 2) residual_norm_ring_kernel(const NormParams p, const int depth) {
    extern __shared__ __align__(16) uint8_t ring[];
    __shared__ __align__(16) float parts[2][kMaxWarps];
    __shared__ __align__(8) uint64_t full[kRingRows];
    __shared__ int abort_flag;
    const int D = p.D;
    const uint32_t stream_bytes = D * static_cast<uint32_t>(sizeof(R)), block_bytes = p.block != nullptr ? D * 2u : 0u,
                   gate_bytes = p.gate != nullptr && p.gate_stride != 0 ? D * 2u : 0u;
    const uint32_t row_bytes = stream_bytes + block_bytes + gate_bytes;
    if (threadIdx.x == 0) {
        for (int i = 0; i < depth; ++i) mbar_init(smem_u32(&full[i]), 1);
        abort_flag = 0;
        fence_mbar_init();
    }
    grid_launch_dependents();
    grid_wait();
    __syncthreads();
    auto fetch = [&](int slot, int64_t row) {  // one thread
        const uint32_t bar = smem_u32(&full[slot]), to = smem_u32(ring) + slot * row_bytes;
        if (!dbg_check(slot < depth && (to & 15u) == 0 && row < p.M, p.status)) return;
        mbar_arrive_expect_tx(bar, row_bytes);
        if (block_bytes != 0) copy_row(to, p.block + row * D, block_bytes, bar);
        copy_row(to + block_bytes, static_cast<const R*>(p.residual) + row * D, stream_bytes, bar);
        if (gate_bytes != 0) copy_row(to + block_bytes + stream_bytes, p.gate + row * D, gate_bytes, bar);
    };
    bool ok = true;
    if (threadIdx.x == 0) {
        for (int i = 0; i < depth; ++i) {
            const int64_t row = blockIdx.x + static_cast<int64_t>(i) * gridDim.x;
            if (row < p.M) fetch(i, row);
        }
        ok = short_limit_ok(smem_u32(&full[0]), 0, &abort_flag, p.status, p.wait_ns);
    }
    Reducer red{parts, static_cast<int>(blockDim.x) >> 5, 0};
    clear(parts);
    const Row<false> r{static_cast<int>(threadIdx.x), static_cast<int>(blockDim.x), D, 0};
    const float inv_d = 1.0f / static_cast<float>(D);
    const int64_t step = gridDim.x;
    int slot = 0;
    uint32_t parity = 0;
    for (int64_t row = blockIdx.x; row < p.M; row += step) {
        ok = wait_warp(smem_u32(&full[slot]), parity, &abort_flag, p.status, p.wait_ns) && ok;
        const bool begun = row != blockIdx.x;
        if (__syncthreads_or(!ok)) {
            if (threadIdx.x == 0)  // the copies under way land before the CTA ends
                for (int i = 0; i < depth - begun && row + i * step < p.M; ++i) {
                    settle(smem_u32(&full[slot]), parity);
                    slot = slot + 1 == depth ? 0 : slot + 1;
                    parity ^= slot == 0;
                }
            return;
        }
        // every thread is done with the row before: its place takes the next one
        if (threadIdx.x == 0 && begun && row + (depth - 1) * step < p.M)
            fetch(slot == 0 ? depth - 1 : slot - 1, row + (depth - 1) * step);
        const uint8_t* const from = ring + slot * row_bytes;
        float x[NV][8];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = r.first(v);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[v][e] = 0.0f;
            if (c < D) {
                if (block_bytes != 0) {
                    ring_values<uint16_t>(from, c, x[v]);
                } else {
                    ring_values<R>(from, c, x[v]);
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[v][e] *= p.residual_scale;
                }
            }
        }
        auto values = [&](const uint8_t* part, auto type, int v, float (&w)[8]) {
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = 0.0f;
            if (r.first(v) < D) ring_values<decltype(type)>(part, r.first(v), w);
        };
        finish_row<true, R, NV, false>(
            p, r, row * D, inv_d, red, x, [&](int v, float (&w)[8]) { values(from + block_bytes, R{}, v, w); },
            [&](int v, float (&w)[8]) { values(from + block_bytes + stream_bytes, uint16_t{}, v, w); });
        slot = slot + 1 == depth ? 0 : slot + 1;
        parity ^= slot == 0;
    }
}

template <typename R>
bool launch_ring(const NormParams& p, int sm_count, cudaStream_t stream, cudaError_t* e) {
    const int row_bytes = p.D * (static_cast<int>(sizeof(R)) + (p.block != nullptr ? 2 : 0) +
                                 (p.gate != nullptr && p.gate_stride != 0 ? 2 : 0));
    const int pieces = p.D / 8, least = (pieces + kRingThreads - 1) / kRingThreads;
    const int nv = least <= 2 ? 2 : least;
    const int threads = ((pieces + nv - 1) / nv + 31) / 32 * 32;
    // as many CTAs an SM as have registers (80 a thread), with two rows each at least
    int ctas = 65536 / (80 * threads);
    if (ctas > 4) ctas = 4;
    while (ctas > 2 && kSmBytes / ctas / row_bytes < 2) --ctas;
    int depth = kSmBytes / ctas / row_bytes;
    if (depth > kRingRows) depth = kRingRows;
    if (depth * row_bytes > kRingBytes) depth = kRingBytes / row_bytes;
    if (depth < 2 || p.M < 2 * ctas * sm_count) return false;
    auto kernel = nv == 2   ? residual_norm_ring_kernel<R, 2>
                  : nv == 3 ? residual_norm_ring_kernel<R, 3>
                            : residual_norm_ring_kernel<R, 4>;
    // (the same limit for every size: calls of several threads set it at the same time)
    *e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRingBytes);
    if (*e == cudaSuccess)
        *e = launch_overlapped(kernel, dim3(ctas * sm_count), threads, depth * row_bytes, stream, p, depth);
    return true;
}

// Rows wider than registers hold, and rows of odd width past a warp's: one CTA to a row, whose values are in
// shared memory in fp32 between the passes; a thread works on its own units alone.
constexpr int kWideThreads = 1024;  // at most

template <typename R, bool ODD>
__global__ void __launch_bounds__(kWideThreads) residual_norm_wide_kernel(const NormParams p) {
    extern __shared__ __align__(16) float values[];
    __shared__ __align__(16) float parts[2][kMaxWarps];
    const int64_t row = blockIdx.x, at = row * p.D;
    grid_launch_dependents();
    grid_wait();
    const int threads = static_cast<int>(blockDim.x);
    Reducer red{parts, threads >> 5, 0};
    clear(parts);
    const Row<ODD> r{static_cast<int>(threadIdx.x), threads, p.D, static_cast<int>(at & 7)};
    const float inv_d = 1.0f / static_cast<float>(p.D), offset = p.weight_offset;
    const int pieces = (p.D + (ODD ? r.shift : 0) + 7) / 8;
    const R* const residual = static_cast<const R*>(p.residual) + at;
    const int own = static_cast<int>(threadIdx.x) < pieces ? (pieces - 1 - static_cast<int>(threadIdx.x)) / threads + 1 : 0;
    auto get = [&](int v, float (&x)[8]) {
        const float4* const from = reinterpret_cast<const float4*>(values + (v * threads + static_cast<int>(threadIdx.x)) * 8);
        const float4 a = from[0], b = from[1];
        x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    };
    auto put = [&](int v, const float (&x)[8]) {
        float4* const to = reinterpret_cast<float4*>(values + (v * threads + static_cast<int>(threadIdx.x)) * 8);
        to[0] = make_float4(x[0], x[1], x[2], x[3]);
        to[1] = make_float4(x[4], x[5], x[6], x[7]);
    };
    if (!dbg_check(at + p.D <= static_cast<int64_t>(p.M) * p.D, p.status)) return;
    auto stats = [&](float* mean, float* rstd) {
        statistics<true>(
            [&](float absent, const auto& f) {
                for (int v = 0; v < own; ++v) {
                    float x[8];
                    get(v, x);
                    piece_pairs(x, r.first(v), r, absent, f);
                }
            },
            [&](float s) {
                for (int v = 0; v < own; ++v) {
                    float x[8];
                    get(v, x);
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] *= s;
                    put(v, x);
                }
            },
            p.layer, static_cast<float>(p.D), inv_d, p.eps, red, mean, rstd);
    };
    float mean, rstd;
    if (p.block != nullptr && p.post_weight != nullptr) {
#pragma unroll 2
        for (int v = 0; v < own; ++v) {
            Raw<uint16_t> raw;
            raw.load(p.block + at, r.first(v), r);
            float x[8];
            raw.values(x);
            put(v, x);
        }
        stats(&mean, &rstd);
    }
#pragma unroll 2
    for (int v = 0; v < own; ++v) {
        const int c = r.first(v);
        float x[8], h[8], w[8];
        Raw<R> raw;
        raw.load(residual, c, r);
        raw.values(h);
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] *= p.residual_scale;
        if (p.block != nullptr) {
            if (p.post_weight != nullptr) {
                get(v, x);
                normalise8<true>(x, mean, rstd, offset, true, load_vector(p.post_weight, c, r), p.post_bias != nullptr,
                           p.post_bias != nullptr ? load_vector(p.post_bias, c, r) : make_uint4(0, 0, 0, 0));
            } else {
                Raw<uint16_t> block;
                block.load(p.block + at, c, r);
                block.values(x);
            }
            if (p.gate != nullptr) {
                if (p.gate_stride == 0) {
                    unpack8(load_vector(p.gate, c, r), w);
                } else {
                    Raw<uint16_t> gate;
                    gate.load(p.gate + at, c, r);
                    gate.values(w);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] *= w[e];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) h[e] += x[e];
        }
        if (p.residual_out != nullptr) store8(static_cast<R*>(p.residual_out) + at, c, r, h);
        put(v, h);
    }
    if (p.out == nullptr) return;
    stats(&mean, &rstd);
#pragma unroll 2
    for (int v = 0; v < own; ++v) {
        const int c = r.first(v);
        float x[8];
        get(v, x);
        const uint4 none = make_uint4(0, 0, 0, 0);
        normalise8<true>(x, mean, rstd, offset, p.weight != nullptr, p.weight != nullptr ? load_vector(p.weight, c, r) : none,
                   p.bias != nullptr, p.bias != nullptr ? load_vector(p.bias, c, r) : none);
        store8(p.out + at, c, r, x);
    }
}

template <typename R, bool ODD>
cudaError_t launch_wide(const NormParams& p, cudaStream_t stream) {
    const int units = (p.D + (ODD ? 14 : 7)) / 8;
    int threads = 256;  // with two to four units each, as far as that goes
    while (threads < kWideThreads && units > 4 * threads) threads *= 2;
    const int smem = (units + threads - 1) / threads * threads * 32;
    constexpr int kMost = ((kNormMaxWidth + 14) / 8 + kWideThreads - 1) / kWideThreads * kWideThreads * 32;
    auto kernel = residual_norm_wide_kernel<R, ODD>;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost);
    if (e != cudaSuccess) return e;
    return launch_overlapped(kernel, dim3(p.M), threads, smem, stream, p);
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
        if (ODD || least > 4) return launch_wide<R, ODD>(p, stream);
        const int nv = least <= 2 ? 2 : least;
        kernel = nv == 2   ? residual_norm_kernel<R, 2, false>
                 : nv == 3 ? residual_norm_kernel<R, 3, false>
                           : residual_norm_kernel<R, 4, false>;
        group = threads = ((pieces + nv - 1) / nv + 31) / 32 * 32;
    }
    const int rows = threads / group;
    return launch_overlapped(kernel, (p.M - 1) / rows + 1, threads, 0, stream, p, group);
}

}  // namespace

cudaError_t launch_residual_norm(const NormParams& p, bool fp32, int sm_count, cudaStream_t stream) {
    const bool whole = p.D % 8 == 0;  // rows of 16-byte units (bases are 16-byte aligned)
    // (a plain bf16 RMS norm is at the copy bandwidth from registers: 39004 rows of 12288 551 us, 613 with the
    // ring; 4097 of 8200 with both layer norms and an fp32 stream 128, 93 with it)
    if (whole && p.D > 1024 && p.D <= 4 * 8 * kRingThreads && (fp32 || p.layer || p.post_weight != nullptr)) {
        cudaError_t e = cudaSuccess;
        if (fp32 ? launch_ring<float>(p, sm_count, stream, &e) : launch_ring<uint16_t>(p, sm_count, stream, &e)) return e;
    }
    return fp32 ? (whole ? launch<float, false>(p, stream) : launch<float, true>(p, stream))
                : (whole ? launch<uint16_t, false>(p, stream) : launch<uint16_t, true>(p, stream));
}

}  // namespace w4a16
