// Attention of one new token per sequence over the paged key-value cache.
//
// out = sum_j softmax_j(q . k_j / sqrt(128)) v_j, the running maximum and sum of the softmax
// in fp32 over one pass of the keys.  A CTA has one row and query head: its warps take
// keys in turn, a lane four of the 128 values, and their parts are joined in shared
// memory.  The new token's key and value come from the projection's row, in the form in
// which the cache holds them, and one CTA per key head stores them.
#include <cuda_runtime.h>
#include <cstdint>

#include "kv.h"
#include "kv_row.cuh"
#include "ptx.cuh"

namespace w4a16 {

namespace {

constexpr int kWarps = 4;

__device__ __forceinline__ float4 bf16_quad(uint2 v) {
    return make_float4(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xFFFF0000u),
                       __uint_as_float(v.y << 16), __uint_as_float(v.y & 0xFFFF0000u));
}
__device__ __forceinline__ float2 half2_floats(uint32_t h) {
    float2 r;
    asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %2;\n\tcvt.f32.f16 %0, lo;\n\tcvt.f32.f16 %1, hi;\n\t}"
        : "=f"(r.x), "=f"(r.y) : "r"(h));
    return r;
}
__device__ __forceinline__ float4 e4m3_floats(uint32_t codes, float s) {
    const float2 a = half2_floats(e4m3_to_half2(static_cast<uint16_t>(codes)));
    const float2 b = half2_floats(e4m3_to_half2(static_cast<uint16_t>(codes >> 16)));
    return make_float4(a.x * s, a.y * s, b.x * s, b.y * s);
}

template <bool E4M3>
__device__ __forceinline__ float4 cache_quad(const KvView& kv, int layer, int which, int page, int head,
                                             int at, int lane) {
    const int64_t row = kv_row(kv, layer, which, page, head, at);
    if constexpr (E4M3)
        return e4m3_floats(reinterpret_cast<const uint32_t*>(kv.pages)[row * 32 + lane],
                           power_of_two(kv.exponents[kv_exponent(kv, layer, which, page, head, at)] - 127));
    else
        return bf16_quad(reinterpret_cast<const uint2*>(kv.pages)[row * 32 + lane]);
}

// The new token's key or value as the cache holds it; stored if `store`.
template <bool E4M3>
__device__ __forceinline__ float4 new_quad(const KvView& kv, const DecodeParams& p, int row, int which,
                                           int page, int head, int at, int lane, bool store) {
    const uint2 v = reinterpret_cast<const uint2*>(
        p.qkv + (static_cast<int64_t>(row) * (p.H + 2 * kv.kv_heads) + p.H + which * kv.kv_heads + head) *
                    kKvHeadDim)[lane];
    const int64_t to = kv_row(kv, p.layer, which, page, head, at);
    const float4 f = bf16_quad(v);
    if constexpr (!E4M3) {
        if (store) reinterpret_cast<uint2*>(kv.pages)[to * 32 + lane] = v;
        return f;
    } else {
        float top = fmaxf(fmaxf(finite_abs(f.x), finite_abs(f.y)), fmaxf(finite_abs(f.z), finite_abs(f.w)));
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        const int e = e4m3_row_exponent(top);
        const float s = power_of_two(-e);
        const uint32_t codes = e4m3_quad(f.x * s, f.y * s, f.z * s, f.w * s);
        if (store) {
            reinterpret_cast<uint32_t*>(kv.pages)[to * 32 + lane] = codes;
            if (lane == 0)
                kv.exponents[kv_exponent(kv, p.layer, which, page, head, at)] = static_cast<uint8_t>(e + 127);
        }
        return e4m3_floats(codes, power_of_two(e));
    }
}

template <bool E4M3>
__global__ void __launch_bounds__(kWarps * 32)
    attention_decode_kernel(const KvView kv, const DecodeParams p) {
    __shared__ float part_m[kWarps], part_l[kWarps];
    __shared__ float4 part_o[kWarps][32];
    const int row = blockIdx.x, h = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int group = p.H / kv.kv_heads, head = h / group;
    uint2* out = reinterpret_cast<uint2*>(p.out + (static_cast<int64_t>(row) * p.H + h) * kKvHeadDim);
    const int slot = p.slots[row];
    int len = 0;
    bool bad = slot < -1 || slot >= kv.num_slots;
    if (!bad && slot >= 0) {
        len = kv.seq_len[slot];
        bad = len < 0 || len > static_cast<int64_t>(kv.max_pages) << kv.page_shift;
    }
    const int low = len > p.window ? len - p.window : 0;
    const int32_t* table = kv.table + static_cast<int64_t>(slot) * kv.max_pages;
    if (!bad)
        for (int e = (low >> kv.page_shift) + threadIdx.x; e << kv.page_shift < len; e += kWarps * 32)
            bad |= table[e] < 0 || table[e] >= kv.num_pages;
    bad = __syncthreads_or(bad);
    if (bad && threadIdx.x == 0) record_status(kv.status, 1 /* W4A16_ERR_INVALID_ARG */);
    if (bad || len == 0) {
        if (warp == 0) out[lane] = make_uint2(0, 0);
        return;
    }
    const float4 q = bf16_quad(reinterpret_cast<const uint2*>(
        p.qkv + (static_cast<int64_t>(row) * (p.H + 2 * kv.kv_heads) + h) * kKvHeadDim)[lane]);
    const float scale = p.scale * 1.4426950408889634f;
    float m = -INFINITY, l = 0.0f;
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int j = low + warp; j < len; j += kWarps) {
        const int page = table[j >> kv.page_shift], at = j & ((1 << kv.page_shift) - 1);
        const bool fresh = j == len - 1, store = h == head * group;
        const float4 k = fresh ? new_quad<E4M3>(kv, p, row, 0, page, head, at, lane, store)
                               : cache_quad<E4M3>(kv, p.layer, 0, page, head, at, lane);
        float s = q.x * k.x + q.y * k.y + q.z * k.z + q.w * k.w;
#pragma unroll
        for (int i = 16; i > 0; i >>= 1) s += __shfl_xor_sync(0xffffffffu, s, i);
        s *= scale;
        const float4 v = fresh ? new_quad<E4M3>(kv, p, row, 1, page, head, at, lane, store)
                               : cache_quad<E4M3>(kv, p.layer, 1, page, head, at, lane);
        const float top = fmaxf(m, s), base = top == -INFINITY ? 0.0f : top;
        const float a = exp2f(m - base), w = exp2f(s - base);
        l = l * a + w;
        o = make_float4(o.x * a + w * v.x, o.y * a + w * v.y, o.z * a + w * v.z, o.w * a + w * v.w);
        m = top;
    }
    if (lane == 0) part_m[warp] = m, part_l[warp] = l;
    part_o[warp][lane] = o;
    __syncthreads();
    if (warp != 0) return;
    float top = -INFINITY;
    for (int w = 0; w < kWarps; ++w) top = fmaxf(top, part_m[w]);
    const float base = top == -INFINITY ? 0.0f : top;
    l = 0.0f;
    o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int w = 0; w < kWarps; ++w) {
        const float a = exp2f(part_m[w] - base);
        const float4 x = part_o[w][lane];
        l += a * part_l[w];
        o = make_float4(o.x + a * x.x, o.y + a * x.y, o.z + a * x.z, o.w + a * x.w);
    }
    auto pair = [](float lo, float hi) {
        uint32_t r;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
        return r;
    };
    out[lane] = make_uint2(pair(o.x / l, o.y / l), pair(o.z / l, o.w / l));
}

}  // namespace

int64_t decode_workspace_bytes(int, int, int) { return 16; }

cudaError_t launch_attention_decode(const KvView& kv, const DecodeParams& p, int, cudaStream_t stream) {
    const dim3 grid(p.n, p.H);
    if (kv.exponents != nullptr)
        attention_decode_kernel<true><<<grid, kWarps * 32, 0, stream>>>(kv, p);
    else
        attention_decode_kernel<false><<<grid, kWarps * 32, 0, stream>>>(kv, p);
    return cudaGetLastError();
}

}  // namespace w4a16
