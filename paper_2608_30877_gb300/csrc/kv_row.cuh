// Rows of the key-value cache: where a token's key or value of one head lies, and the
// 8-bit form of a row.
#pragma once

#include <cstdint>

#include "kv.h"

namespace w4a16 {

// Row of (layer, key or value, page, head, token in the page), in rows of 128 values; a
// long cache passes 32 bits.
__device__ __forceinline__ int64_t kv_row(const KvView& kv, int layer, int which, int page, int head,
                                          int at) {
    return ((((static_cast<int64_t>(layer) * 2 + which) * kv.num_pages + page) * kv.kv_heads + head)
            << kv.page_shift) + at;
}
// Its exponent byte.
__device__ __forceinline__ int64_t kv_exponent(const KvView& kv, int layer, int which, int page,
                                               int head, int at) {
    return ((((static_cast<int64_t>(layer) * kv.num_pages + page) * kv.kv_heads + head)
             << kv.page_shift) + at) * 2 + which;
}

// Whether any slot has a mark, and whether nothing is to be stored for this one: its growth was
// refused.  (The marks alone, read with the length of every row, were 3 us of the 46 that 512 rows of 50
// to 300 tokens take.)
__device__ __forceinline__ bool any_refused(const KvView& kv) {
    return reinterpret_cast<const KvScratch*>(kv.scratch)->refused != 0;
}
__device__ __forceinline__ bool growth_refused(const KvView& kv, bool any, int slot) {
    return any && kv.refused[slot] == kKvRefused;
}

// The 8-bit form takes a power of two per row, not amax / 448: a power of two scales
// exactly, costs an e4m3 code no relative precision, and takes one byte.
constexpr int kKvMinExp = -120;

// The smallest e >= kKvMinExp with amax <= 448 * 2^e, amax finite and not negative:
// 448 = 1.75 * 2^8, so e is amax's exponent less 8, one more if its mantissa is past 1.75.
__device__ __forceinline__ int e4m3_row_exponent(float amax) {
    const uint32_t b = __float_as_uint(amax);
    const int e = static_cast<int>(b >> 23) - 127 - 8 + ((b & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return e < kKvMinExp ? kKvMinExp : e;
}
// |x| for the row's largest; what is not finite does not count.
__device__ __forceinline__ float finite_abs(float x) {
    const float a = fabsf(x);
    return a < __int_as_float(0x7F800000) ? a : 0.0f;
}
// 2^e within the normal range.
__device__ __forceinline__ float power_of_two(int e) {
    return __uint_as_float(static_cast<uint32_t>(e + 127) << 23);
}
// Two values to e4m3, the first in the low byte; round to nearest even, infinities to 448.
__device__ __forceinline__ uint32_t e4m3_pair(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t e4m3_quad(float a, float b, float c, float d) {
    return e4m3_pair(a, b) | (e4m3_pair(c, d) << 16);
}
// A row of 128 bf16 values to codes and its exponent: sixteen lanes (an aligned half of a warp,
// all of them here) with eight values each.
__device__ __forceinline__ int e4m3_row_of_16(uint4 v, uint2* codes) {
    const uint32_t u[4] = {v.x, v.y, v.z, v.w};
    const uint32_t half = 0xFFFFu << (threadIdx.x & 16);
    float f[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(u[i] << 16);
        f[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
    }
    // the largest magnitude's bits, two at a time: magnitudes are in the order of their bits
    uint32_t top2 = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) top2 = __vmaxu2(top2, u[i] & 0x7FFF7FFFu);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) top2 = __vmaxu2(top2, __shfl_xor_sync(half, top2, o));
    float top = __uint_as_float(max(top2 << 16, top2 & 0xFFFF0000u));
    if (!(top < __int_as_float(0x7F800000))) {  // (all 16 lanes, or none)
        top = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = fmaxf(top, finite_abs(f[i]));
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(half, top, o));
    }
    const int e = e4m3_row_exponent(top);
    const float s = power_of_two(-e);
    codes->x = e4m3_quad(f[0] * s, f[1] * s, f[2] * s, f[3] * s);
    codes->y = e4m3_quad(f[4] * s, f[5] * s, f[6] * s, f[7] * s);
    return e;
}
// Two e4m3 codes to a pair of halves, exactly.
__device__ __forceinline__ uint32_t e4m3_to_half2(uint16_t codes) {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(codes));
    return r;
}

}  // namespace w4a16
