// Rotary positions on the queries and keys of a fused projection's rows, in place: pair (a, b) of a
// head becomes (a cos t - b sin t, a sin t + b cos t) with t = position theta_i.
//
// The angle is taken modulo a turn before anything is rounded: a frequency is held as turns per
// token in units of 2^-64, so that position x frequency in 64-bit integers, whose overflow is
// whole turns, is the fraction of a turn, at any position.  Its upper 32 bits go to sincospif.
//
// Bound by HBM: the rotated part is read once and written once.  A CTA has up to four tokens and some of their heads:
// it finds the positions, computes each pair's sine and cosine once into shared memory, and then a thread turns the
// same eight pairs of one head of its token after another.  39004 tokens of 96 + 96 heads 559 us, the copy bandwidth;
// 12156 of 64 + 8 heads, half of each, 45 us (5.0 TB/s: 128-byte pieces, and the way to the positions is half of a
// CTA's time); one step of 64 sequences 3.1.  (Eight tokens to a CTA 568, 47; four CTAs an SM, which spill, 582.)
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <cstdint>

#include "kv.h"
#include "kv_row.cuh"
#include "layer.h"
#include "ptx.cuh"
#include "sequences.cuh"

namespace w4a16 {

namespace {

constexpr int kThreads = 256;
constexpr int kTokens = 4;      // of a CTA, at most
constexpr int kMaxPairs = 128;  // of a head: 256 dimensions

__device__ __forceinline__ float bf16_low(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float bf16_high(uint32_t v) { return __uint_as_float(v & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&p);
}

// Position of row m, -1 where the row is left as it is.
template <bool CACHE>
__device__ int64_t position_of(const KvView& kv, const RotaryParams& p, int m) {
    int begin = m, end = m + 1, s = m;  // (one row each)
    if (p.seq_start != nullptr) {
        s = sequence_of(p.seq_start, p.nseq, m, &begin, &end);
        if (s < 0) return -1;
        if (begin < 0 || end > p.M) {
            record_status(p.status, 1 /* W4A16_ERR_INVALID_ARG */);
            return -1;
        }
    }
    if constexpr (!CACHE) {
        const int first = p.first != nullptr ? p.first[s] : 0;
        return first < 0 ? -1 : static_cast<int64_t>(first) + (m - begin);
    } else {
        const int slot = p.first[s];
        if (slot == -1) return -1;
        bool ok = slot >= 0 && slot < kv.num_slots;
        int len = 0;
        if (ok) {
            len = kv.seq_len[slot];
            const bool refused = growth_refused(kv, true, slot);
            if (p.seq_start == nullptr && len == 0 && !refused) return -1;  // an empty sequence's row
            ok = !refused && len >= end - begin && len <= static_cast<int64_t>(kv.max_pages) << kv.page_shift;
        }
        if (!ok) {
            record_status(p.status, 1);
            return -1;
        }
        return static_cast<int64_t>(len) - end + m;
    }
}

// blockIdx.x: tokens; blockIdx.y: heads.
template <bool PAIRS, bool CACHE>
__global__ void __launch_bounds__(kThreads) rotary_kernel(const KvView kv, const RotaryParams p, const int tokens,
                                                          const int heads_per_cta) {
    __shared__ int64_t position[kTokens];
    __shared__ __align__(16) float2 turned[kTokens][kMaxPairs];  // cosine and sine, times the factor
    const int pairs = p.rot / 2;
    const int64_t m0 = static_cast<int64_t>(blockIdx.x) * tokens;
    // a unit: eight pairs of a head, in two pieces of 16 bytes; the tokens, and heads of each, side by side
    const int units = pairs / 8;
    const int side = kThreads / units / tokens;  // heads of a token
    const int u = threadIdx.x % units, t = threadIdx.x / units / side, h0 = threadIdx.x / units - t * side;
    const int heads = p.H + p.kv_heads;
    const int begin = static_cast<int>(blockIdx.y) * heads_per_cta, end = min(begin + heads_per_cta, heads);
    const int64_t width = static_cast<int64_t>(heads + p.kv_heads) * p.d;
    const int low = PAIRS ? 16 * u : 8 * u, high = PAIRS ? low + 8 : low + pairs;
    const bool there = t < tokens && m0 + t < p.M;
    uint16_t* const row = p.qkv + (m0 + (there ? t : 0)) * width;
    constexpr int kAhead = 4;
    uint4 a[kAhead], b[kAhead];
    auto load = [&](int h) {
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (h + k * side < end) {
                const uint16_t* const head = row + (h + k * side) * p.d;
                a[k] = __ldcs(reinterpret_cast<const uint4*>(head + low));
                b[k] = __ldcs(reinterpret_cast<const uint4*>(head + high));
            }
    };
    grid_launch_dependents();
    grid_wait();
    // (the first heads are on their way while the positions are looked up, a chain of four loads: 46 us of three
    // long contexts of shared heads without this)
    if (there) load(begin + h0);
    if (threadIdx.x < tokens)
        position[threadIdx.x] =
            m0 + threadIdx.x < p.M ? position_of<CACHE>(kv, p, static_cast<int>(m0 + threadIdx.x)) : -1;
    if (p.seq_start != nullptr && blockIdx.y == 0) check_starts(p.seq_start, p.nseq, p.M, p.status);
    __syncthreads();
    for (int i = threadIdx.x; i < tokens * pairs; i += kThreads) {
        const int of = i / pairs, j = i - of * pairs;
        const int64_t pos = position[of];
        if (pos >= 0) {
            const uint64_t turns = static_cast<uint64_t>(pos) * p.turns[j];
            float s, c;
            sincospif(static_cast<float>(static_cast<int32_t>(turns >> 32)) * 4.656612873077393e-10f /* 2^-31 */, &s,
                      &c);
            turned[of][j] = make_float2(c * p.factor, s * p.factor);
        }
    }
    __syncthreads();
    if (!there || position[t] < 0) return;
    if (!dbg_check(end <= heads && high + 8 <= p.rot, p.status)) return;
    float c[8], s[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float2 cs = turned[t][8 * u + e];
        c[e] = cs.x;
        s[e] = cs.y;
    }
    for (int h = begin + h0; h < end; h += kAhead * side) {
        if (h != begin + h0) load(h);
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (h + k * side < end) {
                uint32_t x[4] = {a[k].x, a[k].y, a[k].z, a[k].w}, y[4] = {b[k].x, b[k].y, b[k].z, b[k].w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float x0 = bf16_low(x[i]), x1 = bf16_high(x[i]);
                    const float y0 = bf16_low(y[i]), y1 = bf16_high(y[i]);
                    if constexpr (PAIRS) {
                        x[i] = pack_bf16(x0 * c[i] - x1 * s[i], x0 * s[i] + x1 * c[i]);
                        y[i] = pack_bf16(y0 * c[4 + i] - y1 * s[4 + i], y0 * s[4 + i] + y1 * c[4 + i]);
                    } else {
                        const int e = 2 * i;
                        x[i] = pack_bf16(x0 * c[e] - y0 * s[e], x1 * c[e + 1] - y1 * s[e + 1]);
                        y[i] = pack_bf16(x0 * s[e] + y0 * c[e], x1 * s[e + 1] + y1 * c[e + 1]);
                    }
                }
                uint16_t* const head = row + (h + k * side) * p.d;
                *reinterpret_cast<uint4*>(head + low) = make_uint4(x[0], x[1], x[2], x[3]);
                *reinterpret_cast<uint4*>(head + high) = make_uint4(y[0], y[1], y[2], y[3]);
            }
    }
}

}  // namespace

cudaError_t launch_rotary(const KvView* cache, const RotaryParams& p, int sm_count, cudaStream_t stream) {
    // Tokens to a CTA while there are CTAs for every SM several times over; else heads are split
    // until there are, down to one unit for a thread.
    const int heads = p.H + p.kv_heads, side = kThreads / (p.rot / 16);
    const int64_t want = 8 * static_cast<int64_t>(sm_count);
    int tokens = 1;
    while (tokens < kTokens && p.M / (2 * tokens) >= want) tokens *= 2;
    const int64_t x = (static_cast<int64_t>(p.M) + tokens - 1) / tokens;
    int y = 1;
    while (y < (heads + side - 1) / side && x * y < want) ++y;
    const int per = (heads + y - 1) / y;
    y = (heads + per - 1) / per;
    const KvView none = {};
    auto kernel = cache != nullptr ? (p.pairs ? rotary_kernel<true, true> : rotary_kernel<false, true>)
                                   : (p.pairs ? rotary_kernel<true, false> : rotary_kernel<false, false>);
    return launch_overlapped(kernel, dim3(static_cast<unsigned>(x), static_cast<unsigned>(y)), kThreads, 0, stream,
                             cache != nullptr ? *cache : none, p, tokens, per);
}

}  // namespace w4a16
