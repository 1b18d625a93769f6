// Log probabilities of given tokens, entropy and the best alternatives from a head's logits, which are
// read once.  In base 2, with y = x log2(e) - m for a whole row's m near its largest:
//   log2 p = y - log2 s,  s = sum 2^y;   H = (log2 s - (sum 2^y y) / s) ln 2;
// both terms of H are positive, so nothing cancels, and y is one multiply-add whose rounding of
// m is the same for every logit.  Each thread keeps m, s and the other sum of its part of the row, raised
// to a new m once for 32 (fp32: 16) logits; the parts are joined in a fixed order.  Few rows are split over
// a cluster of CTAs and joined in its first one.  Logits below -2^17 count as that (2^y y = 0, not NaN, for
// -infinity); a row of nothing above -124000, or with one past 726000, is summed again by the formula in natural
// logarithms.
//
// The k largest: the same pass notes the largest logit of each group of neighbours (up to 1024
// groups).  With t the k-th largest of those, all of the k largest logits are among the groups above
// t and the first of those at t, k groups in all: any other group's logits come after k of theirs.
// Only these groups are read again (k * 512 bytes of a row), their logits from t on are collected
// and ranked by counting.  t is searched in the upper half of the keys' bits; what has the same upper half is
// collected as well, unless it is a lot.  Where too many pass, t is raised to the k-th largest logit by
// bisection; where too many are equal to it, they are taken in order.
//
// Bound by HBM where a row is whole: 4099 rows of 131072 in bf16 168 us (6.4 TB/s; 206 with an exponential, two
// comparisons and three sums of its own for each logit, in natural logarithms).  The alternatives cost instructions
// (a warp's maximum for 512 bytes) and the way from the groups to the list, 4 to 8 us a row of which
// four rows an SM overlap: 20 of them 213 us, 64 251; 513 rows of 100003 fp32 logits with 64 47 us.  One row
// with 20: 9 us on a cluster of 8 CTAs.
#include <cuda_runtime.h>
#include <cstdint>
#include <type_traits>

#include "kv.h"
#include "layer.h"
#include "ptx.cuh"

namespace w4a16 {

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kGroups = 1024;     // of a row, at most
constexpr int kCandidates = 1024; // above t, and as many equal to it
constexpr int kMaxCluster = 8;
constexpr int kAhead = 4;         // 16-byte units that a lane has under way
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// Keys whose unsigned order is that of the logits (-0 before +0), a NaN below all numbers.
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t u = __float_as_uint(x);
    if (x != x) return 0u;
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) {
    if (key == 0u) return __uint_as_float(0x7FFFFFFFu);
    return __uint_as_float((key & 0x80000000u) ? key & 0x7FFFFFFFu : ~key);
}

__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ uint4 load_once(const void* p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "l"(p)
                 : "memory");
    return v;
}

// Logits below count as this: small enough that m's rounding is far below one (a thread may see masked logits
// alone, of any size), and a power of two, whose own m is exact.
constexpr float kLeast = -131072.0f;
constexpr uint32_t kLeast2 = 0xC800C800u;  // two of it in bf16
// m of rows that the base-2 form holds: what counts as kLeast has no weight there
constexpr float kFrom = -180000.0f, kTo = 1048576.0f;

// Two fp32 in one register pair.
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
// The larger; a number beats a NaN / a NaN stays one.
__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ uint32_t max_nan_bf16x2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ float max_nan(float a, float b) {
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}

// The largest number of a warp's (a NaN where none is one).
__device__ __forceinline__ float warp_max(float x) {
    float d;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(d) : "f"(x));
    return d;
}

// sum 2^y and sum 2^y y for y = x log2(e) - m.
struct Sums {
    float m, s, t;

    __device__ __forceinline__ void raise(float to) {
        const float y = m - to, f = exp2_approx(y);
        t = f * fmaf(s, y, t);
        s *= f;
        m = to;
    }
};

// Sums of several threads: of the one with the largest logit as it has them, and of the others apart, so that
// what is far smaller is not lost in a sum near one.
struct Joined {
    float m, big, big_t, s, t;
    int owner;

    __device__ __forceinline__ void join(Joined o) {
        if (o.m > m || (o.m == m && o.owner < owner)) {  // (the same on both sides of an exchange)
            const Joined mine = *this;
            *this = o;
            o = mine;
        }
        const float y = o.m - m, f = exp2_approx(y), n = o.big + o.s;
        s = fmaf(f, n, s);
        t = fmaf(f, fmaf(n, y, o.big_t + o.t), t);
    }
};

// A row in 16-byte units of the memory it is in: unit u has the columns from u * N - shift on.
template <bool BF16>
struct RowOf {
    static constexpr int N = BF16 ? 8 : 4;  // columns of a unit
    using T = typename std::conditional<BF16, uint16_t, float>::type;
    const T* row;
    int V, shift, units;

    __device__ __forceinline__ float at(int c) const {
        if constexpr (BF16) return __uint_as_float(static_cast<uint32_t>(row[c]) << 16);
        else return row[c];
    }
    __device__ __forceinline__ bool whole(int u) const {
        const int c = u * N - shift;
        return c >= 0 && c + N <= V;
    }
    // The unit's columns; `absent` where the row has none.
    __device__ __forceinline__ void load_part(int u, float absent, float (&x)[N]) const {
        const int c = u * N - shift;
#pragma unroll
        for (int e = 0; e < N; ++e)
            x[e] = static_cast<unsigned>(c + e) < static_cast<unsigned>(V) ? at(c + e) : absent;
    }
    __device__ __forceinline__ const void* unit(int u) const { return row + (u * N - shift); }
    static __device__ __forceinline__ void unpack(const uint32_t (&w)[4], float (&x)[N]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (BF16) {
                x[2 * i] = __uint_as_float(w[i] << 16);
                x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
            } else {
                x[i] = __uint_as_float(w[i]);
            }
        }
    }
    // The largest of a unit as it is in memory (a NaN where all are), and its columns from kLeast on.
    static __device__ __forceinline__ float largest(const uint32_t (&w)[4]) {
        if constexpr (BF16) {
            const uint32_t v = max_bf16x2(max_bf16x2(w[0], w[1]), max_bf16x2(w[2], w[3]));
            return fmaxf(__uint_as_float(v << 16), __uint_as_float(v & 0xFFFF0000u));
        } else {
            return fmaxf(fmaxf(__uint_as_float(w[0]), __uint_as_float(w[1])),
                         fmaxf(__uint_as_float(w[2]), __uint_as_float(w[3])));
        }
    }
    static __device__ __forceinline__ void from_least(uint32_t (&w)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            w[i] = BF16 ? max_nan_bf16x2(w[i], kLeast2) : __float_as_uint(max_nan(__uint_as_float(w[i]), kLeast));
    }
};

struct Shared {
    uint32_t group_key[kGroups];
    unsigned long long above[kCandidates];  // key << 32 | ~column
    unsigned long long equal[kCandidates];
    int selected[kGroups];                  // groups, ascending
    Joined warp_sums[kWarps], cta_sums[kMaxCluster];
    float refined[kWarps][3];
    int counts[32], digits[4][256], found[3];
    uint32_t threshold;
    int low;  // bits that the threshold leaves out
    int num_selected, num_above, num_equal, count;
};


// f(column, key) for the logits of the selected groups from key `least` on, and for NaNs.
template <bool BF16, typename F>
__device__ __forceinline__ void each_selected(const Shared& sh, const RowOf<BF16>& r, int shift, uint32_t least, const F& f) {
    constexpr int kTogether = 4, N = RowOf<BF16>::N;
    const int total = sh.num_selected << shift;
    const float bound = value_of(least);  // (0: a NaN, below which nothing is)
    for (int i0 = threadIdx.x; i0 < total; i0 += kThreads * kTogether) {
        uint4 v[kTogether];
        int unit[kTogether];
#pragma unroll
        for (int j = 0; j < kTogether; ++j) {
            const int i = i0 + j * kThreads;
            unit[j] = i < total ? (sh.selected[i >> shift] << shift) + (i & ((1 << shift) - 1)) : r.units;
            if (r.whole(unit[j])) v[j] = __ldg(static_cast<const uint4*>(r.unit(unit[j])));
        }
#pragma unroll
        for (int j = 0; j < kTogether; ++j) {
            const int c0 = unit[j] * N - r.shift;
            float x[N];
            uint32_t hits = 0;
            if (r.whole(unit[j])) {
                const uint32_t w[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
                r.unpack(w, x);
#pragma unroll
                for (int e = 0; e < N; ++e) hits |= x[e] < bound ? 0u : 1u << e;
            } else if (unit[j] < r.units) {
                r.load_part(unit[j], 0.0f, x);
#pragma unroll
                for (int e = 0; e < N; ++e)
                    hits |= static_cast<unsigned>(c0 + e) >= static_cast<unsigned>(r.V) || x[e] < bound ? 0u : 1u << e;
            }
            // (few: not worth code for each of the columns)
            for (; hits != 0; hits &= hits - 1) {
                const int e = __ffs(hits) - 1;
                float y = x[0];
#pragma unroll
                for (int i = 1; i < N; ++i) y = e == i ? x[i] : y;
                f(c0 + e, key_of(y));
            }
        }
    }
}

// The selected groups' logits whose keys without their low `low` bits are above t, and equal to it.  All
// threads.
template <bool BF16>
__device__ __noinline__ void collect(Shared& sh, const RowOf<BF16>& r, int shift, uint32_t t, int low) {
    if (threadIdx.x == 0) sh.num_above = sh.num_equal = 0;
    __syncthreads();
    each_selected<BF16>(sh, r, shift, t << low, [&](int c, uint32_t key) {
        const uint32_t q = key >> low;
        if (q < t) return;
        int* const n = q > t ? &sh.num_above : &sh.num_equal;
        unsigned long long* const list = q > t ? sh.above : sh.equal;
        const int at = atomicAdd(n, 1);
        if (at < kCandidates) list[at] = (static_cast<unsigned long long>(key) << 32) | ~static_cast<uint32_t>(c);
    });
    __syncthreads();
}

// The `need` ones of key t of the lowest columns, by one warp.
template <bool BF16>
__device__ __noinline__ void collect_in_order(Shared& sh, const RowOf<BF16>& r, int shift, uint32_t t, int low, int need) {
    constexpr int N = RowOf<BF16>::N;
    const int lane = threadIdx.x;
    const int total = sh.num_selected << shift;
    int found = 0;
    for (int i0 = 0; i0 < total && found < need; i0 += 32) {
        const int i = i0 + lane;
        const int u = i < total ? (sh.selected[i >> shift] << shift) + (i & ((1 << shift) - 1)) : r.units;
        float x[N];
        uint32_t hit = 0;
        if (u < r.units) {
            r.load_part(u, 0.0f, x);
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (static_cast<unsigned>(u * N - r.shift + e) < static_cast<unsigned>(r.V) && key_of(x[e]) >> low == t)
                    hit |= 1u << e;
        }
        int before = __popc(hit);
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, before, o);
            if (lane >= o) before += y;
        }
        const int all = __shfl_sync(0xffffffffu, before, 31);
        before += found - __popc(hit);
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (hit >> e & 1u) {
                if (before < need)
                    sh.equal[before] = (static_cast<unsigned long long>(key_of(x[e])) << 32) |
                                       ~static_cast<uint32_t>(u * N - r.shift + e);
                ++before;
            }
        found += all;
    }
    __syncwarp();
    if (lane == 0) sh.num_equal = found < need ? found : need;
}

// The groups to read again: t (without the keys' low bits), and the list.  All threads; a thread has the
// groups of its number, that plus 256, ...
template <bool BF16>
__device__ __forceinline__ void select_groups(Shared& sh, int groups, int k) {
    constexpr int kMine = kGroups / kThreads;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, tid = threadIdx.x;
    uint32_t key[kMine];
#pragma unroll
    for (int j = 0; j < kMine; ++j) key[j] = sh.group_key[tid + kThreads * j];
    sh.digits[0][tid] = sh.digits[1][tid] = sh.digits[2][tid] = sh.digits[3][tid] = 0;
    __syncthreads();
    // the largest t that k groups reach, eight bits at a time: the digits of the groups that have t's bits so
    // far are counted, and one warp adds the counts up from the top
    int low = 32, above = 0, equal = 0;  // above: groups past t's bits so far
    uint32_t t = 0;
    while (true) {
        low -= 8;
        int* const digits = sh.digits[low >> 3];
#pragma unroll
        for (int j = 0; j < kMine; ++j) {
            if (kThreads * j >= groups) break;
            // (one addition for a warp's equal digits: the first ones are nearly all the same)
            const bool in = tid + kThreads * j < groups && (low == 24 || key[j] >> (low + 8) == t);
            const uint32_t who = __ballot_sync(0xffffffffu, in), digit = key[j] >> low & 255u;
            if (in) {
                const uint32_t same = __match_any_sync(who, digit);
                if (lane == __ffs(same) - 1) atomicAdd(&digits[digit], __popc(same));
            }
        }
        __syncthreads();
        if (warp == 0) {  // lane l has the digits 255 - 8 l and below
            int n[8], sum = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                n[i] = digits[255 - 8 * lane - i];
                sum += n[i];
            }
            int upto = sum;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, upto, o);
                if (lane >= o) upto += y;
            }
            const uint32_t reach = __ballot_sync(0xffffffffu, above + upto >= k);
            // (fewer than k groups: all of them, from digit 0)
            if (lane == (reach != 0 ? __ffs(reach) - 1 : 31)) {
                int digit = 255 - 8 * lane, before = above + upto - sum, here = n[0];
#pragma unroll
                for (int i = 0; i < 7; ++i)
                    if (digit == 255 - 8 * lane - i && before + n[i] < k) {
                        before += n[i];
                        --digit;
                        here = n[i + 1];
                    }
                sh.found[0] = digit;
                sh.found[1] = before;
                sh.found[2] = here;
            }
        }
        __syncthreads();
        t = t << 8 | static_cast<uint32_t>(sh.found[0]);
        above = sh.found[1];
        equal = sh.found[2];
        // (the low half of a bf16's key follows from its sign)
        if (low == 0 || (low == 16 && (BF16 || above + equal <= k + 32))) break;
    }
    // the list, ascending; of the groups at t the first ones, where t is a whole key
    const int take = BF16 || low == 0 ? k - above : equal;
#pragma unroll
    for (int j = 0; j < kMine; ++j) {
        const bool there = tid + kThreads * j < groups;
        const uint32_t more = __ballot_sync(0xffffffffu, there && key[j] >> low > t);
        const uint32_t same = __ballot_sync(0xffffffffu, there && key[j] >> low == t);
        if (lane == 0) sh.counts[j * kWarps + warp] = __popc(more) | __popc(same) << 16;
    }
    __syncthreads();
    static_assert(kMine * kWarps == 32, "a count for each lane");
    int upto = sh.counts[lane];
    const int own = upto;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += y;
    }
    const int before = upto - own;  // of the groups before the lane's 32: above t, and 2^16 times those at it
#pragma unroll
    for (int j = 0; j < kMine; ++j) {
        if (kThreads * j >= groups) break;
        const int b = __shfl_sync(0xffffffffu, before, j * kWarps + warp), same_before = b >> 16;
        const bool there = tid + kThreads * j < groups;
        const uint32_t under = (1u << lane) - 1u;
        const uint32_t same = __ballot_sync(0xffffffffu, there && key[j] >> low == t);
        const bool mine = there && (key[j] >> low > t || (key[j] >> low == t && same_before + __popc(same & under) < take));
        const uint32_t taken = __ballot_sync(0xffffffffu, mine);
        if (mine) sh.selected[(b & 0xFFFF) + min(same_before, max(take, 0)) + __popc(taken & under)] = tid + kThreads * j;
    }
    if (tid == 0) {
        sh.num_selected = min(above + max(take, 0), groups);
        sh.threshold = t;
        sh.low = low;
    }
}

// The k largest of the row, from the groups' keys.  All threads of one CTA.  value(x): x's log probability.
template <bool BF16, typename F>
__device__ __forceinline__ void top(Shared& sh, const RowOf<BF16>& r, int shift, int groups, int k, const F& value,
                                    int32_t* index, float* score, int* status) {
    const int lane = threadIdx.x & 31;
    select_groups<BF16>(sh, groups, k);
    __syncthreads();
    uint32_t t = sh.threshold;
    int low = sh.low;
    collect<BF16>(sh, r, shift, t, low);
    if (sh.num_above > kCandidates || (sh.num_equal > kCandidates && low != 0 && !BF16)) {
        low = BF16 ? 16 : 0;
        t = 0;
        for (uint32_t bit = BF16 ? 1u << 15 : 1u << 31; bit != 0; bit >>= 1) {
            if (threadIdx.x == 0) sh.count = 0;
            __syncthreads();
            int n = 0;
            each_selected<BF16>(sh, r, shift, (t | bit) << low, [&](int, uint32_t key) { n += key >> low >= (t | bit); });
            n = __reduce_add_sync(0xffffffffu, n);
            if (lane == 0 && n > 0) atomicAdd(&sh.count, n);
            __syncthreads();
            if (sh.count >= k) t |= bit;
            __syncthreads();
        }
        collect<BF16>(sh, r, shift, t, low);
    }
    if (sh.num_equal > kCandidates) {
        if (threadIdx.x < 32) collect_in_order<BF16>(sh, r, shift, t, low, k);
        __syncthreads();
    }
    // four threads count for a candidate
    const int na = sh.num_above, n = na + sh.num_equal;
    for (int i0 = 0; i0 < n; i0 += kThreads / 4) {
        const int i = i0 + static_cast<int>(threadIdx.x) / 4;
        const unsigned long long mine = i < na ? sh.above[i] : i < n ? sh.equal[i - na] : 0;
        int rank = 0;
        if (i < n) {
            for (int j = threadIdx.x & 3; j < na; j += 4) rank += sh.above[j] > mine;
            for (int j = threadIdx.x & 3; j < n - na; j += 4) rank += sh.equal[j] > mine;
        }
        rank += __shfl_xor_sync(0xffffffffu, rank, 1);
        rank += __shfl_xor_sync(0xffffffffu, rank, 2);
        const uint32_t column = ~static_cast<uint32_t>(mine);
        if (i < n && rank < k && (threadIdx.x & 3) == 0 && dbg_check(column < static_cast<uint32_t>(r.V), status)) {
            index[rank] = static_cast<int32_t>(column);
            score[rank] = value(value_of(static_cast<uint32_t>(mine >> 32)));
        }
    }
}

// A row's sums about its largest number m, by e^(x - m), for rows that the base-2 form does not hold (m -infinity:
// no number above that).  All threads of one CTA.
template <bool BF16>
__device__ __noinline__ Sums sums_again(Shared& sh, const RowOf<BF16>& r) {
    constexpr int N = RowOf<BF16>::N;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    Sums all{-INFINITY, 0.0f, 0.0f};
    for (int pass = 0; pass < 2; ++pass) {
        Sums mine{-INFINITY, 0.0f, 0.0f};
        const float m = all.m == -INFINITY ? 0.0f : all.m;
        for (int u = threadIdx.x; u < r.units; u += kThreads) {
            float x[N];
            r.load_part(u, -INFINITY, x);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                if (pass == 0) {
                    mine.m = fmaxf(mine.m, x[e]);
                } else {
                    const float y = (x[e] - m) * kLog2e, q = exp2_approx(y);
                    mine.s += q;
                    mine.t = fmaf(q, fmaxf(y, -1e4f), mine.t);
                }
            }
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            mine.m = fmaxf(mine.m, __shfl_xor_sync(0xffffffffu, mine.m, o));
            mine.s += __shfl_xor_sync(0xffffffffu, mine.s, o);
            mine.t += __shfl_xor_sync(0xffffffffu, mine.t, o);
        }
        __syncthreads();
        if (lane == 0) {
            sh.refined[warp][0] = mine.m;
            sh.refined[warp][1] = mine.s;
            sh.refined[warp][2] = mine.t;
        }
        __syncthreads();
        for (int w = 0; w < kWarps; ++w) {
            if (pass == 0) {
                all.m = fmaxf(all.m, sh.refined[w][0]);
            } else {
                all.s += sh.refined[w][1];
                all.t += sh.refined[w][2];
            }
        }
    }
    return all;
}

// One logit stands far above the others: what its thread added to a sum that has it lost its low bits.  That
// thread's logits are added up again without it, by all threads of one CTA; d: the y of that logit, which m's
// rounding keeps from being 0.
template <bool BF16>
__device__ __noinline__ Sums sums_without_largest(Shared& sh, const RowOf<BF16>& r, const Joined& all, int ctas, float* d) {
    constexpr int N = RowOf<BF16>::N;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int from = (all.owner >> 5) * 32 * kAhead + (all.owner & 31), step = ctas * kThreads * kAhead;
    float s = 0.0f, t = 0.0f, top = -INFINITY;
    for (int i = threadIdx.x;; i += kThreads) {
        const int64_t u = from + 32 * (i % kAhead) + static_cast<int64_t>(i / kAhead) * step;
        if (u - 32 * (i % kAhead) >= r.units) break;
        float x[N];
        r.load_part(static_cast<int>(u < r.units ? u : r.units), -INFINITY, x);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float y = fmaf(fmaxf(x[e], kLeast), kLog2e, -all.m);
            if (y > -1.0f) {  // (the others are below 2^-4)
                top = y;
            } else {
                const float q = exp2_approx(y);
                s += q;
                t = fmaf(q, y, t);
            }
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        s += __shfl_xor_sync(0xffffffffu, s, o);
        t += __shfl_xor_sync(0xffffffffu, t, o);
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    }
    __syncthreads();
    if (lane == 0) {
        sh.refined[warp][0] = s;
        sh.refined[warp][1] = t;
        sh.refined[warp][2] = top;
    }
    __syncthreads();
    s = all.s;
    t = all.t;
    top = sh.refined[0][2];
    for (int w = 0; w < kWarps; ++w) {
        s += sh.refined[w][0];
        t += sh.refined[w][1];
        top = fmaxf(top, sh.refined[w][2]);
    }
    // from m to that logit
    const float f = exp2_approx(-top);
    *d = top;
    return {0.0f, s * f, fmaf(-top, s, t) * f};
}

template <bool BF16, bool TOP>
__global__ void __launch_bounds__(kThreads, 4) log_probs_kernel(const LogProbsParams p, const int shift, const int ctas) {
    constexpr int N = RowOf<BF16>::N;
    __shared__ Shared sh;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int rank = ctas > 1 ? static_cast<int>(cluster_ctarank()) : 0;
    const int64_t row = blockIdx.x / ctas;
    RowOf<BF16> r;
    r.row = static_cast<const typename RowOf<BF16>::T*>(p.logits) + row * p.stride;
    r.V = p.V;
    r.shift = static_cast<int>(reinterpret_cast<uintptr_t>(r.row) / sizeof(*r.row)) & (N - 1);
    r.units = (p.V + r.shift + N - 1) / N;
    const int groups = TOP ? (r.units + (1 << shift) - 1) >> shift : 0;
    if constexpr (TOP)
        for (int i = threadIdx.x; i < kGroups; i += kThreads) sh.group_key[i] = 0;
    grid_launch_dependents();
    grid_wait();
    __syncthreads();
    if (ctas > 1) cluster_sync();  // (the first CTA's keys are ready for the others')
    Sums mine{kLeast * kLog2e, 0.0f, 0.0f};
    // a warp's 128 units at a time, the warps of all CTAs side by side
    const int ends = r.shift == 0 && p.V % N == 0 ? 0 : 1;  // units that may be in part the row's
    for (int u0 = (rank * kWarps + warp) * 32 * kAhead; u0 < r.units; u0 += ctas * kThreads * kAhead) {
        uint32_t w[kAhead][4];
        float most[kAhead];
        if (u0 >= ends && u0 + 32 * kAhead <= r.units - ends) {
            const uint4* const from = static_cast<const uint4*>(r.unit(u0 + lane));
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const uint4 v = load_once(from + 32 * i);
                w[i][0] = v.x, w[i][1] = v.y, w[i][2] = v.z, w[i][3] = v.w;
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) most[i] = r.largest(w[i]);
        } else {
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int u = u0 + 32 * i + lane;
                if (r.whole(u)) {
                    const uint4 v = load_once(r.unit(u));
                    w[i][0] = v.x, w[i][1] = v.y, w[i][2] = v.z, w[i][3] = v.w;
                    most[i] = r.largest(w[i]);
                } else {
                    float x[N];
                    r.load_part(u, -INFINITY, x);
                    most[i] = __uint_as_float(0x7FFFFFFFu);  // no number
#pragma unroll
                    for (int e = 0; e < N; ++e)
                        if (static_cast<unsigned>(u * N - r.shift + e) < static_cast<unsigned>(r.V))
                            most[i] = fmaxf(most[i], x[e]);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        w[i][j] = BF16 ? (__float_as_uint(x[(BF16 ? 2 : 1) * j]) >> 16) |
                                             (__float_as_uint(x[BF16 ? 2 * j + 1 : j]) & 0xFFFF0000u)
                                       : __float_as_uint(x[j]);
                }
            }
        }
        float high = most[0];
#pragma unroll
        for (int i = 1; i < kAhead; ++i) high = fmaxf(high, most[i]);
        high *= kLog2e;
        if (high > mine.m) mine.raise(high);
        const uint64_t log2e = pair(kLog2e, kLog2e), minus = pair(-mine.m, -mine.m);
        uint64_t s2 = pair(mine.s, 0.0f), t2 = pair(mine.t, 0.0f);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            float x[N];
            r.from_least(w[i]);
            r.unpack(w[i], x);
#pragma unroll
            for (int e = 0; e < N; e += 2) {
                const uint64_t y = fma2(pair(x[e], x[e + 1]), log2e, minus);
                const float2 v = both(y);
                const uint64_t q = pair(exp2_approx(v.x), exp2_approx(v.y));
                s2 = add2(s2, q);
                t2 = fma2(q, y, t2);
            }
        }
        mine.s = both(s2).x + both(s2).y;
        mine.t = both(t2).x + both(t2).y;
        if constexpr (TOP) {
            auto note = [&](int group, uint32_t key) {
                if (rank == 0) {
                    atomicMax(&sh.group_key[group], key);
                } else {
                    const uint32_t to = mapa_shared(smem_u32(&sh.group_key[group]), 0);
                    asm volatile("red.relaxed.cluster.shared::cluster.max.u32 [%0], %1;" ::"r"(to), "r"(key) : "memory");
                }
            };
            if (shift >= 5) {  // a lane's number is one of the warp's four
                float v = 0.0f;
#pragma unroll
                for (int i = 0; i < kAhead; ++i) {
                    const float all = warp_max(most[i]);
                    if (lane == i) v = all;
                }
                const int u = u0 + 32 * lane;
                if (lane < kAhead && u < r.units) {
                    if (shift == 5 && rank == 0) sh.group_key[u >> 5] = key_of(v);  // (no other warp's)
                    else note(u >> shift, key_of(v));
                }
            } else {
#pragma unroll
                for (int i = 0; i < kAhead; ++i) {
                    uint32_t key = key_of(most[i]);
                    for (int o = 1; o < 1 << shift; o <<= 1) key = max(key, __shfl_xor_sync(0xffffffffu, key, o));
                    const int u = u0 + 32 * i + lane;
                    if ((u & ((1 << shift) - 1)) == 0 && u < r.units) note(u >> shift, key);
                }
            }
        }
    }
    Joined all{mine.m, mine.s, mine.t, 0.0f, 0.0f, (rank * kWarps + warp) * 32 + lane};
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        Joined other;
        other.m = __shfl_xor_sync(0xffffffffu, all.m, o);
        other.big = __shfl_xor_sync(0xffffffffu, all.big, o);
        other.big_t = __shfl_xor_sync(0xffffffffu, all.big_t, o);
        other.s = __shfl_xor_sync(0xffffffffu, all.s, o);
        other.t = __shfl_xor_sync(0xffffffffu, all.t, o);
        other.owner = __shfl_xor_sync(0xffffffffu, all.owner, o);
        all.join(other);
    }
    if (lane == 0) sh.warp_sums[warp] = all;
    __syncthreads();
    all = sh.warp_sums[0];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) all.join(sh.warp_sums[w]);
    if (ctas > 1) {
        if (threadIdx.x == 0 && rank != 0) {
            const uint32_t to = mapa_shared(smem_u32(&sh.cta_sums[rank]), 0);
            st_shared_cluster_u32(to, __float_as_uint(all.m));
            st_shared_cluster_u32(to + 4, __float_as_uint(all.big));
            st_shared_cluster_u32(to + 8, __float_as_uint(all.big_t));
            st_shared_cluster_u32(to + 12, __float_as_uint(all.s));
            st_shared_cluster_u32(to + 16, __float_as_uint(all.t));
            st_shared_cluster_u32(to + 20, static_cast<uint32_t>(all.owner));
        }
        cluster_sync();
        if (rank != 0) return;
        for (int c = 1; c < ctas; ++c) all.join(sh.cta_sums[c]);
    }
    mine = {all.m, all.big + all.s, all.big_t + all.t};
    const bool again = !(mine.m > kFrom && mine.m < kTo), sure = !again && mine.s < 1.0625f;
    float d = 0.0f;
    if (again) mine = sums_again<BF16>(sh, r);
    if (sure) mine = sums_without_largest<BF16>(sh, r, all, ctas, &d);
    const float m = mine.m, ln_s = sure ? log1pf(mine.s) : log2f(mine.s) * kLn2;  // (m: of `again` alone)
    const bool none = mine.s == 0.0f && !sure;  // every logit -infinity
    // (far below the others, x - lse is x)
    const auto value = [=](float x) {
        if (none) return -INFINITY;
        if (again) return (x - m) - ln_s;
        const float y = fmaf(x, kLog2e, -all.m);
        return (x < -1e37f ? x : sure ? fmaf(y - d, kLn2, -ln_s) : fmaf(y, kLn2, -ln_s)) + 0.0f * mine.s;  // (NaN where s is)
    };
    if (threadIdx.x == 0) {
        if (p.entropy != nullptr)
            p.entropy[row] = none ? 0.0f : sure ? ln_s - kLn2 * mine.t / (1.0f + mine.s) : ln_s - kLn2 * (mine.t / mine.s);
        if (p.targets != nullptr) {
            const int target = p.targets[row];
            float logp = 0.0f;
            if (target >= 0 && target < p.V)
                logp = value(r.at(target));
            else if (target != -1)
                record_status(p.status, 1 /* W4A16_ERR_INVALID_ARG */);
            p.logp[row] = logp;
        }
    }
    if constexpr (TOP) top<BF16>(sh, r, shift, groups, p.k, value, p.index + row * p.k, p.score + row * p.k, p.status);
}

template <bool BF16, bool TOP>
cudaError_t launch(const LogProbsParams& p, int sm_count, cudaStream_t stream) {
    constexpr int N = RowOf<BF16>::N;
    const int units = (p.V + 2 * (N - 1)) / N;  // at most, wherever the row begins
    int shift = 5;
    while (units > kGroups << shift) ++shift;
    // four groups for each alternative at least: what passes the k-th largest of their maxima is then little more than
    // k (2000 rows of 32000 with 20 52 us; with eight for each, which takes groups of half a warp's units, 63)
    while (shift > 0 && units >> shift < 4 * p.k) --shift;
    int ctas = 1;
    while (ctas < kMaxCluster && static_cast<int64_t>(p.M) * ctas * 2 <= 4 * sm_count && ctas * kThreads * kAhead < units)
        ctas *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(p.M) * ctas);
    cfg.blockDim = dim3(kThreads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = static_cast<unsigned>(ctas);
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = ctas > 1 ? 2 : 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, log_probs_kernel<BF16, TOP>, p, shift, ctas);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

cudaError_t launch_log_probs(const LogProbsParams& p, bool bf16, int sm_count, cudaStream_t stream) {
    if (bf16) return p.k > 0 ? launch<true, true>(p, sm_count, stream) : launch<true, false>(p, sm_count, stream);
    return p.k > 0 ? launch<false, true>(p, sm_count, stream) : launch<false, false>(p, sm_count, stream);
}

}  // namespace w4a16
