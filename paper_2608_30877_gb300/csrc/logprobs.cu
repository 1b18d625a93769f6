// Log probabilities of given tokens, entropy and the best alternatives from a head's logits, which are
// read once:
//   lse = m + ln s,  s = sum e^(x - m);   H = ln s - (sum e^(x - m) (x - m)) / s,  m the largest;
// both terms of H are positive, so nothing cancels.  Each thread keeps m, s and the other sum of its
// part of the row (in base 2), raised to a new m once for 32 logits; the parts are joined in a
// fixed order.  Few rows are split over a cluster of CTAs and joined in its first one.
//
// The k largest: the same pass notes the largest logit of each group of neighbours (up to 1024
// groups).  With t the k-th largest of those, all of the k largest logits are among the groups above
// t and the first of those at t, k groups in all: any other group's logits come after k of theirs.
// Only these groups are read again (k * 512 bytes of a row), their logits from t on are collected
// and ranked by counting.  Where too many pass, t is raised to the k-th largest logit by
// bisection; where too many are equal to it, they are taken in order.
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

// sum e^(x - m) and sum e^(x - m) (x - m), in base 2.
struct Sums {
    float m, s, t;

    __device__ __forceinline__ void raise(float to) {
        const float y = m == -INFINITY ? 0.0f : (m - to) * kLog2e;
        const float f = m == -INFINITY ? 0.0f : exp2_approx(y);
        t = f * fmaf(s, fmaxf(y, -1e4f), t);
        s *= f;
        m = to;
    }
    __device__ __forceinline__ void join(Sums o) {
        if (o.m > m) raise(o.m);
        if (o.m < m) o.raise(m);
        s += o.s;
        t += o.t;
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
    static __device__ __forceinline__ void unpack(uint4 v, float (&x)[N]) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
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
};

struct Shared {
    uint32_t group_key[kGroups];
    unsigned long long above[kCandidates];  // key << 32 | ~column
    unsigned long long equal[kCandidates];
    int selected[kGroups];                  // groups, ascending
    Sums warp_sums[kWarps], cta_sums[kMaxCluster];
    uint32_t threshold;
    int num_selected, num_above, num_equal, count;
};

template <bool BF16>
__device__ __forceinline__ uint32_t cut(uint32_t key) {
    // (the low half of a bf16's key follows from its sign)
    return BF16 ? key >> 16 : key;
}

// f(column, key) for the logits of the selected groups.
template <bool BF16, typename F>
__device__ __forceinline__ void each_selected(const Shared& sh, const RowOf<BF16>& r, int shift, const F& f) {
    const int total = sh.num_selected << shift;
    for (int i = threadIdx.x; i < total; i += kThreads) {
        const int u = (sh.selected[i >> shift] << shift) + (i & ((1 << shift) - 1));
        if (u >= r.units) continue;
        float x[RowOf<BF16>::N];
        if (r.whole(u))
            r.unpack(__ldg(reinterpret_cast<const uint4*>(r.row + (u * RowOf<BF16>::N - r.shift))), x);
        else
            r.load_part(u, 0.0f, x);
#pragma unroll
        for (int e = 0; e < RowOf<BF16>::N; ++e) {
            const int c = u * RowOf<BF16>::N - r.shift + e;
            if (static_cast<unsigned>(c) < static_cast<unsigned>(r.V)) f(c, key_of(x[e]));
        }
    }
}

// The selected groups' logits above and at the threshold.  All threads.
template <bool BF16>
__device__ void collect(Shared& sh, const RowOf<BF16>& r, int shift, uint32_t t) {
    if (threadIdx.x == 0) sh.num_above = sh.num_equal = 0;
    __syncthreads();
    each_selected<BF16>(sh, r, shift, [&](int c, uint32_t key) {
        const uint32_t q = cut<BF16>(key);
        if (q < t) return;
        int* const n = q > t ? &sh.num_above : &sh.num_equal;
        unsigned long long* const list = q > t ? sh.above : sh.equal;
        const int at = atomicAdd(n, 1);
        if (at < kCandidates) list[at] = (static_cast<unsigned long long>(key) << 32) | ~static_cast<uint32_t>(c);
    });
    __syncthreads();
}

// The `need` equal ones of the lowest columns, by one warp.
template <bool BF16>
__device__ void collect_in_order(Shared& sh, const RowOf<BF16>& r, int shift, uint32_t t, int need) {
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
                if (static_cast<unsigned>(u * N - r.shift + e) < static_cast<unsigned>(r.V) && cut<BF16>(key_of(x[e])) == t)
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

// The k largest of the row, from the groups' keys.  All threads of one CTA.
template <bool BF16>
__device__ void top(Shared& sh, const RowOf<BF16>& r, int shift, int groups, int k, float m, float ln_s,
                    bool none, int32_t* index, float* score) {
    const int lane = threadIdx.x & 31;
    if (threadIdx.x < 32) {
        uint32_t key[kGroups / 32];
#pragma unroll
        for (int j = 0; j < kGroups / 32; ++j) key[j] = j * 32 < groups ? cut<BF16>(sh.group_key[j * 32 + lane]) : 0u;
        // the largest t that k groups reach
        uint32_t t = 0;
        for (uint32_t bit = BF16 ? 1u << 15 : 1u << 31; bit != 0; bit >>= 1) {
            int n = 0;
#pragma unroll
            for (int j = 0; j < kGroups / 32; ++j)
                if (j * 32 < groups) n += key[j] >= (t | bit);
            if (__reduce_add_sync(0xffffffffu, n) >= k) t |= bit;
        }
        int above = 0;
#pragma unroll
        for (int j = 0; j < kGroups / 32; ++j)
            if (j * 32 < groups) above += key[j] > t;
        int equal = k - __reduce_add_sync(0xffffffffu, above);  // to take
        int n = 0;
#pragma unroll
        for (int j = 0; j < kGroups / 32; ++j) {
            if (j * 32 >= groups) break;
            const bool there = j * 32 + lane < groups;
            const uint32_t same = __ballot_sync(0xffffffffu, there && key[j] == t);
            const bool take = there && (key[j] > t || (key[j] == t && __popc(same & ((1u << lane) - 1u)) < equal));
            const uint32_t taken = __ballot_sync(0xffffffffu, take);
            if (take) sh.selected[n + __popc(taken & ((1u << lane) - 1u))] = j * 32 + lane;
            n += __popc(taken);
            equal -= __popc(same);
        }
        if (lane == 0) {
            sh.num_selected = n;
            sh.threshold = t;
        }
    }
    __syncthreads();
    uint32_t t = sh.threshold;
    collect<BF16>(sh, r, shift, t);
    if (sh.num_above > kCandidates) {
        for (uint32_t bit = BF16 ? 1u << 15 : 1u << 31; bit != 0; bit >>= 1) {
            // (t's own bits are those of a value that k logits reach)
            if (threadIdx.x == 0) sh.count = 0;
            if (bit == (BF16 ? 1u << 15 : 1u << 31)) t = 0;
            __syncthreads();
            int n = 0;
            each_selected<BF16>(sh, r, shift, [&](int, uint32_t key) { n += cut<BF16>(key) >= (t | bit); });
            n = __reduce_add_sync(0xffffffffu, n);
            if (lane == 0 && n > 0) atomicAdd(&sh.count, n);
            __syncthreads();
            if (sh.count >= k) t |= bit;
            __syncthreads();
        }
        collect<BF16>(sh, r, shift, t);
    }
    if (sh.num_equal > kCandidates) {
        if (threadIdx.x < 32) collect_in_order<BF16>(sh, r, shift, t, k);
        __syncthreads();
    }
    const int na = sh.num_above, n = na + sh.num_equal;
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const unsigned long long mine = i < na ? sh.above[i] : sh.equal[i - na];
        int rank = 0;
        for (int j = 0; j < na; ++j) rank += sh.above[j] > mine;
        if (i >= na)
            for (int j = 0; j < n - na; ++j) rank += sh.equal[j] > mine;
        if (rank < k) {
            index[rank] = static_cast<int32_t>(~static_cast<uint32_t>(mine));
            // (without a logit above -infinity no token has a probability)
            score[rank] = none ? -INFINITY : (value_of(static_cast<uint32_t>(mine >> 32)) - m) - ln_s;
        }
    }
}

template <bool BF16, bool TOP>
__global__ void __launch_bounds__(kThreads) log_probs_kernel(const LogProbsParams p, const int shift, const int ctas) {
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
    Sums mine{-INFINITY, 0.0f, 0.0f};
    // a warp's 128 units at a time, the warps of all CTAs side by side
    for (int u0 = (rank * kWarps + warp) * 32 * kAhead; u0 < r.units; u0 += ctas * kThreads * kAhead) {
        float x[kAhead][N], most[kAhead];
        uint4 v[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int u = u0 + 32 * i + lane;
            if (r.whole(u)) v[i] = load_once(r.row + (u * N - r.shift));
        }
        float high = -INFINITY;
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int u = u0 + 32 * i + lane;
            if (r.whole(u)) {
                r.unpack(v[i], x[i]);
                most[i] = x[i][0];
#pragma unroll
                for (int e = 1; e < N; ++e) most[i] = fmaxf(most[i], x[i][e]);
            } else {
                r.load_part(u, -INFINITY, x[i]);
                most[i] = __uint_as_float(0x7FFFFFFFu);  // no number
#pragma unroll
                for (int e = 0; e < N; ++e)
                    if (static_cast<unsigned>(u * N - r.shift + e) < static_cast<unsigned>(r.V))
                        most[i] = fmaxf(most[i], x[i][e]);
            }
            high = fmaxf(high, most[i]);
        }
        if (high > mine.m) mine.raise(high);
        const float m = mine.m == -INFINITY ? 0.0f : mine.m;
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float y = (x[i][e] - m) * kLog2e, q = exp2_approx(y);
                mine.s += q;
                mine.t = fmaf(q, fmaxf(y, -1e4f), mine.t);  // (-infinity: 0 times a number)
            }
        if constexpr (TOP) {
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                uint32_t key = key_of(most[i]);
                if (shift >= 5) {
                    key = __reduce_max_sync(0xffffffffu, key);
                } else {
                    for (int o = 1; o < 1 << shift; o <<= 1) key = max(key, __shfl_xor_sync(0xffffffffu, key, o));
                }
                const int u = u0 + 32 * i + lane;
                if ((u & ((1 << min(shift, 5)) - 1)) == 0 && u < r.units && key != 0) {
                    if (rank == 0) {
                        atomicMax(&sh.group_key[u >> shift], key);
                    } else {
                        const uint32_t to = mapa_shared(smem_u32(&sh.group_key[u >> shift]), 0);
                        asm volatile("red.relaxed.cluster.shared::cluster.max.u32 [%0], %1;" ::"r"(to), "r"(key) : "memory");
                    }
                }
            }
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        Sums other;
        other.m = __shfl_xor_sync(0xffffffffu, mine.m, o);
        other.s = __shfl_xor_sync(0xffffffffu, mine.s, o);
        other.t = __shfl_xor_sync(0xffffffffu, mine.t, o);
        mine.join(other);
    }
    if (lane == 0) sh.warp_sums[warp] = mine;
    __syncthreads();
    mine = sh.warp_sums[0];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) mine.join(sh.warp_sums[w]);
    if (ctas > 1) {
        if (threadIdx.x == 0 && rank != 0) {
            const uint32_t to = mapa_shared(smem_u32(&sh.cta_sums[rank]), 0);
            st_shared_cluster_u32(to, __float_as_uint(mine.m));
            st_shared_cluster_u32(to + 4, __float_as_uint(mine.s));
            st_shared_cluster_u32(to + 8, __float_as_uint(mine.t));
        }
        cluster_sync();
        if (rank != 0) return;
        for (int c = 1; c < ctas; ++c) mine.join(sh.cta_sums[c]);
    }
    const float m = mine.m, ln_s = logf(mine.s);
    const bool none = mine.s == 0.0f;  // every logit -infinity
    if (threadIdx.x == 0) {
        if (p.entropy != nullptr) p.entropy[row] = none ? 0.0f : fmaf(-kLn2, mine.t / mine.s, ln_s);
        if (p.targets != nullptr) {
            const int target = p.targets[row];
            float logp = 0.0f;
            if (target >= 0 && target < p.V)
                logp = none ? -INFINITY : (r.at(target) - m) - ln_s;
            else if (target != -1)
                record_status(p.status, 1 /* W4A16_ERR_INVALID_ARG */);
            p.logp[row] = logp;
        }
    }
    if constexpr (TOP) top<BF16>(sh, r, shift, groups, p.k, m, ln_s, none, p.index + row * p.k, p.score + row * p.k);
}

template <bool BF16, bool TOP>
cudaError_t launch(const LogProbsParams& p, int sm_count, cudaStream_t stream) {
    constexpr int N = RowOf<BF16>::N;
    const int units = (p.V + 2 * (N - 1)) / N;  // at most, wherever the row begins
    int shift = 5;
    while (units > kGroups << shift) ++shift;
    while (shift > 0 && units >> shift < 8 * p.k) --shift;
    int ctas = 1;
    while (ctas < kMaxCluster && static_cast<int64_t>(p.M) * ctas * 2 <= 8 * sm_count && ctas * kThreads * kAhead < units)
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
