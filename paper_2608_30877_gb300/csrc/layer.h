// Internal interface of the operators around the linears of a decoder layer: what layer_api.cu and
// kv_api.cu hand to the kernel translation units.  Not part of the public ABI.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <cstdint>

#include "kv.h"

namespace w4a16 {

// The residual stream's update and norm (norm.cu).  Null pointers: absent.
struct NormParams {
    const void* residual;         // [M, D] bf16 or fp32
    const uint16_t* block;        // bf16 [M, D]
    const uint16_t* gate;         // bf16 rows of D, gate_stride apart (0: one for all rows)
    const uint16_t* post_weight;  // bf16 [D], and so on
    const uint16_t* post_bias;
    const uint16_t* weight;
    const uint16_t* bias;
    void* residual_out;           // as residual
    uint16_t* out;                // bf16 [M, D]
    int64_t gate_stride;
    int M, D;
    float residual_scale, eps, weight_offset;
    bool layer;                   // layer norms, else RMS norms
    int* status;
    uint64_t wait_ns;
};
constexpr int kNormMaxWidth = 49152;
cudaError_t launch_residual_norm(const NormParams& p, bool fp32, int sm_count, cudaStream_t stream);

// Rotary positions (rotary.cu).
struct RotaryParams {
    uint16_t* qkv;             // bf16 [M, (H + 2 kv_heads) * d]
    const int32_t* seq_start;  // [nseq + 1]; null: one row for each sequence
    const int32_t* first;      // [nseq]: a sequence's first position (null: 0), or its slot of the cache
    const uint64_t* turns;     // [rot / 2] turns per token, times 2^64
    int* status;
    int M, nseq, H, kv_heads, d, rot;
    float factor;
    bool pairs;                // (2i, 2i + 1), else (i, i + rot / 2)
};
constexpr int kRotaryMaxDim = 256;
cudaError_t launch_rotary(const KvView* cache, const RotaryParams& p, int sm_count, cudaStream_t stream);

// Log probabilities (logprobs.cu).
struct LogProbsParams {
    const void* logits;      // [M] rows of V, stride apart, bf16 or fp32
    const int32_t* targets;  // [M], or null
    float* logp;             // [M], with targets
    float* entropy;          // [M], or null
    int32_t* index;          // [M, k]
    float* score;            // [M, k]
    int* status;
    int64_t stride;
    int M, V, k;
};
constexpr int kLogProbsMaxK = 64;
constexpr int kLogProbsMaxV = 1 << 20;
cudaError_t launch_log_probs(const LogProbsParams& p, bool bf16, int sm_count, cudaStream_t stream);

// Low-rank adapters beside a shared projection (adapters.cu).
struct AdapterParams {
    const uint16_t* x;         // bf16 [M, K]
    const uint16_t* a;         // bf16 [pool, R, K]
    const uint16_t* b;         // bf16 [pool, N, R]
    const float* scale;        // [pool]
    const int32_t* seq_start;  // [nseq + 1]; null: one row for each sequence
    const int32_t* ids;        // [nseq]
    const uint16_t* base;      // bf16 [M, N]
    uint16_t* out;             // bf16 [M, N]; may be base
    uint16_t* t;               // workspace: scale (x A^T), 16 bits each [M, R] (adapters.cu)
    int* status;
    int M, N, K, R, pool, nseq;
    uint64_t wait_ns;
};
constexpr int kAdapterMaxRank = 64;
int64_t adapters_workspace_bytes(int64_t M, int64_t R);
cudaError_t launch_adapters(const AdapterParams& p, int sm_count, cudaStream_t stream);

}  // namespace w4a16
