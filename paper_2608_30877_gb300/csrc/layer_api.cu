// C ABI of the operators around the linears of a decoder layer (declared in include/w4a16.h):
// argument validation and dispatch.
#include "kv.h"
#include "layer.h"
#include "w4a16.h"

#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

namespace w4a16 {
namespace {

constexpr int64_t kMaxDim = (int64_t{1} << 31) - 1;

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// [p, p + bytes); empty where p is null.
struct Span {
    const void* p;
    int64_t bytes;
};
bool overlaps(const Span& a, const Span& b) {
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(a.p), b0 = reinterpret_cast<uintptr_t>(b.p);
    return a.p != nullptr && b.p != nullptr && a0 < b0 + static_cast<uintptr_t>(b.bytes) &&
           b0 < a0 + static_cast<uintptr_t>(a.bytes);
}

// Every span 16-byte aligned, and none of `out` in another of them or in one of `in`.
template <int NI, int NO>
int check_spans(const Span (&in)[NI], const Span (&out)[NO]) {
    for (const Span& s : in)
        if (!aligned16(s.p)) return W4A16_ERR_ALIGNMENT;
    for (const Span& s : out)
        if (!aligned16(s.p)) return W4A16_ERR_ALIGNMENT;
    for (int i = 0; i < NO; ++i) {
        for (const Span& s : in)
            if (overlaps(out[i], s)) return W4A16_ERR_INVALID_ARG;
        for (int j = 0; j < i; ++j)
            if (overlaps(out[i], out[j])) return W4A16_ERR_INVALID_ARG;
    }
    return W4A16_OK;
}

int status_of(cudaError_t e) { return e == cudaSuccess ? W4A16_OK : W4A16_ERR_CUDA; }

}  // namespace
}  // namespace w4a16

using namespace w4a16;

extern "C" int w4a16_residual_norm(const void* residual, int residual_bits, const void* block_bf16,
                                   const void* gate_bf16, int64_t gate_rows, const void* post_weight_bf16,
                                   const void* post_bias_bf16, const void* weight_bf16, const void* bias_bf16,
                                   int64_t M, int64_t D, int norm, float residual_scale, float eps, float weight_offset,
                                   void* residual_out, void* out_bf16, void* stream) {
    if (residual == nullptr || (residual_out == nullptr && out_bf16 == nullptr)) return W4A16_ERR_INVALID_ARG;
    if (residual_bits != 16 && residual_bits != 32) return W4A16_ERR_INVALID_ARG;
    if (norm != W4A16_NORM_RMS && norm != W4A16_NORM_LAYER) return W4A16_ERR_INVALID_ARG;
    if (M <= 0 || D <= 0 || !(eps >= 1e-12f && eps <= 1.0f)) return W4A16_ERR_INVALID_ARG;
    if (!std::isfinite(residual_scale) || !std::isfinite(weight_offset)) return W4A16_ERR_INVALID_ARG;
    if (block_bf16 == nullptr && (gate_bf16 != nullptr || post_weight_bf16 != nullptr)) return W4A16_ERR_INVALID_ARG;
    if (post_bias_bf16 != nullptr && post_weight_bf16 == nullptr) return W4A16_ERR_INVALID_ARG;
    if (out_bf16 == nullptr && (weight_bf16 != nullptr || bias_bf16 != nullptr)) return W4A16_ERR_INVALID_ARG;
    if (gate_bf16 != nullptr && gate_rows != 1 && gate_rows != M) return W4A16_ERR_INVALID_ARG;
    if (M > kMaxDim || D > kNormMaxWidth) return W4A16_ERR_UNSUPPORTED;
    const int64_t stream_bytes = M * D * (residual_bits / 8);
    const Span in[6] = {{block_bf16, M * D * 2},      {gate_bf16, gate_bf16 != nullptr ? gate_rows * D * 2 : 0},
                        {post_weight_bf16, D * 2},    {post_bias_bf16, D * 2},
                        {weight_bf16, D * 2},         {bias_bf16, D * 2}};
    const Span outs[2] = {{residual_out, stream_bytes}, {out_bf16, M * D * 2}};
    const int rc = check_spans(in, outs);
    if (rc != W4A16_OK) return rc;
    if (!aligned16(residual)) return W4A16_ERR_ALIGNMENT;
    const Span from{residual, stream_bytes};
    if ((residual_out != residual && overlaps(from, outs[0])) || overlaps(from, outs[1])) return W4A16_ERR_INVALID_ARG;
    LibraryState st;
    const int state = library_state(&st);
    if (state != W4A16_OK) return state;
    NormParams p;
    p.residual = residual;
    p.block = static_cast<const uint16_t*>(block_bf16);
    p.gate = static_cast<const uint16_t*>(gate_bf16);
    p.post_weight = static_cast<const uint16_t*>(post_weight_bf16);
    p.post_bias = static_cast<const uint16_t*>(post_bias_bf16);
    p.weight = static_cast<const uint16_t*>(weight_bf16);
    p.bias = static_cast<const uint16_t*>(bias_bf16);
    p.residual_out = residual_out;
    p.out = static_cast<uint16_t*>(out_bf16);
    p.gate_stride = gate_rows == 1 ? 0 : D;
    p.M = static_cast<int>(M);
    p.D = static_cast<int>(D);
    p.residual_scale = residual_scale;
    p.eps = eps;
    p.weight_offset = weight_offset;
    p.layer = norm == W4A16_NORM_LAYER;
    p.status = st.status;
    p.wait_ns = wait_limit_ns();
    return status_of(launch_residual_norm(p, residual_bits == 32, st.sm_count, static_cast<cudaStream_t>(stream)));
}

extern "C" int w4a16_rotary_table(int64_t rot_dim, double base, int scaling, double factor, int64_t trained_tokens,
                                  double low_turns, double high_turns, uint64_t* turns) {
    constexpr double kTwoPi = 6.283185307179586476925;
    if (turns == nullptr || rot_dim <= 0 || !(base >= 1.0) || !std::isfinite(base)) return W4A16_ERR_INVALID_ARG;
    if (scaling < W4A16_ROTARY_SCALE_NONE || scaling > W4A16_ROTARY_SCALE_BY_INDEX) return W4A16_ERR_INVALID_ARG;
    if (rot_dim % 16 != 0 || rot_dim > kRotaryMaxDim) return W4A16_ERR_UNSUPPORTED;
    const bool parts = scaling == W4A16_ROTARY_SCALE_BY_TURNS || scaling == W4A16_ROTARY_SCALE_BY_INDEX;
    if (scaling != W4A16_ROTARY_SCALE_NONE && !(factor >= 1.0 && std::isfinite(factor))) return W4A16_ERR_INVALID_ARG;
    if (parts && (trained_tokens <= 0 || !(low_turns > 0.0) || !(high_turns > low_turns) || !std::isfinite(high_turns)))
        return W4A16_ERR_INVALID_ARG;
    if (scaling == W4A16_ROTARY_SCALE_BY_INDEX && base == 1.0) return W4A16_ERR_INVALID_ARG;
    const double dims = static_cast<double>(rot_dim), trained = static_cast<double>(trained_tokens);
    double first = 0.0, last = 0.0;
    if (scaling == W4A16_ROTARY_SCALE_BY_INDEX) {
        // the i at which a frequency makes so many turns over the trained length
        const auto index = [&](double n) { return dims * std::log(trained / (kTwoPi * n)) / (2.0 * std::log(base)); };
        first = std::max(std::floor(index(high_turns)), 0.0);
        last = std::min(std::ceil(index(low_turns)), dims - 1.0);
    }
    for (int64_t i = 0; i < rot_dim / 2; ++i) {
        const double theta = std::pow(base, -2.0 * static_cast<double>(i) / dims);
        double kept = 1.0;
        if (scaling == W4A16_ROTARY_SCALE_LINEAR) kept = 0.0;
        if (scaling == W4A16_ROTARY_SCALE_BY_TURNS)
            kept = (trained * theta / kTwoPi - low_turns) / (high_turns - low_turns);
        if (scaling == W4A16_ROTARY_SCALE_BY_INDEX)
            kept = 1.0 - (static_cast<double>(i) - first) / std::max(last - first, 0.001);
        kept = std::min(std::max(kept, 0.0), 1.0);
        const double scaled = scaling == W4A16_ROTARY_SCALE_NONE ? theta : theta * kept + theta / factor * (1.0 - kept);
        turns[i] = static_cast<uint64_t>(std::ldexp(scaled / kTwoPi, 64));  // (theta <= 1)
    }
    return W4A16_OK;
}

extern "C" int w4a16_rotary(void* qkv_bf16, const void* seq_start_i32, const void* first_i32, int64_t nseq, int64_t M,
                            int64_t H, int64_t kv_heads, int64_t d, const void* turns_u64, int64_t rot_dim, int layout,
                            float factor, void* stream) {
    if (qkv_bf16 == nullptr || turns_u64 == nullptr) return W4A16_ERR_INVALID_ARG;
    if (nseq <= 0 || M <= 0 || H < 0 || kv_heads < 0 || H + kv_heads <= 0 || d <= 0 || rot_dim <= 0 || rot_dim > d ||
        !std::isfinite(factor))
        return W4A16_ERR_INVALID_ARG;
    if (layout != W4A16_ROTARY_HALF && layout != W4A16_ROTARY_PAIRS) return W4A16_ERR_INVALID_ARG;
    if (seq_start_i32 == nullptr && nseq != M) return W4A16_ERR_INVALID_ARG;
    if (d % 8 != 0 || rot_dim % 16 != 0 || rot_dim > kRotaryMaxDim || M > kMaxDim || nseq > kMaxDim / 2 || H > 65535 ||
        kv_heads > 65535 || d > 65536 || (H + 2 * kv_heads) * d > kMaxDim)
        return W4A16_ERR_UNSUPPORTED;
    const Span in[3] = {{seq_start_i32, (nseq + 1) * 4}, {first_i32, nseq * 4}, {turns_u64, rot_dim / 2 * 8}};
    const Span out[1] = {{qkv_bf16, M * (H + 2 * kv_heads) * d * 2}};
    int rc = check_spans(in, out);
    if (rc != W4A16_OK) return rc;
    LibraryState st;
    rc = library_state(&st);
    if (rc != W4A16_OK) return rc;
    RotaryParams p;
    p.qkv = static_cast<uint16_t*>(qkv_bf16);
    p.seq_start = static_cast<const int32_t*>(seq_start_i32);
    p.first = static_cast<const int32_t*>(first_i32);
    p.turns = static_cast<const uint64_t*>(turns_u64);
    p.status = st.status;
    p.M = static_cast<int>(M);
    p.nseq = static_cast<int>(nseq);
    p.H = static_cast<int>(H);
    p.kv_heads = static_cast<int>(kv_heads);
    p.d = static_cast<int>(d);
    p.rot = static_cast<int>(rot_dim);
    p.factor = factor;
    p.pairs = layout == W4A16_ROTARY_PAIRS;
    return status_of(launch_rotary(nullptr, p, st.sm_count, static_cast<cudaStream_t>(stream)));
}

extern "C" int w4a16_log_probs(const void* logits, int logit_bits, int64_t M, int64_t V, int64_t row_stride,
                               const void* targets_i32, int64_t k, void* out_logp_f32, void* out_entropy_f32,
                               void* out_index_i32, void* out_score_f32, void* stream) {
    if (logits == nullptr || (logit_bits != 16 && logit_bits != 32)) return W4A16_ERR_INVALID_ARG;
    if (M <= 0 || V <= 0 || row_stride < V || k < 0 || k > V) return W4A16_ERR_INVALID_ARG;
    if ((targets_i32 != nullptr) != (out_logp_f32 != nullptr)) return W4A16_ERR_INVALID_ARG;
    if ((k > 0) != (out_index_i32 != nullptr) || (k > 0) != (out_score_f32 != nullptr)) return W4A16_ERR_INVALID_ARG;
    if (out_logp_f32 == nullptr && out_entropy_f32 == nullptr && k == 0) return W4A16_ERR_INVALID_ARG;
    if (k > kLogProbsMaxK || V > kLogProbsMaxV || M > kMaxDim / 8 || row_stride > kMaxDim) return W4A16_ERR_UNSUPPORTED;
    const Span in[2] = {{logits, ((M - 1) * row_stride + V) * (logit_bits / 8)}, {targets_i32, M * 4}};
    const Span out[4] = {{out_logp_f32, M * 4}, {out_entropy_f32, M * 4}, {out_index_i32, M * k * 4}, {out_score_f32, M * k * 4}};
    int rc = check_spans(in, out);
    if (rc != W4A16_OK) return rc;
    LibraryState st;
    rc = library_state(&st);
    if (rc != W4A16_OK) return rc;
    LogProbsParams p;
    p.logits = logits;
    p.targets = static_cast<const int32_t*>(targets_i32);
    p.logp = static_cast<float*>(out_logp_f32);
    p.entropy = static_cast<float*>(out_entropy_f32);
    p.index = static_cast<int32_t*>(out_index_i32);
    p.score = static_cast<float*>(out_score_f32);
    p.status = st.status;
    p.stride = row_stride;
    p.M = static_cast<int>(M);
    p.V = static_cast<int>(V);
    p.k = static_cast<int>(k);
    return status_of(launch_log_probs(p, logit_bits == 16, st.sm_count, static_cast<cudaStream_t>(stream)));
}

namespace {

int check_adapters(int64_t M, int64_t nseq, int64_t K, int64_t R) {
    if (M <= 0 || nseq <= 0 || K <= 0 || R <= 0) return W4A16_ERR_INVALID_ARG;
    if (M > kMaxDim / 64 || nseq > kMaxDim / 64 || K % 64 != 0 || K > kMaxDim / 64 || R % 8 != 0 || R > kAdapterMaxRank)
        return W4A16_ERR_UNSUPPORTED;
    return W4A16_OK;
}

}  // namespace

extern "C" int64_t w4a16_add_adapters_workspace(int64_t M, int64_t R) {
    return check_adapters(M, 1, 64, R) == W4A16_OK ? adapters_workspace_bytes(M, R) : 0;
}

extern "C" int w4a16_add_adapters(const void* x_bf16, const void* a_bf16, const void* b_bf16, const void* scale_f32,
                                  int64_t pool, const void* seq_start_i32, const void* adapters_i32, int64_t nseq,
                                  int64_t M, int64_t N, int64_t K, int64_t R, const void* base_bf16, void* out_bf16,
                                  void* workspace, void* stream) {
    if (x_bf16 == nullptr || a_bf16 == nullptr || b_bf16 == nullptr || scale_f32 == nullptr || adapters_i32 == nullptr ||
        base_bf16 == nullptr || out_bf16 == nullptr || workspace == nullptr)
        return W4A16_ERR_INVALID_ARG;
    if (N <= 0 || pool <= 0) return W4A16_ERR_INVALID_ARG;
    int rc = check_adapters(M, nseq, K, R);
    if (rc != W4A16_OK) return rc;
    if (seq_start_i32 == nullptr && nseq != M) return W4A16_ERR_INVALID_ARG;
    if (N > kMaxDim / 64 || pool > kMaxDim / 64) return W4A16_ERR_UNSUPPORTED;
    const Span in[6] = {{x_bf16, M * K * 2},  {a_bf16, pool * R * K * 2},         {b_bf16, pool * N * R * 2},
                  {scale_f32, pool * 4}, {seq_start_i32, (nseq + 1) * 4}, {adapters_i32, nseq * 4}};
    const Span base{base_bf16, M * N * 2};
    const Span out[2] = {{out_bf16, M * N * 2}, {workspace, adapters_workspace_bytes(M, R)}};
    rc = check_spans(in, out);
    if (rc != W4A16_OK) return rc;
    if (!aligned16(base_bf16)) return W4A16_ERR_ALIGNMENT;
    if ((base_bf16 != out_bf16 && overlaps(base, out[0])) || overlaps(base, out[1])) return W4A16_ERR_INVALID_ARG;
    LibraryState st;
    rc = library_state(&st);
    if (rc != W4A16_OK) return rc;
    AdapterParams p;
    p.x = static_cast<const uint16_t*>(x_bf16);
    p.a = static_cast<const uint16_t*>(a_bf16);
    p.b = static_cast<const uint16_t*>(b_bf16);
    p.scale = static_cast<const float*>(scale_f32);
    p.seq_start = static_cast<const int32_t*>(seq_start_i32);
    p.ids = static_cast<const int32_t*>(adapters_i32);
    p.base = static_cast<const uint16_t*>(base_bf16);
    p.out = static_cast<uint16_t*>(out_bf16);
    p.t = static_cast<uint16_t*>(workspace);
    p.status = st.status;
    p.M = static_cast<int>(M);
    p.N = static_cast<int>(N);
    p.K = static_cast<int>(K);
    p.R = static_cast<int>(R);
    p.pool = static_cast<int>(pool);
    p.nseq = static_cast<int>(nseq);
    p.wait_ns = wait_limit_ns();
    return status_of(launch_adapters(p, st.sm_count, static_cast<cudaStream_t>(stream)));
}

// (here: api.cu decides which kernels a linear runs, and counters captured of those are kept by its contents)
extern "C" int w4a16_version(void) { return 300; }
