// token_calls.h -- what the C-ABI layer (token_api.hip) passes to the kernels on rows of token
// logits, and the workspace that they need.  Not part of the public interface.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace tsc {

// Rows of logits [B, N, V]: elements from a sequence, a row to the next
struct Rows {
    const void* p;
    int64_t sb, sn;
};

struct Scale {
    float c;       // log2(e) / T
    float inv_t;   // 1 / T
    float most;    // logits up to here have exponents of at most 2^29
};
inline Scale make_scale(float t) {
    const double c = 1.4426950408889634 / (double)t;
    return {(float)c, (float)(1.0 / (double)t), (float)(536870912.0 / c)};
}

struct TopArgs {
    Rows logits;
    int dtype;
    const int32_t* lengths;
    int64_t B, N;
    int V, K;
    Scale scale;
    void* values;             // with tokens: their log-probabilities, float32
    int32_t* indices;
    float* lse;
    void* ws;
    const int32_t* tokens;    // the scores of these are asked for, and the rows' entropies
    float* logp;
    float* entropy;
};
size_t top_workspace(int64_t B, int64_t N, int64_t V, int64_t K);
hipError_t launch_top(const TopArgs& a, hipStream_t s);

struct DistillArgs {
    Rows logits;
    const void* top_values;
    const int32_t* top_indices;
    const float* top_lse;
    const float* weights;
    const int32_t* lengths;
    int64_t B, N, V;
    float* loss;
    void* grad;   // NULL: the loss alone
    int dtype, top_dtype, K;
    Scale scale;
    void* ws;
};
size_t distill_workspace(int op, int64_t B, int64_t N, int64_t V, int64_t K);
hipError_t launch_distill(const DistillArgs& a, hipStream_t s);

struct ScoreArgs {
    Rows logits;
    const int32_t* tokens;
    const float* weights;
    const float* entropy_weights;
    const int32_t* lengths;
    int64_t B, N;
    float* logp;
    float* entropy;
    void* grad;   // NULL: the scores alone
    int V, dtype;
    Scale scale;
    void* ws;
};
size_t score_workspace(int64_t B, int64_t N, int64_t V);
hipError_t launch_score(const ScoreArgs& a, hipStream_t s);

struct VerifyArgs {
    Rows target, draft;
    int target_dtype, draft_dtype;
    const float* draft_lse;
    const int32_t* tokens;
    const float* uniforms;
    const float* noise;
    const int32_t* lengths;
    int64_t B, G;
    int V;
    Scale scale, draft_scale;
    int32_t* out;
    int32_t* accepted;
    float* logp;
    void* ws;
};
size_t verify_workspace(int64_t B, int64_t G, int64_t V);
hipError_t launch_verify(const VerifyArgs& a, hipStream_t s);

}  // namespace tsc
