// token_api.hip -- the C ABI declared in include/ts_token.h: argument checks, workspace sizes
// and the choice of kernels.  The kernels are in token_top.hip, token_distill.hip, token_score.hip
// and token_verify.hip.
#include <hip/hip_runtime.h>

#include <cmath>
#include <string>
#include <vector>

#include "call_checks.h"
#include "token.h"
#include "token_calls.h"

namespace tsc {
namespace {

bool dims_ok(int64_t B, int64_t N, int64_t V) {
    return B >= 1 && N >= 1 && V >= 1 && V <= kMaxVocab && B <= kMaxRows && N <= kMaxRows &&
           B * N <= kMaxRows;
}

ts_status check_dims(const char* call, int64_t B, int64_t N, int64_t V) {
    if (dims_ok(B, N, V)) return TS_OK;
    return bad(call, TS_ERR_BAD_DIM,
               "B, N, V must be >= 1, V <= " + std::to_string(kMaxVocab) +
                   " and B * N <= 2^29 (got " + std::to_string(B) + ", " + std::to_string(N) +
                   ", " + std::to_string(V) + ")");
}

ts_status check_top(const char* call, int64_t V, int64_t K) {
    if (K >= 1 && K <= V && K <= kMaxTop) return TS_OK;
    return bad(call, TS_ERR_BAD_DIM, "K must be in [1, min(V, " + std::to_string(kMaxTop) +
                                         ")] (got " + std::to_string(K) + ")");
}

ts_status check_rows(const char* call, const char* name, int dtype, int64_t sb, int64_t sn) {
    if (ts_status st = check_type(call, name, dtype)) return st;
    if (sb >= 0 && sn >= 0 && sb <= kMaxStride && sn <= kMaxStride) return TS_OK;
    return bad(call, TS_ERR_BAD_ARG, std::string("strides of ") + name +
                                         " must be in [0, 2^40] elements");
}

ts_status check_temperature(const char* call, const char* name, float t) {
    // 1 / T and log2(e) / T have to be normal floats, and every finite logit's quotient a sum
    if (t >= 1e-6f && t <= 1e6f) return TS_OK;
    return bad(call, TS_ERR_BAD_ARG, std::string(name) + " must be in [1e-6, 1e6]");
}

// TS_CHECK=1: W whole numbers of every row within [lo, V), no two of a row alike where
// `distinct` (-1 may repeat)
ts_status check_tokens(const char* call, const char* name, const int32_t* at, int64_t B, int64_t N,
                       int64_t W, int64_t lo, int64_t V, bool distinct,
                       const std::vector<int32_t>& len, hipStream_t s) {
    std::vector<int32_t> h((size_t)(B * N * W));
    if (h.empty()) return TS_OK;
    if (hipMemcpyAsync(h.data(), at, sizeof(int32_t) * h.size(), hipMemcpyDeviceToHost, s) !=
            hipSuccess ||
        hipStreamSynchronize(s) != hipSuccess)
        return bad(call, TS_ERR_HIP, std::string("could not read ") + name + " for TS_CHECK");
    std::vector<int64_t> seen(distinct ? (size_t)V : 0, -1);
    for (int64_t b = 0; b < B; ++b)
        for (int64_t n = 0; n < len[b]; ++n)
            for (int64_t k = 0; k < W; ++k) {
                const int64_t row = b * N + n, i = h[(size_t)(row * W + k)];
                const bool twice = distinct && i >= 0 && i < V && seen[(size_t)i] == row;
                if (i < lo || i >= V || twice)
                    return bad(call, TS_ERR_LABELS,
                               std::string(name) + "[" + std::to_string(b) + ", " +
                                   std::to_string(n) + (W > 1 ? ", " + std::to_string(k) : "") +
                                   "] = " + std::to_string(i) +
                                   (twice ? " is in its row twice" : " is out of range"));
                if (distinct && i >= 0) seen[(size_t)i] = row;
            }
    return TS_OK;
}

ts_status distill_call(const char* call, DistillArgs& a, int dtype, int top_dtype, int64_t K,
                       float temperature, int op, void* ws, size_t ws_bytes, void* stream) {
    ts_status st;
    if ((st = check_dims(call, a.B, a.N, a.V)) || (st = check_top(call, a.V, K)) ||
        (st = check_rows(call, "logits", dtype, a.logits.sb, a.logits.sn)) ||
        (st = check_type(call, "top_values", top_dtype)) ||
        (st = check_temperature(call, "temperature", temperature)) ||
        (st = check_ptr(call, "logits", a.logits.p)) ||
        (st = check_ptr(call, "top_values", a.top_values)) ||
        (st = check_ptr(call, "top_indices", a.top_indices)) ||
        (st = op == TS_TOKEN_DISTILL ? check_ptr(call, "loss", a.loss)
                                     : check_ptr(call, "grad", a.grad)) ||
        (st = check_ws(call, distill_workspace(op, a.B, a.N, a.V, K), ws, ws_bytes)))
        return st;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (checked()) {
        std::vector<int32_t> len;
        if ((st = check_lengths(call, a.lengths, a.B, a.N, s, &len)) ||
            (st = check_tokens(call, "top_indices", a.top_indices, a.B, a.N, K, -1, a.V, true, len,
                               s)))
            return st;
    }
    a.dtype = dtype;
    a.top_dtype = top_dtype;
    a.K = (int)K;
    a.scale = make_scale(temperature);
    a.ws = ws;
    return done(call, launch_distill(a, s));
}

}  // namespace
}  // namespace tsc

using namespace tsc;

extern "C" {

int ts_token_max_vocab(void) { return kMaxVocab; }
int ts_token_max_top(void) { return kMaxTop; }

size_t ts_token_workspace_bytes(int op, int64_t B, int64_t N, int64_t V, int64_t K) {
    if (op == TS_TOKEN_VERIFY)
        return N >= 0 && N < kMaxRows && dims_ok(B, N + 1, V) ? verify_workspace(B, N, V) : 0;
    if (op == TS_TOKEN_SCORE_GRAD || (op == TS_TOKEN_SCORE && K == 0))
        return dims_ok(B, N, V) ? score_workspace(B, N, V) : 0;
    if (!dims_ok(B, N, V) || K < 1 || K > V || K > kMaxTop) return 0;
    if (op == TS_TOKEN_TOP || op == TS_TOKEN_SCORE) return top_workspace(B, N, V, K);
    if (op == TS_TOKEN_DISTILL || op == TS_TOKEN_DISTILL_GRAD)
        return distill_workspace(op, B, N, V, K);
    return 0;
}

ts_status ts_token_top(const void* logits, int dtype, int64_t stride_b, int64_t stride_n,
                       const int32_t* lengths, int64_t B, int64_t N, int64_t V, int64_t K,
                       float temperature, void* values, int32_t* indices, float* lse, void* ws,
                       size_t ws_bytes, void* stream) {
    return guarded([&]() -> ts_status {
        const char* call = "ts_token_top";
        ts_status st;
        if ((st = check_dims(call, B, N, V)) || (st = check_top(call, V, K)) ||
            (st = check_rows(call, "logits", dtype, stride_b, stride_n)) ||
            (st = check_temperature(call, "temperature", temperature)) ||
            (st = check_ptr(call, "logits", logits)) || (st = check_ptr(call, "values", values)) ||
            (st = check_ptr(call, "indices", indices)) ||
            (st = check_ws(call, top_workspace(B, N, V, K), ws, ws_bytes)))
            return st;
        const hipStream_t s = static_cast<hipStream_t>(stream);
        if (checked()) {
            std::vector<int32_t> len;
            if ((st = check_lengths(call, lengths, B, N, s, &len))) return st;
        }
        const TopArgs a{{logits, stride_b, stride_n}, dtype, lengths, B, N, (int)V, (int)K,
                        make_scale(temperature), values, indices, lse, ws, nullptr, nullptr, nullptr};
        return done(call, launch_top(a, s));
    });
}

ts_status ts_token_distill(const void* logits, int dtype, int64_t stride_b, int64_t stride_n,
                           const void* top_values, int top_dtype, const int32_t* top_indices,
                           const float* top_lse, const int32_t* lengths, int64_t B, int64_t N,
                           int64_t V, int64_t K, float temperature, float* loss, void* ws,
                           size_t ws_bytes, void* stream) {
    return guarded([&]() -> ts_status {
        DistillArgs a{};
        a.logits = {logits, stride_b, stride_n};
        a.top_values = top_values;
        a.top_indices = top_indices;
        a.top_lse = top_lse;
        a.lengths = lengths;
        a.B = B;
        a.N = N;
        a.V = V;
        a.loss = loss;
        return distill_call("ts_token_distill", a, dtype, top_dtype, K, temperature,
                            TS_TOKEN_DISTILL, ws, ws_bytes, stream);
    });
}

ts_status ts_token_distill_grad(const void* logits, int dtype, int64_t stride_b,
                                int64_t stride_n, const void* top_values, int top_dtype,
                                const int32_t* top_indices, const float* top_lse,
                                const float* weights, const int32_t* lengths, int64_t B,
                                int64_t N, int64_t V, int64_t K, float temperature, float* loss,
                                void* grad, void* ws, size_t ws_bytes, void* stream) {
    return guarded([&]() -> ts_status {
        DistillArgs a{};
        a.logits = {logits, stride_b, stride_n};
        a.top_values = top_values;
        a.top_indices = top_indices;
        a.top_lse = top_lse;
        a.weights = weights;
        a.lengths = lengths;
        a.B = B;
        a.N = N;
        a.V = V;
        a.loss = loss;
        a.grad = grad;
        return distill_call("ts_token_distill_grad", a, dtype, top_dtype, K, temperature,
                            TS_TOKEN_DISTILL_GRAD, ws, ws_bytes, stream);
    });
}

ts_status ts_token_score(const void* logits, int dtype, int64_t stride_b, int64_t stride_n,
                         const int32_t* tokens, const int32_t* lengths, int64_t B, int64_t N,
                         int64_t V, int64_t K, float temperature, float* logp, float* entropy,
                         int32_t* alternatives, float* alternative_logp, void* ws,
                         size_t ws_bytes, void* stream) {
    return guarded([&]() -> ts_status {
        const char* call = "ts_token_score";
        ts_status st;
        if ((st = check_dims(call, B, N, V)) || (K && (st = check_top(call, V, K))) ||
            (st = check_rows(call, "logits", dtype, stride_b, stride_n)) ||
            (st = check_temperature(call, "temperature", temperature)) ||
            (st = check_ptr(call, "logits", logits)) || (st = check_ptr(call, "tokens", tokens)) ||
            (st = check_ptr(call, "logp", logp)) || (st = check_ptr(call, "entropy", entropy)) ||
            (K && ((st = check_ptr(call, "alternatives", alternatives)) ||
                   (st = check_ptr(call, "alternative_logp", alternative_logp)))) ||
            (st = check_ws(call, ts_token_workspace_bytes(TS_TOKEN_SCORE, B, N, V, K), ws, ws_bytes)))
            return st;
        const hipStream_t s = static_cast<hipStream_t>(stream);
        if (checked()) {
            std::vector<int32_t> len;
            if ((st = check_lengths(call, lengths, B, N, s, &len))) return st;
        }
        if (K) {
            const TopArgs a{{logits, stride_b, stride_n}, dtype, lengths, B, N, (int)V, (int)K,
                            make_scale(temperature), alternative_logp, alternatives, nullptr, ws,
                            tokens, logp, entropy};
            return done(call, launch_top(a, s));
        }
        ScoreArgs a{};
        a.logits = {logits, stride_b, stride_n};
        a.tokens = tokens;
        a.lengths = lengths;
        a.B = B;
        a.N = N;
        a.logp = logp;
        a.entropy = entropy;
        a.V = (int)V;
        a.dtype = dtype;
        a.scale = make_scale(temperature);
        a.ws = ws;
        return done(call, launch_score(a, s));
    });
}

ts_status ts_token_score_grad(const void* logits, int dtype, int64_t stride_b, int64_t stride_n,
                              const int32_t* tokens, const float* weights,
                              const float* entropy_weights, const int32_t* lengths, int64_t B,
                              int64_t N, int64_t V, float temperature, float* logp,
                              float* entropy, void* grad, void* ws, size_t ws_bytes,
                              void* stream) {
    return guarded([&]() -> ts_status {
        const char* call = "ts_token_score_grad";
        ts_status st;
        if ((st = check_dims(call, B, N, V)) ||
            (st = check_rows(call, "logits", dtype, stride_b, stride_n)) ||
            (st = check_temperature(call, "temperature", temperature)) ||
            (st = check_ptr(call, "logits", logits)) || (st = check_ptr(call, "tokens", tokens)) ||
            (st = check_ptr(call, "grad", grad)) ||
            (st = check_ws(call, score_workspace(B, N, V), ws, ws_bytes)))
            return st;
        const hipStream_t s = static_cast<hipStream_t>(stream);
        if (checked()) {
            std::vector<int32_t> len;
            if ((st = check_lengths(call, lengths, B, N, s, &len))) return st;
        }
        const ScoreArgs a{{logits, stride_b, stride_n}, tokens, weights, entropy_weights, lengths, B, N,
                          logp, entropy, grad, (int)V, dtype, make_scale(temperature), ws};
        return done(call, launch_score(a, s));
    });
}

ts_status ts_token_verify(const void* target, int target_dtype, int64_t target_stride_b,
                          int64_t target_stride_n, const void* draft, int draft_dtype,
                          int64_t draft_stride_b, int64_t draft_stride_n, const float* draft_lse,
                          const int32_t* tokens, const float* uniforms, const float* noise,
                          const int32_t* lengths, int64_t B, int64_t G, int64_t V,
                          float temperature, float draft_temperature, int32_t* out,
                          int32_t* accepted, float* logp, void* ws, size_t ws_bytes,
                          void* stream) {
    return guarded([&]() -> ts_status {
        const char* call = "ts_token_verify";
        ts_status st;
        if (G < 0 || G >= kMaxRows)
            return bad(call, TS_ERR_BAD_DIM, "G must be >= 0 and B * (G + 1) <= 2^29");
        if ((st = check_dims(call, B, G + 1, V)) ||
            (st = check_rows(call, "target", target_dtype, target_stride_b, target_stride_n)) ||
            (st = check_rows(call, "draft", draft_dtype, draft_stride_b, draft_stride_n)) ||
            (st = check_temperature(call, "temperature", temperature)) ||
            (st = check_temperature(call, "draft_temperature", draft_temperature)) ||
            (st = check_ptr(call, "target", target)) ||
            (st = check_ptr(call, "noise", noise)) || (st = check_ptr(call, "out", out)) ||
            (st = check_ptr(call, "accepted", accepted)) ||
            (G > 0 && ((st = check_ptr(call, "draft", draft)) ||
                       (st = check_ptr(call, "tokens", tokens)) ||
                       (st = check_ptr(call, "uniforms", uniforms)))) ||
            (st = check_ws(call, verify_workspace(B, G, V), ws, ws_bytes)))
            return st;
        const hipStream_t s = static_cast<hipStream_t>(stream);
        if (checked()) {
            std::vector<int32_t> len;
            if ((st = check_lengths(call, lengths, B, G, s, &len)) ||
                (st = check_tokens(call, "tokens", tokens, B, G, 1, 0, V, false, len, s)))
                return st;
        }
        const VerifyArgs a{{target, target_stride_b, target_stride_n},
                           {draft, draft_stride_b, draft_stride_n},
                           target_dtype, draft_dtype, draft_lse, tokens, uniforms, noise, lengths,
                           B, G, (int)V, make_scale(temperature), make_scale(draft_temperature),
                           out, accepted, logp, ws};
        return done(call, launch_verify(a, s));
    });
}

}  // extern "C"
