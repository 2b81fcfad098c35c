// cache_api.hip -- the C ABI declared in include/ts_cache.h: argument checks and workspace sizes.  The
// kernels are in cache_append.hip and cache_attend.hip.
#include <hip/hip_runtime.h>

#include <cmath>
#include <string>
#include <vector>

#include "cache_calls.h"
#include "call_checks.h"
#include "ts_cache.h"

namespace tsc {
namespace {

constexpr int64_t kMaxQueryHeads = 1024;
constexpr int64_t kMaxSlots = (int64_t)1 << 30;

bool heads_ok(int64_t B, int64_t N, int64_t Hq, int64_t Hk, int64_t D) {
    return B >= 1 && N >= 1 && Hq >= 1 && Hk >= 1 && Hq <= kMaxQueryHeads && Hq % Hk == 0 &&
           D >= 8 && D <= kMaxHead && D % 8 == 0 && B <= kMaxRows && N <= kMaxRows &&
           B * N <= kMaxRows && B * N * Hq <= kMaxRows;
}

ts_status check_heads(const char* call, int64_t B, int64_t N, int64_t Hq, int64_t Hk, int64_t D) {
    if (heads_ok(B, N, Hq, Hk, D)) return TS_OK;
    return bad(call, TS_ERR_BAD_DIM,
               "B, N must be >= 1, Hq a multiple of Hk up to 1024, D a multiple of 8 up to " +
                   std::to_string(kMaxHead) + " and B * N * Hq <= 2^29 (got B " + std::to_string(B) +
                   ", N " + std::to_string(N) + ", Hq " + std::to_string(Hq) + ", Hk " +
                   std::to_string(Hk) + ", D " + std::to_string(D) + ")");
}

ts_status check_half(const char* call, int dtype) {
    if (dtype == TS_BFLOAT16 || dtype == TS_FLOAT16) return TS_OK;
    return bad(call, TS_ERR_BAD_ARG, "the element type must be bfloat16 or float16 (got code " +
                                         std::to_string(dtype) + ")");
}

ts_status check_aligned(const char* call, const char* name, const void* p, const int64_t* strides) {
    for (int i = 0; i < 3; ++i)
        if (strides[i] < 0 || strides[i] > kMaxStride || strides[i] % 8)
            return bad(call, TS_ERR_BAD_ARG, std::string("strides of ") + name +
                                                 " must be multiples of 8 in [0, 2^40] elements");
    if (reinterpret_cast<uintptr_t>(p) % 16)
        return bad(call, TS_ERR_BAD_ARG, std::string(name) + " must start at a multiple of 16 bytes");
    return TS_OK;
}

ts_status check_layout(const char* call, const ts_cache_layout* c, const void* k, const void* v,
                       const int32_t* pages, int64_t M, const int32_t* starts) {
    ts_status st;
    if ((st = check_ptr(call, "layout", c)) || (st = check_ptr(call, "k_cache", k)) ||
        (st = check_ptr(call, "v_cache", v)) || (st = check_ptr(call, "pages", pages)) ||
        (st = check_ptr(call, "starts", starts)))
        return st;
    if (c->pages < 1 || c->pages > INT32_MAX || c->page_size < 1 || c->page_size > kMaxSlots ||
        M < 1 || M > kMaxSlots || M * c->page_size > kMaxSlots)
        return bad(call, TS_ERR_BAD_DIM,
                   "P, S and M must be >= 1, P < 2^31 and M * S <= 2^30 (got P " +
                       std::to_string(c->pages) + ", S " + std::to_string(c->page_size) + ", M " +
                       std::to_string(M) + ")");
    const int64_t strides[3] = {c->stride_page, c->stride_token, c->stride_head};
    if ((st = check_aligned(call, "k_cache", k, strides)) ||
        (st = check_aligned(call, "v_cache", v, strides)))
        return st;
    return TS_OK;
}

Cache cache_of(const ts_cache_layout& c, void* k, void* v, const int32_t* pages, int64_t M,
               const int32_t* starts, const int32_t* lengths) {
    const uint64_t inv = ((uint64_t)1 << 32) / (uint64_t)c.page_size;
    return {k, v, c.stride_page, c.stride_token, c.stride_head, pages, starts, lengths, c.pages,
            (int32_t)M, (int32_t)c.page_size, inv > 0xffffffffu ? 0xffffffffu : (uint32_t)inv};
}

bool copy_ints(std::vector<int32_t>* to, const int32_t* from, int64_t n, hipStream_t s) {
    to->resize((size_t)n);
    return hipMemcpyAsync(to->data(), from, sizeof(int32_t) * n, hipMemcpyDeviceToHost, s) ==
               hipSuccess &&
           hipStreamSynchronize(s) == hipSuccess;
}

// TS_CHECK=1: lengths, starts and the pages of slots [from the first new one or 0, the last new one]
ts_status check_slots(const char* call, const Cache& c, int64_t B, int64_t N, bool all, hipStream_t s,
                      std::vector<int32_t>* len) {
    if (ts_status st = check_lengths(call, c.lengths, B, N, s, len)) return st;
    std::vector<int32_t> starts, pages;
    if (!copy_ints(&starts, c.starts, B, s) || !copy_ints(&pages, c.pages, B * c.M, s))
        return bad(call, TS_ERR_HIP, "could not read starts and pages for TS_CHECK");
    for (int64_t b = 0; b < B; ++b) {
        const int64_t n = (*len)[b], start = starts[b], end = start + n;
        if (start < 0 || end > (int64_t)c.M * c.S)
            return bad(call, TS_ERR_LENGTHS, "starts[" + std::to_string(b) + "] = " +
                                                 std::to_string(start) + " with " + std::to_string(n) +
                                                 " new tokens is outside [0, M * S]");
        if (n == 0) continue;   // nothing of the sequence is read or written
        for (int64_t m = all ? 0 : start / c.S; m * c.S < end; ++m)
            if (pages[b * c.M + m] < 0 || pages[b * c.M + m] >= c.P)
                return bad(call, TS_ERR_LABELS, "pages[" + std::to_string(b) + ", " +
                                                    std::to_string(m) + "] = " +
                                                    std::to_string(pages[b * c.M + m]) +
                                                    " is outside [0, P)");
    }
    return TS_OK;
}

}  // namespace
}  // namespace tsc

using namespace tsc;

extern "C" {

int ts_cache_max_head(void) { return kMaxHead; }
int ts_cache_max_nodes(void) { return kMaxNodes; }

ts_status ts_cache_append(const void* k, const void* v, const void* q, const int64_t strides[9],
                          int dtype, const float* freqs, int64_t R, int neighbours,
                          const int32_t* positions, void* k_cache, void* v_cache,
                          const ts_cache_layout* layout, const int32_t* pages, int64_t M,
                          const int32_t* starts, const int32_t* lengths, int64_t B, int64_t N,
                          int64_t Hq, void* q_out, void* stream) {
    return guarded([&]() -> ts_status {
        const char* call = "ts_cache_append";
        ts_status st;
        if ((st = check_ptr(call, "k", k)) || (st = check_ptr(call, "v", v)) ||
            (st = check_ptr(call, "strides", strides)) ||
            (st = check_layout(call, layout, k_cache, v_cache, pages, M, starts)))
            return st;
        if (!q != !q_out) return bad(call, TS_ERR_NULL_ARG, "q and q_out are both given or both NULL");
        const int64_t Hk = layout->heads, D = layout->head_size;
        if ((st = check_heads(call, B, N, q ? Hq : Hk, Hk, D)) || (st = check_half(call, dtype)) ||
            (st = check_aligned(call, "k", k, strides)) ||
            (st = check_aligned(call, "v", v, strides + 3)) ||
            (q && ((st = check_aligned(call, "q", q, strides + 6)) ||
                   (reinterpret_cast<uintptr_t>(q_out) % 16 &&
                    (st = bad(call, TS_ERR_BAD_ARG, "q_out must start at a multiple of 16 bytes"))))))
            return st;
        if (!freqs) R = 0;
        if (R < 0 || R > D || R % 16)
            return bad(call, TS_ERR_BAD_DIM, "R must be a multiple of 16 in [0, D] (got " +
                                                 std::to_string(R) + ")");
        AppendArgs a{};
        a.k = {k, strides[0], strides[1], strides[2]};
        a.v = {v, strides[3], strides[4], strides[5]};
        if (q) a.q = {q, strides[6], strides[7], strides[8]};
        a.dtype = dtype;
        a.freqs = freqs;
        a.positions = positions;
        a.c = cache_of(*layout, k_cache, v_cache, pages, M, starts, lengths);
        a.B = B;
        a.N = N;
        a.Hq = q ? (int)Hq : 0;
        a.Hk = (int)Hk;
        a.D = (int)D;
        a.R = (int)R;
        a.neighbours = neighbours != 0;
        a.q_out = q_out;
        const hipStream_t s = static_cast<hipStream_t>(stream);
        std::vector<int32_t> len;
        if (checked() && (st = check_slots(call, a.c, B, N, false, s, &len))) return st;
        return done(call, launch_append(a, s));
    });
}

size_t ts_cache_attend_workspace_bytes(int64_t B, int64_t N, int64_t Hq, int64_t Hk, int64_t D) {
    return heads_ok(B, N, Hq, Hk, D) && N <= kMaxNodes ? attend_workspace(B, N, Hq, Hk, D) : 0;
}

ts_status ts_cache_attend(const void* q, const int64_t strides[3], int dtype, const void* k_cache,
                          const void* v_cache, const ts_cache_layout* layout,
                          const int32_t* pages, int64_t M, const int32_t* starts,
                          const int32_t* parents, const int32_t* lengths, int64_t B, int64_t N,
                          int64_t Hq, float scale, void* out, float* lse, void* ws,
                          size_t ws_bytes, void* stream) {
    return guarded([&]() -> ts_status {
        const char* call = "ts_cache_attend";
        ts_status st;
        if ((st = check_ptr(call, "q", q)) || (st = check_ptr(call, "strides", strides)) ||
            (st = check_ptr(call, "out", out)) ||
            (st = check_layout(call, layout, k_cache, v_cache, pages, M, starts)))
            return st;
        const int64_t Hk = layout->heads, D = layout->head_size;
        if ((st = check_heads(call, B, N, Hq, Hk, D))) return st;
        if (N > kMaxNodes || !attend_fits(B, N, Hq, Hk, D, M * layout->page_size))
            return bad(call, TS_ERR_BAD_DIM, "N must be at most " + std::to_string(kMaxNodes) +
                                                 ", row tiles of all key heads 2^23, and a head's tiles of "
                                                 "32 slots of them all 2^31 a workgroup");
        if ((st = check_half(call, dtype)) || (st = check_aligned(call, "q", q, strides))) return st;
        if (!(scale >= 1e-6f && scale <= 1e6f))
            return bad(call, TS_ERR_BAD_ARG, "scale must be in [1e-6, 1e6]");
        if (reinterpret_cast<uintptr_t>(out) % 16)
            return bad(call, TS_ERR_BAD_ARG, "out must start at a multiple of 16 bytes");
        if ((st = check_ws(call, attend_workspace(B, N, Hq, Hk, D), ws, ws_bytes))) return st;
        AttendArgs a{};
        a.q = {q, strides[0], strides[1], strides[2]};
        a.dtype = dtype;
        a.c = cache_of(*layout, const_cast<void*>(k_cache), const_cast<void*>(v_cache), pages, M, starts,
                       lengths);
        a.parents = parents;
        a.B = B;
        a.N = (int)N;
        a.Hq = (int)Hq;
        a.Hk = (int)Hk;
        a.D = (int)D;
        a.c2 = (float)((double)scale * 1.4426950408889634);
        a.scale = scale;
        a.out = out;
        a.lse = lse;
        a.ws = ws;
        const hipStream_t s = static_cast<hipStream_t>(stream);
        if (checked()) {
            std::vector<int32_t> len, up;
            if ((st = check_slots(call, a.c, B, N, true, s, &len))) return st;
            if (parents && !copy_ints(&up, parents, B * N, s))
                return bad(call, TS_ERR_HIP, "could not read parents for TS_CHECK");
            for (int64_t b = 0; parents && b < B; ++b)
                for (int64_t n = 0; n < len[b]; ++n)
                    if (up[b * N + n] < -1 || up[b * N + n] >= n)
                        return bad(call, TS_ERR_LABELS, "parents[" + std::to_string(b) + ", " +
                                                            std::to_string(n) + "] = " +
                                                            std::to_string(up[b * N + n]) +
                                                            " is outside [-1, " + std::to_string(n) +
                                                            ")");
        }
        return done(call, launch_attend(a, s));
    });
}

}  // extern "C"
