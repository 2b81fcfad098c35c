// call_checks.h -- argument checks shared by the C-ABI layers of the calls around a larger model's
// tokens (token_api.hip, cache_api.hip).  Not part of the public interface.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdlib>
#include <cstring>
#include <exception>
#include <string>
#include <vector>

#include "internal.h"
#include "ts_token.h"

namespace tsc {

constexpr int64_t kMaxRows = (int64_t)1 << 29;
constexpr int64_t kMaxStride = (int64_t)1 << 40;

inline bool checked() {
    const char* env = std::getenv("TS_CHECK");
    return env && std::strcmp(env, "1") == 0;
}

// Runs a call's body; nothing is thrown through the C boundary
template <class F>
ts_status guarded(F f) {
    try {
        return f();
    } catch (const std::exception&) {
        return TS_ERR_HIP;   // host memory ran out while a check or a message was being made
    }
}

inline ts_status bad(const char* call, ts_status code, const std::string& what) {
    return report_error(code, (std::string(call) + ": " + what).c_str());
}

inline ts_status done(const char* call, hipError_t e) {
    if (e == hipSuccess) return TS_OK;
    return bad(call, TS_ERR_HIP, std::string("HIP: ") + hipGetErrorString(e));
}

inline ts_status check_type(const char* call, const char* name, int dtype) {
    if (dtype >= TS_FLOAT32 && dtype <= TS_FLOAT16) return TS_OK;
    return bad(call, TS_ERR_BAD_ARG, std::string(name) + " has no element type of code " +
                                         std::to_string(dtype));
}

inline ts_status check_ptr(const char* call, const char* name, const void* p) {
    if (p) return TS_OK;
    return bad(call, TS_ERR_NULL_ARG, std::string(name) + " is NULL");
}

inline ts_status check_ws(const char* call, size_t need, const void* ws, size_t ws_bytes) {
    if (need == 0) return TS_OK;
    if (!ws) return bad(call, TS_ERR_NULL_ARG, "ws is NULL");
    if (ws_bytes >= need && reinterpret_cast<uintptr_t>(ws) % 256 == 0) return TS_OK;
    return bad(call, TS_ERR_WORKSPACE, "the workspace needs " + std::to_string(need) +
                                           " bytes aligned to 256 (got " +
                                           std::to_string(ws_bytes) + ")");
}

// TS_CHECK=1: lengths within [0, N], read on the host; len keeps them
inline ts_status check_lengths(const char* call, const int32_t* lengths, int64_t B, int64_t N,
                                hipStream_t s, std::vector<int32_t>* len) {
    len->assign((size_t)B, (int32_t)N);
    if (!lengths) return TS_OK;
    if (hipMemcpyAsync(len->data(), lengths, sizeof(int32_t) * B, hipMemcpyDeviceToHost, s) !=
            hipSuccess ||
        hipStreamSynchronize(s) != hipSuccess)
        return bad(call, TS_ERR_HIP, "could not read lengths for TS_CHECK");
    for (int64_t b = 0; b < B; ++b)
        if ((*len)[b] < 0 || (*len)[b] > N)
            return bad(call, TS_ERR_LENGTHS, "lengths[" + std::to_string(b) + "] = " +
                                                 std::to_string((*len)[b]) +
                                                 " is outside [0, N]");
    return TS_OK;
}

}  // namespace tsc
