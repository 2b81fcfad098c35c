// cache_calls.h -- what the C-ABI layer (cache_api.hip) passes to the kernels on a paged cache, and
// the workspace that they need.  Not part of the public interface.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace tsc {

constexpr int kMaxHead = 256;
constexpr int kMaxNodes = 256;

// Heads of [B, N, H, D]: elements from a sequence, a token, a head to the next
struct Heads {
    const void* p;
    int64_t sb, sn, sh;
};

struct Cache {
    void* k;
    void* v;
    int64_t sp, st, sh;      // elements from a page, a token, a head to the next
    const int32_t* pages;    // [B, M]
    const int32_t* starts;
    const int32_t* lengths;
    int64_t P;
    int32_t M, S;            // pages of a sequence, tokens of a page
    uint32_t inv;            // floor(2^32 / S), or 2^32 - 1: j / S is umulhi(j, inv) or one more
};

struct AppendArgs {
    Heads k, v, q;
    int dtype;
    const float* freqs;
    const int32_t* positions;
    Cache c;
    int64_t B, N;
    int Hq, Hk, D, R, neighbours;
    void* q_out;
};
hipError_t launch_append(const AppendArgs& a, hipStream_t s);

struct AttendArgs {
    Heads q;
    int dtype;
    Cache c;
    const int32_t* parents;
    int64_t B;
    int N, Hq, Hk, D;
    float c2;       // scale * log2(e)
    float scale;
    void* out;
    float* lse;
    void* ws;
};
size_t attend_workspace(int64_t B, int64_t N, int64_t Hq, int64_t Hk, int64_t D);
// Whether the call's workgroups, and a workgroup's units where sequences have `slots` slots at most, are
// numbers that its kernels hold
bool attend_fits(int64_t B, int64_t N, int64_t Hq, int64_t Hk, int64_t D, int64_t slots);
hipError_t launch_attend(const AttendArgs& a, hipStream_t s);

}  // namespace tsc
