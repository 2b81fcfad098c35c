// cache.h -- device pieces shared by the kernels on a paged cache.  Not part of the public interface.
#pragma once
#include "cache_calls.h"
#include "token.h"

namespace tsc {

__device__ __forceinline__ int clamp_to(int x, int hi) { return x < 0 ? 0 : (x > hi ? hi : x); }

// New tokens of a sequence, and its slots that are taken before them
__device__ __forceinline__ int new_tokens(const Cache& c, int64_t b, int N) {
    return c.lengths ? clamp_to(c.lengths[b], N) : N;
}
__device__ __forceinline__ int slots_before(const Cache& c, int64_t b) {
    return clamp_to(c.starts[b], c.M * c.S);
}

// Slot j's page, counted in its sequence's, and its place there
__device__ __forceinline__ int page_of(const Cache& c, int j, int* at) {
    int page = (int)__umulhi((uint32_t)j, c.inv);
    *at = j - page * c.S;
    if (*at >= c.S) ++page, *at -= c.S;
    return page;
}
// Elements from the caches' start to token `at` of page id (of head 0); -1: it is not there
__device__ __forceinline__ int64_t token_offset(const Cache& c, int id, int at) {
    return id >= 0 && id < c.P ? id * c.sp + at * c.st : -1;
}

}  // namespace tsc
