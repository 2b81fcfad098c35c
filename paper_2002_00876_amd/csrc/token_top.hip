// token_top.hip -- the K largest logits of every row, in order, and the row's log-sum-exp.
//
// Logits are compared as 32-bit keys, a monotone image of the float (-0 counted as 0); a logit
// and its index make one 64-bit word (key, ~index), so that the words of a row are all
// different and their order is that of the result: larger logits first, equal ones by the
// lowest index.
//
// One workgroup takes a row.  The first walk keeps every thread's largest key and the running
// maximum and sum of the softmax.  A threshold that at least K of the threads' largest keys
// reach is one that at least K logits reach; as the K largest rarely share threads, few more
// do (of 1024 threads' maxima the 256th is reached by some 300 logits).  The second walk
// collects the logits that reach it, and each of them finds its place among them by counting.
// Where more reach it than the list holds -- many equal logits, or the largest all in a few
// threads -- the threshold is raised by bisection over the whole row, and logits equal to the
// last threshold are taken in the order of their indices.
#include <hip/hip_runtime.h>

#include "token.h"

namespace tsc {
namespace {

constexpr int kCap = 1024;   // logits that the list holds

__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t u = __float_as_uint(x + 0.0f);   // -0 + 0 = 0
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float of_key(uint32_t k) {
    return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}
__device__ __forceinline__ uint64_t word_of(uint32_t key, int index) {
    return (uint64_t)key << 32 | (uint32_t)~index;
}

template <int NT>
__device__ __forceinline__ int block_count(bool x) {
    if constexpr (NT == kWave) return __popcll(__ballot(x));
    return __syncthreads_count(x);
}
template <int NT>
__device__ __forceinline__ int block_sum_int(int x, int* red) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, kWave);
    if constexpr (NT == kWave) return x;
    if (threadIdx.x % kWave == 0) red[threadIdx.x / kWave] = x;
    __syncthreads();
    int s = 0;
#pragma unroll
    for (int w = 0; w < NT / kWave; ++w) s += red[w];
    __syncthreads();
    return s;
}

struct TopShared {
    uint64_t list[kCap];
    float2 red[16];
    int redi[16];
    int n;
};

// Appends the row's logits whose keys reach lo to the list, as far as it holds them; sh.n is
// their number
template <class T, int NT>
__device__ void collect(const T* row, int V, uint32_t lo, TopShared& sh) {
    if (threadIdx.x == 0) sh.n = 0;
    __syncthreads();
    const float least = of_key(lo);
    walk_row<T, NT, 4>(row, 0, V, threadIdx.x, [&](const float* v, int at, int num) {
#pragma unroll
        for (int k = 0; k < kVec<T>; ++k)
            if (k < num && (lo == 0 || v[k] >= least)) {
                const int i = atomicAdd(&sh.n, 1);
                if (i < kCap) sh.list[i] = word_of(key_of(v[k]), at + k);
            }
    });
    __syncthreads();
}

template <class T, int NT>
__device__ int count_row(const T* row, int V, uint32_t lo, TopShared& sh) {
    int c = 0;
    const float least = of_key(lo);
    walk_row<T, NT, 4>(row, 0, V, threadIdx.x, [&](const float* v, int, int num) {
#pragma unroll
        for (int k = 0; k < kVec<T>; ++k) c += k < num && v[k] >= least;
    });
    return block_sum_int<NT>(c, sh.redi);
}

// The largest threshold found that K of the threads' keys reach, 0 where fewer than K threads
// have one
template <int NT>
__device__ uint32_t threshold(uint32_t key, int K) {
    uint32_t lo = 0, hi = 0xffffffffu;
    while (hi - lo > 1) {
        const uint32_t mid = lo + (hi - lo) / 2;
        const int c = block_count<NT>(key >= mid);
        if (c >= K) {
            lo = mid;
            if (c <= K + K / 4) break;
        } else {
            hi = mid;
        }
    }
    return lo;
}

// Leaves in the list the row's K largest words and perhaps others, and in sh.n their number
template <class T, int NT>
__device__ void select(const T* row, int V, int K, uint32_t lo, TopShared& sh) {
    collect<T, NT>(row, V, lo, sh);
    const int n = sh.n;
    __syncthreads();
    if (n <= kCap) return;
    // more than the list holds reach lo, and none reaches the key of +inf's successor
    uint32_t hi = key_of(INFINITY) + 1;
    int c = n;
    while (hi - lo > 1 && c > kCap) {
        const uint32_t mid = lo + (hi - lo) / 2;
        const int m = count_row<T, NT>(row, V, mid, sh);
        if (m >= K) {
            lo = mid;
            c = m;
        } else {
            hi = mid;
        }
    }
    if (c <= kCap) {
        collect<T, NT>(row, V, lo, sh);
        return;
    }
    // fewer than K logits lie above lo, and more equal it than the list holds: the first ones
    collect<T, NT>(row, V, hi, sh);
    int have = sh.n;
    __syncthreads();
    for (int base = 0; base < V && have < K; base += NT) {
        const int e = base + (int)threadIdx.x;
        const bool hit = e < V && key_of(to_f(row[e])) == lo;
        const uint64_t votes = __ballot(hit);
        if (threadIdx.x % kWave == 0) sh.redi[threadIdx.x / kWave] = __popcll(votes);
        __syncthreads();
        int before = 0, all = 0;
        for (int w = 0; w < NT / kWave; ++w) {
            if (w < (int)threadIdx.x / kWave) before += sh.redi[w];
            all += sh.redi[w];
        }
        before += __popcll(votes & ((1ull << (threadIdx.x % kWave)) - 1));
        if (hit && have + before < K) sh.list[have + before] = word_of(lo, e);
        have += all;
        __syncthreads();
    }
    if (threadIdx.x == 0) sh.n = have < K ? have : K;
    __syncthreads();
}

template <class T, int NT>
__global__ __launch_bounds__(NT) void k_top(TopArgs a) {
    __shared__ TopShared sh;
    const int tid = threadIdx.x, K = a.K;
    for (int64_t row = blockIdx.x; row < a.B * a.N; row += gridDim.x) {
        const int64_t b = row / a.N, n = row % a.N;
        T* values = (T*)a.values + row * K;
        int32_t* indices = a.indices + row * K;
        if (n >= clamp_rows(a.lengths, b, a.N)) {
            for (int k = tid; k < K; k += NT) {
                values[k] = from_f<T>(-INFINITY);
                indices[k] = -1;
            }
            if (a.lse && tid == 0) a.lse[row] = -INFINITY;
            continue;
        }
        const T* x = row_of<T>(a.logits, b, n);
        Soft soft = soft_empty();
        float most = -INFINITY;
        bool any = false;
        walk_row<T, NT, 4>(x, 0, a.V, tid, [&](const float (&v)[kVec<T>], int, int) {
            soft_push(soft, v, a.scale.c);
#pragma unroll
            for (int k = 0; k < kVec<T>; ++k) most = fmaxf(most, v[k]);
            any = true;
        });
        soft = block_soft<NT>(soft, a.scale.c, sh.red);
        if (a.lse && tid == 0) a.lse[row] = soft_lse(soft, a.scale.inv_t);
        const uint32_t lo = a.V <= 128 ? 0 : threshold<NT>(any ? key_of(most) : 0, K);
        select<T, NT>(x, a.V, K, lo, sh);
        const int c = sh.n;
        for (int i = tid; i < c; i += NT) {
            const uint64_t w = sh.list[i];
            int place = 0;
            for (int j = 0; j < c; ++j) place += sh.list[j] > w;
            if (place < K) {
                values[place] = from_f<T>(of_key((uint32_t)(w >> 32)));
                indices[place] = (int32_t)~(uint32_t)w;
            }
        }
        __syncthreads();   // the list is free for the next row
    }
}

}  // namespace

size_t top_workspace(int64_t, int64_t, int64_t, int64_t) { return 0; }

hipError_t launch_top(const TopArgs& a, hipStream_t s) {
    with_type(a.dtype, [&](auto t) {
        using T = decltype(t);
        const int64_t rows = a.B * a.N;
        if (a.V <= 512)
            k_top<T, 64><<<row_grid(rows, 64), 64, 0, s>>>(a);
        else if (a.V <= 8192)
            k_top<T, 256><<<row_grid(rows, 256), 256, 0, s>>>(a);
        else
            k_top<T, 1024><<<row_grid(rows, 1024), 1024, 0, s>>>(a);
    });
    return hipGetLastError();
}

}  // namespace tsc
