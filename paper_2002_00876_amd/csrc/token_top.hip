// token_top.hip -- the K largest logits of every row, in order, and the row's log-sum-exp.
//
// Logits are compared as 32-bit keys, a monotone image of the float (-0 counted as 0); a logit
// and its index make one 64-bit word (key, ~index), so that the words of a row are all
// different and their order is that of the result: larger logits first, equal ones by the
// lowest index.
//
// A threshold that K logits reach is found, the logits that reach it go into a list in LDS, and
// each of them finds its place there by counting the larger ones.
//   Rows of up to 8192 logits are held in registers: the threshold is found by bisection over
// all of them (k_top_short).
//   Longer rows are read once (k_top), in chunks that are each spread over the whole row.  After
// the first chunk, and as the part read grows fourfold, the threshold is guessed: a chunk that
// holds the part f of a row holds about K f of its K largest logits, and the logit of rank
// K f + 4 sqrt(K f) + 4 in it lies below the row's K-th except once in a million rows (ranks are
// taken among the maxima of groups of logits, kU groups a thread).  The vectors of logits that
// reach the guess are noted in LDS, and at the end those that do are the list, if there are K of
// them.  Where there are not, the K-th of the groups' maxima is a threshold that at least K logits
// reach, and the row is read again.
//   Where more reach it than the list holds -- many equal logits, or the largest all in a few
// groups -- the threshold is raised by bisection over the whole row, and logits equal to the
// last threshold are taken in the order of their indices.
#include <hip/hip_runtime.h>

#include "token.h"

namespace tsc {
namespace {

constexpr int kCap = 1024;   // logits that the list holds
constexpr int kU = 4;        // vectors of a chunk, and groups, a thread

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

struct TopShared {
    uint64_t list[kCap];
    float2 red[16];
    int redi[2][16];
    int n;   // words in the list, or vectors noted
};

// Number of the workgroup's keys that reach lo; `turn` alternates between calls, which makes
// one barrier enough
template <int NT, int J>
__device__ __forceinline__ int count_keys(const uint32_t (&key)[J], uint32_t lo, int turn,
                                          TopShared& sh) {
    int c = 0;
#pragma unroll
    for (int j = 0; j < J; ++j) c += __popcll(__ballot(key[j] >= lo));
    if constexpr (NT == kWave) return c;
    if (threadIdx.x % kWave == 0) sh.redi[turn & 1][threadIdx.x / kWave] = c;
    __syncthreads();
    c = 0;
#pragma unroll
    for (int w = 0; w < NT / kWave; ++w) c += sh.redi[turn & 1][w];
    return c;
}

// A threshold in [lo, hi) that at least K of the keys reach, K / 2 + 8 more at most where the
// keys allow it; lo where fewer than K reach any other.  hi: none reaches it.  count: how many
// reach the result, if it is not lo.
template <int NT, int J>
__device__ uint32_t threshold(const uint32_t (&key)[J], int K, uint32_t lo, uint32_t hi, int* count,
                              TopShared& sh) {
    int turn = 0;
    while (hi - lo > 1) {
        const uint32_t mid = lo + (hi - lo) / 2;
        const int c = count_keys<NT, J>(key, mid, turn++, sh);
        if (c >= K) {
            lo = mid;
            *count = c;
            if (c <= K + K / 2 + 8) break;
        } else {
            hi = mid;
        }
    }
    if constexpr (NT > kWave) __syncthreads();   // redi is free for the next search
    return lo;
}

// The least and the largest of the workgroup's values
template <int NT>
__device__ __forceinline__ void block_range(uint32_t* low, uint32_t* high, TopShared& sh) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        *low = min(*low, __shfl_xor(*low, o, kWave));
        *high = max(*high, __shfl_xor(*high, o, kWave));
    }
    if constexpr (NT == kWave) return;
    if (threadIdx.x % kWave == 0) {
        sh.redi[0][threadIdx.x / kWave] = (int)*low;
        sh.redi[1][threadIdx.x / kWave] = (int)*high;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NT / kWave; ++w) {
        *low = min(*low, (uint32_t)sh.redi[0][w]);
        *high = max(*high, (uint32_t)sh.redi[1][w]);
    }
    __syncthreads();
}

// The list's words each find their place among them
template <class T, int NT>
__device__ __forceinline__ void write_places(const TopArgs& a, uint32_t row, int n,
                                             const TopShared& sh) {
    T* values = (T*)a.values + (size_t)row * a.K;
    int32_t* indices = a.indices + (size_t)row * a.K;
    for (int i = threadIdx.x; i < n; i += NT) {
        const uint64_t w = sh.list[i];
        int place = 0, j = 0;
        for (; j + 4 <= n; j += 4)
#pragma unroll
            for (int k = 0; k < 4; ++k) place += sh.list[j + k] > w;
        for (; j < n; ++j) place += sh.list[j] > w;
        if (place < a.K) {
            values[place] = from_f<T>(of_key((uint32_t)(w >> 32)));
            indices[place] = (int32_t)~(uint32_t)w;
        }
    }
}

template <class T, int NT>
__device__ __forceinline__ void write_padding(const TopArgs& a, uint32_t row) {
    for (int k = threadIdx.x; k < a.K; k += NT) {
        ((T*)a.values)[(size_t)row * a.K + k] = from_f<T>(-INFINITY);
        a.indices[(size_t)row * a.K + k] = -1;
    }
    if (a.lse && threadIdx.x == 0) a.lse[row] = -INFINITY;
}

// Puts the threads' hits into the list in the order of (call, thread); have: the words in it
template <int NT>
__device__ __forceinline__ int append_ordered(bool hit, uint64_t word, int have, int most,
                                              TopShared& sh) {
    const uint64_t votes = __ballot(hit);
    int before = 0, all = __popcll(votes);
    if constexpr (NT > kWave) {
        if (threadIdx.x % kWave == 0) sh.redi[0][threadIdx.x / kWave] = all;
        __syncthreads();
        all = 0;
#pragma unroll
        for (int w = 0; w < NT / kWave; ++w) {
            if (w < (int)threadIdx.x / kWave) before += sh.redi[0][w];
            all += sh.redi[0][w];
        }
        __syncthreads();
    }
    before += have + __popcll(votes & ((1ull << (threadIdx.x % kWave)) - 1));
    if (hit && before < most) sh.list[before] = word;
    return min(have + all, most);
}

// Rows of up to NT * J logits
template <class T, int NT, int J>
__global__ __launch_bounds__(NT) void k_top_short(TopArgs a) {
    __shared__ TopShared sh;
    const int tid = threadIdx.x, K = a.K, V = a.V;
    const uint32_t rows = (uint32_t)(a.B * a.N), N = (uint32_t)a.N;
    for (uint32_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const uint32_t b = row / N, n = row % N;
        if (n >= clamp_rows(a.lengths, b, N)) {
            write_padding<T, NT>(a, row);
            continue;
        }
        const T* x = row_of<T>(a.logits, b, n);
        float v[J];
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int e = j * NT + tid;
            v[j] = e < V ? to_f(x[e]) : -INFINITY;
        }
        Soft soft = soft_empty();
        uint32_t key[J];
#pragma unroll
        for (int j = 0; j < J; ++j) {
            soft.m = fmaxf(soft.m, v[j]);
            key[j] = j * NT + tid < V ? key_of(v[j]) : 0u;   // 0: below every logit's
        }
#pragma unroll
        for (int j = 0; j < J; ++j) soft.s += exp2_((v[j] - soft.m) * a.scale.c);
        soft = block_soft<NT>(soft, a.scale.c, sh.red);
        if (a.lse && tid == 0) a.lse[row] = soft_lse(soft, a.scale.inv_t);
        int have = 0, c;
        if (V <= kCap && V <= 2 * K + 64) {   // a search would leave out little
#pragma unroll
            for (int j = 0; j < J; ++j)
                if (j * NT + tid < V) sh.list[j * NT + tid] = word_of(key[j], j * NT + tid);
            have = V;
        } else {
            c = V;
            const uint32_t lo = threshold<NT, J>(key, K, 0, key_of(INFINITY) + 1, &c, sh);
            const uint32_t first = c > kCap ? lo + 1 : lo;   // too many equal lo
            if (tid == 0) sh.n = 0;
            __syncthreads();
#pragma unroll
            for (int j = 0; j < J; ++j)
                if (key[j] >= first) sh.list[atomicAdd(&sh.n, 1)] = word_of(key[j], j * NT + tid);
            __syncthreads();
            have = sh.n;
            if (c > kCap)
                for (int j = 0; j < J && have < K; ++j) {
                    uint32_t kj = key[0];
#pragma unroll
                    for (int i = 1; i < J; ++i) kj = i == j ? key[i] : kj;
                    have = append_ordered<NT>(kj == lo, word_of(lo, j * NT + tid), have, K, sh);
                }
        }
        __syncthreads();
        write_places<T, NT>(a, row, have, sh);
        __syncthreads();   // the list is free for the next row
    }
}

// ---- longer rows ----

// Appends the row's logits whose keys reach lo, that of a finite logit, to the list, as far as it
// holds them; sh.n is their number
template <class T, int NT>
__device__ void collect(const T* row, int V, uint32_t lo, TopShared& sh) {
    if (threadIdx.x == 0) sh.n = 0;
    __syncthreads();
    const float least = of_key(lo);
    walk_row<T, NT, 4>(row, 0, V, threadIdx.x, [&](const float (&v)[kVec<T>], int at, int num) {
#pragma unroll
        for (int k = 0; k < kVec<T>; ++k)
            if (k < num && v[k] >= least) {
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
    walk_row<T, NT, 4>(row, 0, V, threadIdx.x, [&](const float (&v)[kVec<T>], int, int num) {
#pragma unroll
        for (int k = 0; k < kVec<T>; ++k) c += k < num && v[k] >= least;
    });
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) c += __shfl_xor(c, o, kWave);
    if (threadIdx.x % kWave == 0) sh.redi[0][threadIdx.x / kWave] = c;
    __syncthreads();
    c = 0;
#pragma unroll
    for (int w = 0; w < NT / kWave; ++w) c += sh.redi[0][w];
    __syncthreads();
    return c;
}

// The logits equal to the one of key `tie`, in the order of their indices, until the list has
// K words
template <class T, int NT>
__device__ int append_equal(const T* row, int V, int K, uint32_t tie, int have, TopShared& sh) {
    for (int base = 0; base < V && have < K; base += NT) {
        const int e = base + (int)threadIdx.x;
        const bool hit = e < V && key_of(to_f(row[e])) == tie;
        have = append_ordered<NT>(hit, word_of(tie, e), have, K, sh);
    }
    __syncthreads();
    return have;
}

// The list from the row itself, where more logits than it holds reach lo.  Leaves the row's K
// largest words in it and perhaps others; returns their number.
template <class T, int NT>
__device__ int select_again(const T* row, int V, int K, uint32_t lo, TopShared& sh) {
    uint32_t hi = key_of(INFINITY) + 1;
    collect<T, NT>(row, V, lo, sh);
    int c = sh.n;
    __syncthreads();
    if (c <= kCap) return c;
    uint32_t mid = lo + 1;   // the usual reason: many that equal lo
    while (hi - lo > 1 && c > kCap) {
        const int m = count_row<T, NT>(row, V, mid, sh);
        if (m >= K) {
            lo = mid;
            c = m;
        } else {
            hi = mid;
        }
        mid = lo + (hi - lo) / 2;
    }
    collect<T, NT>(row, V, c <= kCap ? lo : hi, sh);
    const int have = sh.n;
    __syncthreads();
    return c <= kCap ? have : append_equal<T, NT>(row, V, K, lo, have, sh);
}

// The threshold that K of the groups' maxima reach, at least that of key lo
template <int NT>
__device__ uint32_t group_threshold(const float (&group)[kU], int K, uint32_t lo, TopShared& sh) {
    uint32_t key[kU], low = 0xffffffffu, high = 0;
#pragma unroll
    for (int u = 0; u < kU; ++u) {
        key[u] = key_of(group[u]);
        low = min(low, key[u]);
        high = max(high, key[u]);
    }
    // the search starts between the groups' least, which all of them reach, and their largest
    block_range<NT>(&low, &high, sh);
    if (NT * kU >= K) lo = max(lo, low);
    int reach = NT * kU;
    return threshold<NT, kU>(key, K, lo, high + 1, &reach, sh);
}

template <class T, int NT>
__global__ __launch_bounds__(NT) void k_top(TopArgs a) {
    __shared__ TopShared sh;
    __shared__ int noted[kCap];   // vectors with a logit that reaches the threshold
    constexpr int W = kVec<T>, kSlots = NT / kWave * kU;
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    const int K = a.K, V = a.V, nv = V / W;
    // a unit is what a wave loads at once; chunk ch holds units ch, ch + chunks, ch + 2 chunks ...
    const int units = (nv + kWave - 1) / kWave, chunks = (units + kSlots - 1) / kSlots;
    const float c = a.scale.c;
    const uint32_t rows = (uint32_t)(a.B * a.N), N = (uint32_t)a.N;
    const uint32_t finite = key_of(-FLT_MAX);   // -inf is none of the K largest before every
                                                // finite logit is
    for (uint32_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const uint32_t b = row / N, n = row % N;
        if (n >= clamp_rows(a.lengths, b, N)) {
            write_padding<T, NT>(a, row);
            continue;
        }
        const T* x = row_of<T>(a.logits, b, n);
        if (tid == 0) sh.n = 0;
        __syncthreads();
        ChunkSoft soft;
        soft.init(c);
        float group[kU], least = -FLT_MAX;
#pragma unroll
        for (int u = 0; u < kU; ++u) group[u] = -INFINITY;
        uint32_t lo = finite;   // the threshold's key
        int next = 0;           // the chunk after which it is guessed again
        auto note = [&](int i) {
            const int at = atomicAdd(&sh.n, 1);
            if (at < kCap) noted[at] = i;
        };
        auto chunk = [&](auto whole, int ch) {
            constexpr bool kWhole = decltype(whole)::value;
            const int i0 = (wave * kU * chunks + ch) * kWave + lane, step = chunks * kWave;
            Raw<T> r[kU];
            float top[kU];
#pragma unroll
            for (int u = 0; u < kU; ++u)
                if (kWhole || i0 + u * step < nv)
                    r[u] = *(const Raw<T>*)((const char*)x + (uint32_t)(i0 + u * step) * 16u);
#pragma unroll
            for (int h = 0; h < kU; h += 2) {
                float v[2][W];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    top[h + u] = -INFINITY;
                    if (kWhole || i0 + (h + u) * step < nv) {
                        unpack<T>(r[h + u], v[u]);
                        top[h + u] = max_of(v[u]);
                    }
                    group[h + u] = fmaxf(group[h + u], top[h + u]);
                }
                soft.raise(fmaxf(top[h], top[h + 1]), c);
#pragma unroll
                for (int u = 0; u < 2; ++u)
                    if (kWhole || i0 + (h + u) * step < nv) soft.push(v[u], c);
            }
            if (ch == next) {
                const float part = K * (float)(ch + 1) / (float)chunks;
                const int rank = min(K, (int)(part + 4.f * sqrtf(part) + 4.f));
                lo = group_threshold<NT>(group, rank, lo, sh);
                least = of_key(lo);
                next = 4 * ch + 3;
            }
#pragma unroll
            for (int u = 0; u < kU; ++u)
                if (top[u] >= least) note(i0 + u * step);
        };
        // all units of the last slot's chunks [0, full) are whole
        const int full = nv / kWave - (kSlots - 1) * chunks;
        for (int ch = 0; ch < min(full, chunks); ++ch) chunk(std::true_type{}, ch);
        for (int ch = max(full, 0); ch < chunks; ++ch) chunk(std::false_type{}, ch);
        const int e = nv * W + tid;   // the row's last few logits, always in the list
        const float last = e < V ? to_f(x[e]) : -INFINITY;
        float one[1] = {last};
        soft.raise(last, c);
        soft.push(one, c);
        const float mine = fmaxf(fmaxf(fmaxf(group[0], group[1]), fmaxf(group[2], group[3])), last);
        Soft all = block_soft<NT>(soft.value(c), c, sh.red);
        if (far(block_max<NT>(mine, (float*)sh.red))) {
            Soft again = soft_empty();
            walk_row<T, NT, 4>(x, 0, V, tid,
                               [&](const float (&v)[W], int, int) { soft_push(again, v, c); });
            all = block_soft<NT>(again, c, sh.red);
        }
        if (a.lse && tid == 0) a.lse[row] = soft_lse(all, a.scale.inv_t);
        // the noted vectors' logits that reach the last threshold
        const int vectors = sh.n;
        __syncthreads();
        if (tid == 0) sh.n = 0;
        __syncthreads();
        auto append = [&](float v, int at) {
            const int i = atomicAdd(&sh.n, 1);
            if (i < kCap) sh.list[i] = word_of(key_of(v), at);
        };
        if (last >= least) append(last, e);
        for (int i = tid; i < min(vectors, kCap); i += NT) {
            float v[W];
            unpack<T>(*(const Raw<T>*)(x + (size_t)noted[i] * W), v);
#pragma unroll
            for (int k = 0; k < W; ++k)
                if (v[k] >= least) append(v[k], noted[i] * W + k);
        }
        __syncthreads();
        int have = sh.n;
        __syncthreads();
        if (vectors > kCap || have > kCap || (have < K && lo > finite)) {
            lo = group_threshold<NT>(group, K, finite, sh);
            have = select_again<T, NT>(x, V, K, lo, sh);
        }
        if (have < K) have = append_equal<T, NT>(x, V, K, key_of(-INFINITY), have, sh);
        write_places<T, NT>(a, row, have, sh);
        __syncthreads();   // the list is free for the next row
    }
}

}  // namespace

size_t top_workspace(int64_t, int64_t, int64_t, int64_t) { return 0; }

hipError_t launch_top(const TopArgs& a, hipStream_t s) {
    with_type(a.dtype, [&](auto t) {
        using T = decltype(t);
        const int64_t rows = a.B * a.N;
        const unsigned g1 = row_grid(rows, 64), g4 = row_grid(rows, 256);
        if (a.V <= 64)
            k_top_short<T, 64, 1><<<g1, 64, 0, s>>>(a);
        else if (a.V <= 256)
            k_top_short<T, 64, 4><<<g1, 64, 0, s>>>(a);
        else if (a.V <= 1024)
            k_top_short<T, 64, 16><<<g1, 64, 0, s>>>(a);
        else if (a.V <= 4096)
            k_top_short<T, 256, 16><<<g4, 256, 0, s>>>(a);
        else if (a.V <= 8192)
            k_top_short<T, 256, 32><<<g4, 256, 0, s>>>(a);
        else
            k_top<T, 256><<<g4, 256, 0, s>>>(a);
    });
    return hipGetLastError();
}

}  // namespace tsc
