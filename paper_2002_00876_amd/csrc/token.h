// token.h -- device pieces shared by the kernels on rows of token logits: element types, the
// walk over a row, the running maximum and sum of its softmax, and workgroup reductions.
// Not part of the public interface.
//
// Exponents are base 2: with a = log2(e) / T a row's probabilities are
// 2^(a (x_v - m)) / s, m the row's maximum and s the sum of the numerators.  The difference to
// m is taken before the product, so that what is rounded stays small for the tokens that count.
#pragma once
#include <float.h>
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "device.h"
#include "token_calls.h"
#include "ts_token.h"

namespace tsc {

constexpr int kMaxVocab = 1 << 19;   // one bit a token fits 64 KiB of LDS
constexpr int kMaxTop = 256;

struct Bf16 {
    uint16_t u;
};
struct F16 {
    uint16_t u;
};

// A row of logits is read 16 bytes a lane at whatever address it starts: rows of an odd
// vocabulary are aligned to their elements only, which gfx950 loads as they are.
template <class T>
struct __attribute__((packed, aligned(sizeof(T)))) Raw {
    uint32_t w[4];
};

template <class T>
constexpr int kVec = 16 / (int)sizeof(T);

typedef uint32_t Vec4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t Vec2 __attribute__((ext_vector_type(4), aligned(2)));

// Reads a vector.  kOnce: nothing will read it again, so it is not kept in the caches: a walk over
// 2 GiB reads 7.0 TB/s so, and 6.2 otherwise.
template <class T, bool kOnce>
__device__ __forceinline__ Raw<T> load_raw(const T* at) {
    using Vec = std::conditional_t<sizeof(T) == 4, Vec4, Vec2>;
    Vec v;
    if constexpr (kOnce)
        v = __builtin_nontemporal_load((const Vec*)at);
    else
        v = *(const Vec*)at;
    return {{v.x, v.y, v.z, v.w}};
}

// Stores a vector that nothing will read soon
template <class T>
__device__ __forceinline__ void store_raw(T* at, const Raw<T>& r) {
    using Vec = std::conditional_t<sizeof(T) == 4, Vec4, Vec2>;
    __builtin_nontemporal_store(Vec{r.w[0], r.w[1], r.w[2], r.w[3]}, (Vec*)at);
}

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(Bf16 x) { return __uint_as_float((uint32_t)x.u << 16); }
__device__ __forceinline__ float to_f(F16 x) { return (float)__builtin_bit_cast(_Float16, x.u); }

template <class T>
__device__ __forceinline__ T from_f(float x);
template <>
__device__ __forceinline__ float from_f<float>(float x) {
    return x;
}
template <>
__device__ __forceinline__ Bf16 from_f<Bf16>(float x) {   // nearest, ties to even
    return {__builtin_bit_cast(uint16_t, (__bf16)x)};
}
template <>
__device__ __forceinline__ F16 from_f<F16>(float x) {
    return {__builtin_bit_cast(uint16_t, (_Float16)x)};
}

template <class T>
__device__ __forceinline__ void unpack(const Raw<T>& r, float (&v)[kVec<T>]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(r.w[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = to_f(T{(uint16_t)(r.w[i] & 0xffff)});
            v[2 * i + 1] = to_f(T{(uint16_t)(r.w[i] >> 16)});
        }
    }
}
template <class T>
__device__ __forceinline__ Raw<T> pack(const float (&v)[kVec<T>]) {
    Raw<T> r;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) r.w[i] = __float_as_uint(v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            r.w[i] = (uint32_t)from_f<T>(v[2 * i]).u | (uint32_t)from_f<T>(v[2 * i + 1]).u << 16;
    }
    return r;
}

// Reads elements [lo, hi) of a row with NT threads, U vectors a thread in flight:
// f(values, first index, number) with number = kVec<T>, or 1 for the last few elements (the
// other values then are -inf).
template <class T, int NT, int U, bool kOnce = false, class F>
__device__ __forceinline__ void walk_row(const T* row, int lo, int hi, int tid, F f) {
    constexpr int W = kVec<T>;
    const int nv = (hi - lo) / W;
    const T* p = row + lo;
    int i = tid;
    for (; i + (U - 1) * NT < nv; i += U * NT) {
        Raw<T> r[U];
#pragma unroll
        for (int u = 0; u < U; ++u) r[u] = load_raw<T, kOnce>(p + (size_t)(i + u * NT) * W);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float v[W];
            unpack<T>(r[u], v);
            f(v, lo + (i + u * NT) * W, W);
        }
    }
    for (; i < nv; i += NT) {
        const Raw<T> r = load_raw<T, kOnce>(p + (size_t)i * W);
        float v[W];
        unpack<T>(r, v);
        f(v, lo + i * W, W);
    }
    const int e = lo + nv * W + tid;
    if (e < hi) {
        float v[W];
#pragma unroll
        for (int k = 1; k < W; ++k) v[k] = -INFINITY;
        v[0] = to_f(row[e]);
        f(v, e, 1);
    }
}

// The same of what nothing will read again.  Rows that start within a vector are read through the
// caches all the same: two waves share the line between them, and it would be fetched for each
// (statistics of 1150 rows of 100003 bfloat16: 60 us, 52 through the caches).
template <class T, int NT, int U, class F>
__device__ __forceinline__ void walk_once(const T* row, int lo, int hi, int tid, F f) {
    if (reinterpret_cast<uintptr_t>(row + lo) % 16 == 0)
        walk_row<T, NT, U, true>(row, lo, hi, tid, f);
    else
        walk_row<T, NT, U, false>(row, lo, hi, tid, f);
}

// Running maximum and sum of numerators.  Sums are not contracted, so that kernels which share these
// give the same bits, however each of them is compiled.  The empty state's maximum is the lowest float, not
// -inf, so that differences to it are never NaN.
struct Soft {
    float m, s;
};
__device__ __forceinline__ Soft soft_empty() { return {-FLT_MAX, 0.f}; }
__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float exp_(float x) { return exp2_(x * 1.44269504f); }
template <int W>
__device__ __forceinline__ void soft_push(Soft& a, const float (&v)[W], float c) {
#pragma clang fp contract(off)
    float m = a.m;
#pragma unroll
    for (int k = 0; k < W; ++k) m = fmaxf(m, v[k]);
    float s = a.s * exp2_((a.m - m) * c);
#pragma unroll
    for (int k = 0; k < W; ++k) s += exp2_((v[k] - m) * c);
    a = {m, s};
}
__device__ __forceinline__ Soft soft_merge(Soft a, Soft b, float c) {
#pragma clang fp contract(off)
    const float m = fmaxf(a.m, b.m);
    return {m, a.s * exp2_((a.m - m) * c) + b.s * exp2_((b.m - m) * c)};
}
__device__ __forceinline__ Soft wave_soft(Soft a, float c) {
#pragma clang fp contract(off)
    const float m = wave_max_fast(a.m);
    return {m, wave_sum_fast(a.s * exp2_((a.m - m) * c))};
}
// Every thread gets the workgroup's; red holds NT / 64 pairs and is free again on return.  The
// waves' results are joined by the lanes of each wave (read by every thread for itself, sixteen
// of them would take the registers of a vector each).
template <int NT>
__device__ __forceinline__ Soft block_soft(Soft a, float c, float2* red) {
    a = wave_soft(a, c);
    if constexpr (NT == kWave) return a;
    const int lane = threadIdx.x % kWave;
    if (lane == 0) red[threadIdx.x / kWave] = make_float2(a.m, a.s);
    __syncthreads();
    const float2 r = lane < NT / kWave ? red[lane] : make_float2(-FLT_MAX, 0.f);
    __syncthreads();
    return wave_soft({r.x, r.y}, c);
}
template <int NT>
__device__ __forceinline__ float block_sum(float x, float* red) {
    x = wave_sum_fast(x);
    if constexpr (NT == kWave) return x;
    const int lane = threadIdx.x % kWave;
    if (lane == 0) red[threadIdx.x / kWave] = x;
    __syncthreads();
    const float r = lane < NT / kWave ? red[lane] : 0.f;
    __syncthreads();
    return wave_sum_fast(r);
}
template <int NT>
__device__ __forceinline__ float block_max(float x, float* red) {
    x = wave_max_fast(x);
    if constexpr (NT == kWave) return x;
    const int lane = threadIdx.x % kWave;
    if (lane == 0) red[threadIdx.x / kWave] = x;
    __syncthreads();
    const float r = lane < NT / kWave ? red[lane] : -INFINITY;
    __syncthreads();
    return wave_max_fast(r);
}

// The same for whole chunks of a row, at one fma, one exponential and one sum a logit: the
// maximum is brought up to date once a chunk, and numerators are 2^(v c - r), r = m c rounded.
// What r is rounded by is common to all numerators and goes into the sum when the pair is read
// off (value()), so a numerator's exponent is rounded once, as a difference.  |m c| <= 2^29 keeps
// that rounding within 32, so that numerators and their sums stay far inside the floats: a thread
// begins at m = -k.most (|m c| = 2^29), below which tokens count for nothing beside a row's
// maximum that is not itself beyond it.  Rows whose maximum lies beyond +-k.most (3.7e8 at T = 1)
// are walked again, by soft_push, and what was summed here is dropped.
struct ChunkSoft {
    float m, r, s;
    __device__ __forceinline__ void init(const Scale& k) {
#pragma clang fp contract(off)
        m = -k.most, r = m * k.c, s = 0.f;
    }
    __device__ __forceinline__ void raise(float most, float c) {
#pragma clang fp contract(off)
        if (most > m) {
            const float r2 = most * c;
            s *= exp2_(r - r2);
            m = most;
            r = r2;
        }
    }
    template <int W>
    __device__ __forceinline__ void push(const float (&v)[W], float c) {
#pragma clang fp contract(off)
        float t[W];
#pragma unroll
        for (int k = 0; k < W; ++k) t[k] = exp2_(fmaf(v[k], c, -r));
#pragma unroll
        for (int d = W / 2; d > 0; d /= 2)
#pragma unroll
            for (int k = 0; k < d; ++k) t[k] += t[k + d];
        s += t[0];
    }
    __device__ __forceinline__ Soft value(float c) const {
#pragma clang fp contract(off)
        // 2^(v c - r) = 2^((v - m) c) 2^(m c - r).  A thread that has summed nothing (rows shorter than
        // a wave's vectors, parts that end, masked stretches) is empty.
        return s > 0.f ? Soft{m, s * exp2_(-fmaf(m, c, -r))} : soft_empty();
    }
};
__device__ __forceinline__ bool far(float most, const Scale& k) { return !(fabsf(most) <= k.most); }

template <int W>
__device__ __forceinline__ float max_of(const float (&v)[W]) {
    float a = fmaxf(v[0], fmaxf(v[1], v[2]));
    if constexpr (W == 4) {
        return fmaxf(a, v[3]);
    } else {
        const float b = fmaxf(v[3], fmaxf(v[4], v[5]));
        return fmaxf(a, fmaxf(b, fmaxf(v[6], v[7])));
    }
}

// The same with the entropy's sum beside it: t = sum of d 2^d over exponents d = (x - m) c, none of them
// positive, so that the row's entropy log s - t ln 2 / s is made of two terms that are not negative.
// Exponents below -200, whose numerators are 0, count as that: 0 times -inf would be no number.
//
// What the others of a row with a nearly certain token add up to keeps its digits: one of the largest logits is
// left out of the sum (log s then is log1p of it; t has nothing of that logit anyway).  Where none is, s is
// negative, -0 in the empty state, and its magnitude is the whole sum.
struct Spread {
    float m, s, t;
    __device__ __forceinline__ bool whole() const { return __float_as_int(s) < 0; }
    __device__ __forceinline__ float sum() const { return whole() ? -s : 1.f + s; }
    // What all but one of the largest add up to
    __device__ __forceinline__ float rest() const { return whole() ? -s - 1.f : s; }
};
constexpr float kNoTerm = -200.f;
constexpr float kLn2 = 0.693147180559945f;
__device__ __forceinline__ Spread spread_empty() { return {-FLT_MAX, -0.f, 0.f}; }
// The sums beside a larger logit, which is the one that is left out then
__device__ __forceinline__ Spread spread_raise(Spread a, float m, float c) {
#pragma clang fp contract(off)
    const float d = fmaxf((a.m - m) * c, kNoTerm), f = exp2_(d), s = a.sum();
    return {m, s * f, (a.t + s * d) * f};
}
// Takes the first logit that is `most` out
template <int W>
__device__ __forceinline__ void leave_first_out(float (&v)[W], float most) {
    bool left = false;
#pragma unroll
    for (int k = 0; k < W; ++k) {
        const bool it = !left && v[k] == most;
        v[k] = it ? -INFINITY : v[k];
        left |= it;
    }
}
// Whether the calling lane is the first of those that say so
__device__ __forceinline__ bool first_lane(bool yes) {
    const uint64_t votes = __ballot(yes);
    return yes && __builtin_amdgcn_mbcnt_hi((uint32_t)(votes >> 32),
                                            __builtin_amdgcn_mbcnt_lo((uint32_t)votes, 0)) == 0;
}
template <int W>
__device__ __forceinline__ void spread_push(Spread& a, const float (&x)[W], float c) {
#pragma clang fp contract(off)
    float v[W], most = x[0];
#pragma unroll
    for (int k = 0; k < W; ++k) v[k] = x[k], most = fmaxf(most, x[k]);
    if (most > a.m || (a.whole() && most == a.m)) {
        a = spread_raise(a, most, c);
        leave_first_out(v, most);
    }
    if (a.whole()) return;   // no logit yet but -inf
#pragma unroll
    for (int k = 0; k < W; ++k) {
        const float d = fmaxf((v[k] - a.m) * c, kNoTerm), e = exp2_(d);
        a.s += e;
        a.t += d * e;
    }
}
__device__ __forceinline__ Spread wave_spread(Spread a, float c) {
#pragma clang fp contract(off)
    const float m = wave_max_fast(a.m);
    const bool one = a.m == m && !a.whole(), leaves = first_lane(one);
    const Spread b = spread_raise(a, m, c);
    const float s = wave_sum_fast(leaves ? a.s : b.s);
    return {m, __any(one) ? s : -s, wave_sum_fast(b.t)};
}
// Every thread gets the workgroup's from its waves'; red holds NT / 64 of them and is free again on return
template <int NT>
__device__ __forceinline__ Spread join_spread(Spread a, float c, float4* red) {
    if constexpr (NT == kWave) return a;
    const int lane = threadIdx.x % kWave;
    if (lane == 0) red[threadIdx.x / kWave] = make_float4(a.m, a.s, a.t, 0.f);
    __syncthreads();
    const float4 r = lane < NT / kWave ? red[lane] : make_float4(-FLT_MAX, -0.f, 0.f, 0.f);
    __syncthreads();
    return wave_spread({r.x, r.y, r.z}, c);
}
template <int NT>
__device__ __forceinline__ Spread block_spread(Spread a, float c, float4* red) {
    return join_spread<NT>(wave_spread(a, c), c, red);
}

// Numerators 2^(v c - r) of a chunk, and their products with the exponents, to the sums of them
template <int W>
__device__ __forceinline__ void push_chunk(const float (&v)[W], float c, float r, float& s, float& t) {
    float e[W];
#pragma unroll
    for (int k = 0; k < W; ++k) {
        const float d = fmaxf(fmaf(v[k], c, -r), kNoTerm);
        e[k] = exp2_(d);
        t = fmaf(d, e[k], t);
    }
#pragma unroll
    for (int d = W / 2; d > 0; d /= 2)
#pragma unroll
        for (int k = 0; k < d; ++k) e[k] += e[k + d];
    s += e[0];
}

// ChunkSoft's sums with the entropy's, of vectors of T of a whole wave, whose lanes have one maximum and call all
// this together: it is hardly ever raised.  The vectors with the maximum are not pushed by the lane that has them
// but wait as `words`, a word a lane, to be summed when they have it no longer, or without one m in the end.  (The
// scan of top logits with it, 4096 rows of 131072 and 3000 of 32000 bfloat16: 185 and 45.9 us; with lanes that
// each take a logit out of 16 at every raise of their own 191 and 48.2; with sums that leave none out and have no
// digits beside 1 185 and 44.4.)
template <class T>
struct WaveSpread {
    float m, r, s, t;
    uint32_t words;
    static constexpr int kEach = 4 / sizeof(T);   // logits of a word; -inf: nothing
    static constexpr uint32_t kNothing = kEach == 1 ? 0xff800000u : std::is_same_v<T, Bf16> ? 0xff80ff80u : 0xfc00fc00u;
    // reached: what some logit of the row is known to reach; m begins just below that
    __device__ __forceinline__ void init(const Scale& k, float reached) {
#pragma clang fp contract(off)
        const float below = reached - fmaxf(fabsf(reached) * 0x1p-22f, 1e-30f);
        m = fminf(fmaxf(below, -k.most), k.most), r = m * k.c, s = t = 0.f;
        words = kNothing;
    }
    __device__ __forceinline__ void logits(float (&v)[kEach]) const {
#pragma unroll
        for (int k = 0; k < kEach; ++k)
            if constexpr (kEach == 1)
                v[k] = __uint_as_float(words);
            else
                v[k] = to_f(T{(uint16_t)(words >> 16 * k)});
    }
    // Before the vectors q are pushed, whose largest logit is `most` (but for the one at `skip`, which is not
    // pushed either); where it says so, pushed() follows
    template <int U>
    __device__ __forceinline__ bool raise(const Raw<T> (&q)[U], float most, float c, int skip = -1) {
#pragma clang fp contract(off)
        if (!__any(most > m)) return false;
        const float top = wave_max_fast(most), r2 = top * c, d = fmaxf(r - r2, kNoTerm), f = exp2_(d);
        float v[kEach];
        logits(v);
        t = (t + s * d) * f;
        s *= f;
        m = top, r = r2;
        push_chunk(v, c, r, s, t);
        const int lane = threadIdx.x % kWave, who = __builtin_ctzll(__ballot(most == top));
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t x = __builtin_amdgcn_readlane(q[u].w[k], who);
                words = lane == u * 4 + k ? x : words;
            }
        if (U == 1 && lane >= 4) words = kNothing;
        skip = __builtin_amdgcn_readlane(skip, who);
        if (kEach == 1) {
            if (lane == skip) words = kNothing;
        } else if (skip >= 0 && lane == skip / 2) {
            words = skip & 1 ? (words & 0xffffu) | (kNothing & 0xffff0000u) : (words & 0xffff0000u) | (kNothing & 0xffffu);
        }
        if (lane == who) r = INFINITY;   // nothing of its vectors then has a numerator
        return true;
    }
    __device__ __forceinline__ void pushed(float c) {
#pragma clang fp contract(off)
        r = m * c;
    }
    template <int W>
    __device__ __forceinline__ void push(const float (&v)[W], float c) {
        push_chunk(v, c, r, s, t);
    }
    // The wave's
    __device__ __forceinline__ Spread value(float c) {
#pragma clang fp contract(off)
        float v[kEach];
        logits(v);
        bool top = false;
#pragma unroll
        for (int k = 0; k < kEach; ++k) top |= v[k] == m;
        const bool one = __any(top);
        if (first_lane(top)) leave_first_out(v, m);
        push_chunk(v, c, r, s, t);
        s = wave_sum_fast(s);
        t = wave_sum_fast(t);
        if (!one && !(s > 0.f)) return spread_empty();
        const float d = -fmaf(m, c, -r), f = exp2_(d);
        return {m, one ? s * f : -(s * f), (t + s * d) * f};
    }
};

// log(1 + x), x >= 0.  Up to 1/2: 2 atanh(x / (2 + x)) by its series, whose first term left out is below 2^-26 of it
// (log1pf, for any x, takes a row of 300 tokens 14 % of its time).
__device__ __forceinline__ float log1p_(float x) {
    if (x > 0.5f) return logf(1.f + x);
    const float s = x * __builtin_amdgcn_rcpf(2.f + x), q = s * s;
    return 2.f * s * fmaf(q, fmaf(q, fmaf(q, fmaf(q, 1.f / 9, 1.f / 7), 1.f / 5), 1.f / 3), 1.f);
}

// What a row's scores are made of, from the sums of its softmax: log p_v = (x_v - m) / T - ls, and the
// entropy.  (A rest below 0 is rounding, or that of a row without a finite logit, which has no p: its log p are
// -inf, its entropy 0.)
struct RowScore {
    float m, ls, below, entropy;   // below: the entropy less log s
    __device__ __forceinline__ explicit RowScore(Spread a)
        : m(a.m), ls(log1p_(fmaxf(a.rest(), 0.f))), below(-kLn2 * fminf(a.t, 0.f) / fmaxf(a.sum(), 1.f)),
          entropy(ls + below) {}
    __device__ __forceinline__ float logp(float x, float inv_t) const { return (x - m) * inv_t - ls; }
};

// log sum exp(x / T) of a row; -inf where it has no finite logit
__device__ __forceinline__ float soft_lse(Soft a, float inv_t) {
    return a.s > 0.f ? fmaf(a.m, inv_t, logf(a.s)) : -INFINITY;
}

__device__ __forceinline__ int64_t clamp_rows(const int32_t* lengths, int64_t b, int64_t N) {
    if (!lengths) return N;
    const int64_t L = lengths[b];
    return L < 0 ? 0 : (L > N ? N : L);
}

template <class T>
__device__ __forceinline__ const T* row_of(const Rows& x, int64_t b, int64_t n) {
    return (const T*)x.p + b * x.sb + n * x.sn;
}

// i / d of an item i < items: in 32 bits where they do, as 64-bit divisions take as long as a small
// part of a row
__device__ __forceinline__ uint32_t item_row(uint64_t i, int d, uint64_t items) {
    return items >> 32 ? (uint32_t)(i / (uint64_t)d) : (uint32_t)i / (uint32_t)d;
}

// A launch holds fewer than 2^32 threads: kernels walk the rows with this many workgroups
inline unsigned row_grid(int64_t rows, int threads) {
    const int64_t most = (int64_t)0xffffffff / threads;
    return (unsigned)(rows < most ? rows : most);
}

// Calls f with a value of the element type that dtype names
template <class F>
inline auto with_type(int dtype, F f) {
    switch (dtype) {
        case TS_FLOAT32: return f(float{});
        case TS_BFLOAT16: return f(Bf16{});
        default: return f(F16{});
    }
}

}  // namespace tsc
