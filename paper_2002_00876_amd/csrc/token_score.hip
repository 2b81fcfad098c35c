// token_score.hip -- log-probabilities of given tokens and rows' entropies without alternatives, and
// their gradient.  (With alternatives the kernels of token_top.hip make them on their way.)
//
// With p = softmax(x / T), L = log p_z and H = - sum_v p_v log p_v,
//   d L / d x_v = ([v = z] - p_v) / T,      d H / d x_v = - p_v (log p_v + H) / T.
// In exponents to base 2, d = (x_v - m) log2(e) / T, p_v = 2^d / s and log p_v = d ln 2 - log s, so
//   w dL + u dH = 2^d (gain + slope d) + [v = z] w / T,
//   gain = -(w + u X) / (T s),      slope = -u ln 2 / (T s),      X = - ln 2 sum_v p_v d_v = H - log s:
// one walk over the row gives its sums, a second one writes the gradient.  The sums leave z out, so that 1 - p
// of a token that is nearly certain, and its log p, keep their digits: they are the others' sum; and one of
// the others' largest logits, so that they do where another token is nearly certain.  X is never
// formed as the difference: log s is about 12 in a row of 131072 that is nearly uniform, and its rounding would
// be an error that all tokens of the row share.
//
// Bound by reading and writing, and by what of the second read crosses the fabric: 8192 rows of 131072
// bfloat16 with their gradient 819 us, 5.2 TB/s of one read and one write.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "token.h"

namespace tsc {
namespace {

// Few long rows are divided among workgroups, in two launches.  The second one costs 4 us of a call, which a row
// walked by one workgroup takes at about 50000 bfloat16 tokens, and from some 500 rows on the chip is full without.
// Divided and whole, us, the gradient: 16 rows of 32000 12.5 and 11.3, of 50001 12.6 and 15.3, of 131072 13.4 and
// 28.3; 320 rows of 131072 46 and 50, 512 rows 71 and 59.
constexpr int kPartThreads = 256;
constexpr int kLongRow = 49152;    // tokens
constexpr int kFewRows = 512;
constexpr int kWantParts = 1024;   // workgroups that fill the chip (320 rows of 131072 with 512: 53 us)
constexpr int kMinPart = 4096;     // tokens of a part (no difference from 2048 to 8192)
// Vectors of a row that a thread holds in LDS between the two walks.  8192 rows of 131072 bfloat16 with
// their gradient by 512 threads, us (with sums that took 4 less): 870 without, 850 with 2, 832 with 4, 815 with 6,
// 825 with 9 (two workgroups a CU instead of three), 1026 with 10 (one); 859 by 1024 threads with 9.
constexpr int kHold = 6;

struct Row {
    float m, gain, slope;   // elsewhere
    float at_z;
};

// The row's given token, -1: none
__device__ __forceinline__ int token_of(const ScoreArgs& a, uint32_t row) {
    const int z = a.tokens[row];
    return z < a.V ? z : -1;
}

// A vector's logits for the sums: without z, which lies at z - at of it or elsewhere
template <int W>
__device__ __forceinline__ void leave_out(float (&v)[W], int at, int z) {
    if ((unsigned)(z - at) < (unsigned)W)
#pragma unroll
        for (int k = 0; k < W; ++k) v[k] = z - at == k ? -INFINITY : v[k];
}

// The row's scores, and what its gradient is made of, from the others' sums
template <class T, bool kGrad>
__device__ __forceinline__ Row finish(const ScoreArgs& a, uint32_t row, const T* x, int z, Spread others,
                                      bool write) {
    const float inv_t = a.scale.inv_t, c = a.scale.c, xz = z >= 0 ? to_f(x[z]) : -INFINITY;
    const bool top = xz >= others.m;   // the given token is the one that the sums leave out
    const float m = fmaxf(others.m, xz), d = fmaxf((xz - m) * c, kNoTerm), e = exp2_(d);
    Spread all = others;
    if (top) {
        all = spread_raise(others, m, c);
    } else {
        all.s += all.whole() ? -e : e;
        all.t += d * e;
    }
    const RowScore score(all);
    if (write) {
        if (a.logp) a.logp[row] = z >= 0 ? score.logp(xz, inv_t) : 0.f;
        if (a.entropy) a.entropy[row] = score.entropy;
    }
    Row r{};
    if constexpr (kGrad) {
        const float s = all.sum(), without = top ? all.s : others.sum();
        float w = z >= 0 ? (a.weights ? a.weights[row] : 1.f) * inv_t : 0.f;
        float u = a.entropy_weights ? a.entropy_weights[row] * inv_t : 0.f;
        if (!(s > 0.f)) w = u = 0.f;   // no finite logit
        const float f = s > 0.f ? 1.f / s : 0.f, p = e * f;
        r.m = m;
        r.gain = -(w + u * score.below) * f;
        r.slope = -u * kLn2 * f;
        r.at_z = w * (s > 0.f ? without * f : 1.f) - (p > 0.f ? u * p * ((xz - m) * inv_t + score.below) : 0.f);
    }
    return r;
}

template <bool kEntropy>
__device__ __forceinline__ float grad_of(float x, const Row& r, float c) {
    if constexpr (kEntropy) {
        const float d = fmaxf((x - r.m) * c, kNoTerm);
        return exp2_(d) * fmaf(r.slope, d, r.gain);
    } else {
        return r.gain * exp2_((x - r.m) * c);
    }
}

// The gradient of the vector at token `at`
template <class T, bool kEntropy>
__device__ __forceinline__ void store_grad(T* grad, const Raw<T>& q, const Row& r, int at, int z, float c) {
    constexpr int W = kVec<T>;
    float v[W];
    unpack<T>(q, v);
#pragma unroll
    for (int k = 0; k < W; ++k) v[k] = grad_of<kEntropy>(v[k], r, c);
    if ((unsigned)(z - at) < (unsigned)W)
#pragma unroll
        for (int k = 0; k < W; ++k) v[k] = z - at == k ? r.at_z : v[k];
    store_raw<T>(grad, pack<T>(v));
}

template <class T, int NT>
__device__ __forceinline__ void write_zeros(T* grad, int lo, int hi) {
    const int nv = (hi - lo) / kVec<T>;
    for (int i = threadIdx.x; i < nv; i += NT) store_raw<T>(grad + lo + (size_t)i * kVec<T>, Raw<T>{});
    const int e = lo + nv * kVec<T> + (int)threadIdx.x;
    if (e < hi) grad[e] = from_f<T>(0.f);
}

// A wave's sums without z: its lanes call all this together, for vectors that begin at token `at`
template <class T>
struct RowSums {
    static constexpr int W = kVec<T>;
    WaveSpread<T> sums;
    float most, c;   // the largest logit
    int z;
    __device__ __forceinline__ void init(const Scale& k, int z_) {
        sums.init(k, -INFINITY);
        most = -INFINITY, c = k.c, z = z_;
    }
    // there: otherwise the lane has no vector
    __device__ __forceinline__ void push(const Raw<T>& r, int at, bool there) {
        float v[W];
        unpack<T>(r, v);
        leave_out(v, at, z);
        const float t = there ? max_of(v) : -INFINITY;
        most = fmaxf(most, t);
        const Raw<T> q[1] = {r};
        const bool raised = sums.raise(q, t, c, (unsigned)(z - at) < (unsigned)W ? z - at : -1);
        if (there) sums.push(v, c);
        if (raised) sums.pushed(c);
    }
    // Token e alone, where it is below `end`
    __device__ __forceinline__ Raw<T> one(const T* x, int e, int end) const {
        float v[W];
#pragma unroll
        for (int k = 0; k < W; ++k) v[k] = -INFINITY;
        if (e < end) v[0] = to_f(x[e]);
        return pack<T>(v);
    }
};

// Sums of tokens [lo, hi) the slow way that any logits allow
template <class T, int NT>
__device__ Spread sums_again(const T* x, int lo, int hi, int z, float c, float4* red) {
    Spread s = spread_empty();
    walk_row<T, NT, 1>(x, lo, hi, threadIdx.x, [&](float (&v)[kVec<T>], int at, int) {
        leave_out(v, at, z);
        spread_push(s, v, c);
    });
    return block_spread<NT>(s, c, red);
}

// kGrad: the row is read again, backwards: what was read last is nearest.  kEntropy: of the gradient.
template <class T, int NT, bool kGrad, bool kEntropy>
__global__ __launch_bounds__(NT) void k_score(ScoreArgs a, int hold) {
    extern __shared__ uint4 held[];   // kGrad: a thread's first `hold` vectors
    __shared__ float4 red[NT / kWave];
    constexpr int W = kVec<T>, kU = kGrad ? 2 : 4;   // vectors asked for at once
    const int tid = threadIdx.x, V = a.V, nv = V / W;
    const float c = a.scale.c;
    const uint32_t rows = (uint32_t)(a.B * a.N), N = (uint32_t)a.N;
    for (uint32_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const uint32_t b = row / N, n = row % N;
        T* grad = (T*)a.grad + (size_t)row * V;
        if (n >= clamp_rows(a.lengths, b, N)) {
            if (tid == 0) {
                if (a.logp) a.logp[row] = 0.f;
                if (a.entropy) a.entropy[row] = 0.f;
            }
            if constexpr (kGrad) write_zeros<T, NT>(grad, 0, V);
            continue;
        }
        const T* x = row_of<T>(a.logits, b, n);
        auto from = [&](int i) { return (const T*)((const char*)x + (uint32_t)i * 16u); };
        auto to = [&](int i) { return (T*)((char*)grad + (uint32_t)i * 16u); };
        const int z = token_of(a, row);
        RowSums<T> sums;
        sums.init(a.scale, z);
        int i = tid;
        const int kept = kGrad ? min(hold * NT, nv) : 0;   // vectors that are
        if constexpr (kGrad) {
            for (; (i | (kWave - 1)) + (kU - 1) * NT < kept; i += kU * NT) {
                Raw<T> r[kU];
#pragma unroll
                for (int u = 0; u < kU; ++u) r[u] = load_raw<T, true>(from(i + u * NT));
#pragma unroll
                for (int u = 0; u < kU; ++u) {
                    held[i + u * NT] = make_uint4(r[u].w[0], r[u].w[1], r[u].w[2], r[u].w[3]);
                    sums.push(r[u], (i + u * NT) * W, true);
                }
            }
            for (; (i & ~(kWave - 1)) < kept; i += NT) {
                const Raw<T> r = load_raw<T, true>(from(min(i, kept - 1)));
                if (i < kept) held[i] = make_uint4(r.w[0], r.w[1], r.w[2], r.w[3]);
                sums.push(r, i * W, i < kept);
            }
        }
        for (; (i | (kWave - 1)) + (kU - 1) * NT < nv; i += kU * NT) {
            Raw<T> r[kU];
#pragma unroll
            for (int u = 0; u < kU; ++u) r[u] = load_raw<T, !kGrad>(from(i + u * NT));
#pragma unroll
            for (int u = 0; u < kU; ++u) sums.push(r[u], (i + u * NT) * W, true);
        }
        for (; (i & ~(kWave - 1)) < nv; i += NT) sums.push(load_raw<T, !kGrad>(from(min(i, nv - 1))), i * W, i < nv);
        const int e = nv * W + tid;   // the row's last few tokens
        if (nv * W < V) sums.push(sums.one(x, e, V), e, true);
        Spread all = join_spread<NT>(sums.sums.value(c), c, red);
        if (far(block_max<NT>(sums.most, (float*)red), a.scale)) all = sums_again<T, NT>(x, 0, V, z, c, red);
        const Row r = finish<T, kGrad>(a, row, x, z, all, tid == 0);
        if constexpr (kGrad) {
            if (e < V) grad[e] = from_f<T>(e == z ? r.at_z : grad_of<kEntropy>(to_f(x[e]), r, c));
            i = tid + (nv > tid ? (nv - 1 - tid) / NT * NT : -NT);
            for (; i - (kU - 1) * NT >= kept; i -= kU * NT) {
                Raw<T> q[kU];
#pragma unroll
                for (int u = 0; u < kU; ++u) q[u] = load_raw<T, true>(from(i - u * NT));
#pragma unroll
                for (int u = 0; u < kU; ++u)
                    store_grad<T, kEntropy>(to(i - u * NT), q[u], r, (i - u * NT) * W, z, c);
            }
            for (; i >= kept; i -= NT)
                store_grad<T, kEntropy>(to(i), load_raw<T, true>(from(i)), r, i * W, z, c);
            for (; i >= 0; i -= NT) {
                const uint4 q = held[i];
                store_grad<T, kEntropy>(to(i), {{q.x, q.y, q.z, q.w}}, r, i * W, z, c);
            }
        }
    }
}

// ---- few rows: each is divided among workgroups ----

struct ScorePlan {
    int parts;
    float4* sums;   // [rows][parts]: maximum and sum, entropy's sum, largest logit
    size_t bytes;
};
ScorePlan score_plan(int64_t rows, int64_t V, void* ws) {
    ScorePlan p;
    int64_t parts = V > kLongRow && rows < kFewRows ? (kWantParts + rows - 1) / rows : 1;
    const int64_t most = (V + kMinPart - 1) / kMinPart;
    if (parts > most) parts = most;
    if (parts > kWave) parts = kWave;
    p.parts = (int)parts;
    p.sums = (float4*)ws;
    p.bytes = parts > 1 ? ((size_t)rows * parts * sizeof(float4) + 255) / 256 * 256 : 0;
    return p;
}
// Tokens [lo, hi) of a part: a multiple of 64, so that parts of an aligned row are aligned
__device__ __forceinline__ void part_range(int V, int parts, int part, int* lo, int* hi) {
    const int per = ((V + parts - 1) / parts + 63) / 64 * 64;
    *lo = min(part * per, V);
    *hi = min(*lo + per, V);
}

template <class T>
__global__ __launch_bounds__(kPartThreads) void k_score_sums(ScoreArgs a, ScorePlan p) {
    __shared__ float4 red[kPartThreads / kWave];
    constexpr int NT = kPartThreads, W = kVec<T>;
    const uint32_t row = blockIdx.x / (uint32_t)p.parts;   // fewer than kWantParts of them
    const int part = (int)(blockIdx.x % (uint32_t)p.parts);
    const uint32_t b = row / (uint32_t)a.N, n = row % (uint32_t)a.N;
    if (n >= clamp_rows(a.lengths, b, a.N)) return;
    const T* x = row_of<T>(a.logits, b, n);
    const float c = a.scale.c;
    int lo, hi;
    part_range(a.V, p.parts, part, &lo, &hi);
    const int z = token_of(a, row);
    RowSums<T> sums;
    sums.init(a.scale, z);
    constexpr int kU = 4;
    const int nv = (hi - lo) / W;
    int i = threadIdx.x;
    for (; (i | (kWave - 1)) + (kU - 1) * NT < nv; i += kU * NT) {
        Raw<T> r[kU];
#pragma unroll
        for (int u = 0; u < kU; ++u) r[u] = load_raw<T, false>(x + lo + (size_t)(i + u * NT) * W);
#pragma unroll
        for (int u = 0; u < kU; ++u) sums.push(r[u], lo + (i + u * NT) * W, true);
    }
    for (; (i & ~(kWave - 1)) < nv; i += NT)
        sums.push(load_raw<T, false>(x + lo + (size_t)min(i, nv - 1) * W), lo + i * W, i < nv);
    const int e = lo + nv * W + (int)threadIdx.x;
    if (lo + nv * W < hi) sums.push(sums.one(x, e, hi), e, true);
    Spread s = join_spread<NT>(sums.sums.value(c), c, red);
    const float most = block_max<NT>(sums.most, (float*)red);
    if (most != -INFINITY && far(most, a.scale)) s = sums_again<T, NT>(x, lo, hi, z, c, red);
    if (threadIdx.x == 0) p.sums[blockIdx.x] = make_float4(s.m, s.s, s.t, 0.f);
}

template <class T, bool kGrad, bool kEntropy>
__global__ __launch_bounds__(kPartThreads) void k_score_parts(ScoreArgs a, ScorePlan p) {
    constexpr int NT = kPartThreads, W = kVec<T>;
    const int parts = kGrad ? p.parts : 1;
    const uint32_t row = blockIdx.x / (uint32_t)parts;
    const int part = (int)(blockIdx.x % (uint32_t)parts);
    const uint32_t b = row / (uint32_t)a.N, n = row % (uint32_t)a.N;
    T* grad = (T*)a.grad + (size_t)row * a.V;
    int lo, hi;
    part_range(a.V, p.parts, part, &lo, &hi);
    const bool first = part == 0 && threadIdx.x == 0;
    if (n >= clamp_rows(a.lengths, b, a.N)) {
        if (first) {
            if (a.logp) a.logp[row] = 0.f;
            if (a.entropy) a.entropy[row] = 0.f;
        }
        if constexpr (kGrad) write_zeros<T, NT>(grad, lo, hi);
        return;
    }
    const T* x = row_of<T>(a.logits, b, n);
    const float c = a.scale.c;
    const int lane = threadIdx.x % kWave;
    const float4 s = lane < p.parts ? p.sums[(size_t)row * p.parts + lane]
                                    : make_float4(-FLT_MAX, -0.f, 0.f, 0.f);
    const int z = token_of(a, row);
    const Row r = finish<T, kGrad>(a, row, x, z, wave_spread({s.x, s.y, s.z}, c), first);
    if constexpr (kGrad)
        walk_row<T, NT, 4, true>(x, lo, hi, threadIdx.x, [&](const float (&v)[W], int at, int num) {
            float y[W];
#pragma unroll
            for (int k = 0; k < W; ++k)
                y[k] = at + k == z ? r.at_z : grad_of<kEntropy>(v[k], r, c);
            if (num == W)
                store_raw<T>(grad + at, pack<T>(y));
            else
                grad[at] = from_f<T>(y[0]);
        });
}

template <class T>
void launch_parts(const ScoreArgs& a, const ScorePlan& p, hipStream_t s) {
    const unsigned rows = (unsigned)(a.B * a.N), grid = rows * (unsigned)p.parts;
    k_score_sums<T><<<grid, kPartThreads, 0, s>>>(a, p);
    if (!a.grad)
        k_score_parts<T, false, false><<<rows, kPartThreads, 0, s>>>(a, p);
    else if (a.entropy_weights)
        k_score_parts<T, true, true><<<grid, kPartThreads, 0, s>>>(a, p);
    else
        k_score_parts<T, true, false><<<grid, kPartThreads, 0, s>>>(a, p);
}

}  // namespace

size_t score_workspace(int64_t B, int64_t N, int64_t V) { return score_plan(B * N, V, nullptr).bytes; }

hipError_t launch_score(const ScoreArgs& a, hipStream_t s) {
    with_type(a.dtype, [&](auto t) {
        using T = decltype(t);
        const int64_t rows = a.B * a.N;
        const ScorePlan p = score_plan(rows, a.V, a.ws);
        if (p.parts > 1) return launch_parts<T>(a, p, s);
        auto go = [&](auto nt) {
            constexpr int NT = decltype(nt)::value;
            const unsigned g = row_grid(rows, NT);
            if (!a.grad) {
                k_score<T, NT, false, false><<<g, NT, 0, s>>>(a, 0);
                return;
            }
            const int64_t vectors = a.V / kVec<T>;
            const int hold = (int)std::min<int64_t>((vectors + NT - 1) / NT, kHold);
            const size_t lds = (size_t)hold * NT * sizeof(uint4);
            if (a.entropy_weights)
                k_score<T, NT, true, true><<<g, NT, lds, s>>>(a, hold);
            else
                k_score<T, NT, true, false><<<g, NT, lds, s>>>(a, hold);
        };
        // Threads of a row, by what was measured (us, bfloat16, the gradient but where scores are named).  64 and
        // 256: 16000 rows of 300 17.5 and 49, 4000 of 8192 28 and 33, 1000 of 4096 8.7 and 8.2, of 9000 17 and 13.
        // 256 and 512: few rows, 16 of 20000 10.7 and 9.3, 512 of 50001 36 and 26; many, 2900 of 8192 27 and 34, of
        // 32000 76 and 81, of 36000 95 and 87, of 131072 346 and 314; scores alone, which hold nothing of the row,
        // 129 and 137.
        const int64_t bytes = (int64_t)a.V * sizeof(T);
        if (a.V <= 1024 || (a.V <= 8192 && rows >= 2048))
            go(std::integral_constant<int, 64>{});
        else if (rows <= kFewRows ? bytes > 16384 : a.grad && bytes > 65536)
            go(std::integral_constant<int, 512>{});
        else
            go(std::integral_constant<int, 256>{});
    });
    return hipGetLastError();
}

}  // namespace tsc
