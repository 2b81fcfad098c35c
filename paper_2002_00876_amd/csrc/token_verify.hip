// token_verify.hip -- verification of drafted tokens against the target's probabilities.
//
// Draft t is accepted while u_t q_t(z_t) < p_t(z_t); after a accepted drafts the next token is
// argmax_v r_v / e_v, r = max(p_a - q_a, 0) where draft a was refused and p_a otherwise, e_v the
// given exponentials: v's clock, of rate r_v, rings first with probability r_v / sum r.
//
// Two launches: the softmax statistics of every row in parts, one workgroup each; then, for
// every sequence, the tests (a few numbers, which each of its workgroups does by itself) and
// the race over the one row that the next token is drawn from, in parts whose winners meet in
// a maximum over (score, ~index) words, which no order of arrival changes.
#include <hip/hip_runtime.h>

#include "token.h"

namespace tsc {
namespace {

constexpr int kThreads = 256;
constexpr int kPartElems = 16384;   // elements of a row that one workgroup sums

__host__ __device__ inline int parts_of(int64_t V) {
    return (int)((V + kPartElems - 1) / kPartElems);
}
__device__ __forceinline__ void part_range(int V, int parts, int part, int* lo, int* hi) {
    // multiples of 64 elements, so that parts of an aligned row are aligned
    const int per = ((V + parts - 1) / parts + 63) / 64 * 64;
    *lo = min(part * per, V);
    *hi = min(*lo + per, V);
}

struct Plan {
    int parts;
    float2* stats;    // [B][2][G + 1][parts]: target's, draft's maximum and sum
    uint64_t* best;   // [B] the race's largest word so far
    int32_t* left;    // [B] parts of the race that have not arrived
    size_t bytes;
};
inline Plan plan_of(int64_t B, int64_t G, int64_t V, void* ws) {
    Plan p;
    p.parts = parts_of(V);
    char* base = (char*)ws;
    const size_t n = (size_t)B * 2 * (G + 1) * p.parts;
    p.stats = (float2*)base;
    size_t off = (n * sizeof(float2) + 255) / 256 * 256;
    p.best = (uint64_t*)(base + off);
    off += ((size_t)B * sizeof(uint64_t) + 255) / 256 * 256;
    p.left = (int32_t*)(base + off);
    off += ((size_t)B * sizeof(int32_t) + 255) / 256 * 256;
    p.bytes = off;
    return p;
}

// One workgroup per (side, position, part, sequence): maximum and sum of a part of a row
template <class TT, class TD>
__global__ __launch_bounds__(kThreads) void k_verify_stats(VerifyArgs a, Plan p) {
    __shared__ float2 red[kThreads / kWave];
    const int64_t per = (int64_t)p.parts * (2 * a.G + 1);
    for (int64_t i = blockIdx.x; i < per * a.B; i += gridDim.x) {
        const int64_t b = i / per;
        const int part = (int)(i % p.parts);
        const int64_t r = i % per / p.parts;
        const bool drafted = r > a.G;
        const int64_t t = drafted ? r - a.G - 1 : r;
        if (r == 0 && part == 0 && threadIdx.x == 0) {
            p.best[b] = 0;
            p.left[b] = p.parts;
        }
        if (t >= clamp_rows(a.lengths, b, a.G) + (drafted ? 0 : 1) || (drafted && a.draft_lse))
            continue;
        int lo, hi;
        part_range(a.V, p.parts, part, &lo, &hi);
        Soft s = soft_empty();
        const float c = drafted ? a.draft_scale.c : a.scale.c;
        if (drafted)
            walk_row<TD, kThreads, 4>(row_of<TD>(a.draft, b, t), lo, hi, threadIdx.x,
                                      [&](const float (&v)[kVec<TD>], int, int) { soft_push(s, v, c); });
        else
            walk_row<TT, kThreads, 4>(row_of<TT>(a.target, b, t), lo, hi, threadIdx.x,
                                      [&](const float (&v)[kVec<TT>], int, int) { soft_push(s, v, c); });
        s = block_soft<kThreads>(s, c, red);
        if (threadIdx.x == 0)
            p.stats[((b * 2 + drafted) * (a.G + 1) + t) * p.parts + part] = make_float2(s.m, s.s);
    }
}

__device__ __forceinline__ Soft row_stats(const Plan& p, int64_t b, int side, int64_t G, int64_t t,
                                          float c) {
    Soft s = soft_empty();
    const float2* q = p.stats + ((b * 2 + side) * (G + 1) + t) * p.parts;
    for (int k = 0; k < p.parts; ++k) s = soft_merge(s, {q[k].x, q[k].y}, c);
    return s;
}

// log-probability of a logit, in 64 bits: what is decided by it are whole tokens
__device__ __forceinline__ double log_prob(float x, Soft s, const Scale& k) {
    return ((double)x - (double)s.m) * (double)k.inv_t - log((double)s.s);
}

template <class TT, class TD>
__global__ __launch_bounds__(kThreads) void k_verify_draw(VerifyArgs a, Plan p) {
    __shared__ int stop;
    __shared__ uint64_t words[kThreads / kWave];
    const int tid = threadIdx.x;
    for (int64_t i = blockIdx.x; i < a.B * p.parts; i += gridDim.x) {
        const int64_t b = i / p.parts;
        const int part = (int)(i % p.parts);
        const int64_t n = clamp_rows(a.lengths, b, a.G);
        // the first draft that is refused
        if (tid == 0) stop = (int)n;
        __syncthreads();
        for (int64_t t = tid; t < n; t += kThreads) {
            const int z = a.tokens[b * a.G + t];
            bool ok = false;
            if (z >= 0 && z < a.V) {
                const Soft s = row_stats(p, b, 0, a.G, t, a.scale.c);
                const float x = to_f(row_of<TT>(a.target, b, t)[z]);
                const float y = to_f(row_of<TD>(a.draft, b, t)[z]);
                double lq;
                if (a.draft_lse)
                    lq = (double)y * (double)a.draft_scale.inv_t - (double)a.draft_lse[b * a.G + t];
                else
                    lq = log_prob(y, row_stats(p, b, 1, a.G, t, a.draft_scale.c), a.draft_scale);
                if (x > -INFINITY) {
                    const double lp = log_prob(x, s, a.scale);
                    ok = y == -INFINITY || (double)a.uniforms[b * a.G + t] * exp(lq) < exp(lp);
                }
            }
            if (!ok) atomicMin(&stop, (int)t);
        }
        __syncthreads();
        const int64_t at = stop;
        const bool refused = at < n;
        // the race over the row that the next token is drawn from
        const TT* x = row_of<TT>(a.target, b, at);
        const TD* y = refused ? row_of<TD>(a.draft, b, at) : nullptr;
        const float* e = a.noise + b * a.V;
        const Soft sp = row_stats(p, b, 0, a.G, at, a.scale.c);
        const float ip = sp.s > 0.f ? 1.f / sp.s : 0.f, cp = a.scale.c, cq = a.draft_scale.c;
        float mq = 0.f, iq = 0.f;
        if (refused) {
            if (a.draft_lse) {
                mq = a.draft_lse[b * a.G + at] / a.draft_scale.inv_t;
                iq = 1.f;
            } else {
                const Soft sq = row_stats(p, b, 1, a.G, at, cq);
                mq = sq.m;
                iq = sq.s > 0.f ? 1.f / sq.s : 0.f;
            }
        }
        int lo, hi;
        part_range(a.V, p.parts, part, &lo, &hi);
        uint64_t best = 0;
        for (int v = lo + tid; v < hi; v += kThreads) {
#pragma clang fp contract(off)   // where p and q are the same number their difference is 0
            const float pv = exp2_((to_f(x[v]) - sp.m) * cp) * ip;
            const float r = refused ? pv - exp2_((to_f(y[v]) - mq) * cq) * iq : pv;
            // a token of positive r stands above all others, which run by their p
            const float rate = r > 0.f ? r : pv;
            const float score = rate > 0.f ? rate / e[v] : 0.f;
            const uint32_t key = (__float_as_uint(score) & 0x7fffffffu) | (r > 0.f ? 0x80000000u : 0u);
            const uint64_t word = (uint64_t)key << 32 | (uint32_t)~v;
            best = best > word ? best : word;
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            const uint64_t other = __shfl_xor((unsigned long long)best, o, kWave);
            best = best > other ? best : other;
        }
        if (tid % kWave == 0) words[tid / kWave] = best;
        __syncthreads();
        if (tid == 0) {
            for (int w = 1; w < kThreads / kWave; ++w) best = best > words[w] ? best : words[w];
            atomicMax((unsigned long long*)&p.best[b], (unsigned long long)best);
            __threadfence();
            stop = atomicSub(&p.left[b], 1) == 1 ? 1 : 0;
        }
        __syncthreads();
        if (stop) {   // the last part to arrive writes what is emitted
            __threadfence();
            const uint64_t w =
                __hip_atomic_load(&p.best[b], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            const int token = (int)~(uint32_t)w;
            for (int64_t t = tid; t <= a.G; t += kThreads) {
                const int z = t < at ? a.tokens[b * a.G + t] : t == at ? token : -1;
                a.out[b * (a.G + 1) + t] = z;
                if (!a.logp) continue;
                float lp = 0.f;
                if (t <= at) {
                    const Soft s = row_stats(p, b, 0, a.G, t, a.scale.c);
                    lp = s.s > 0.f
                             ? (float)log_prob(to_f(row_of<TT>(a.target, b, t)[z]), s, a.scale)
                             : -INFINITY;
                }
                a.logp[b * (a.G + 1) + t] = lp;
            }
            if (tid == 0) a.accepted[b] = (int32_t)at;
        }
        __syncthreads();
    }
}

}  // namespace

size_t verify_workspace(int64_t B, int64_t G, int64_t V) { return plan_of(B, G, V, nullptr).bytes; }

hipError_t launch_verify(const VerifyArgs& a, hipStream_t s) {
    const Plan p = plan_of(a.B, a.G, a.V, a.ws);
    with_type(a.target_dtype, [&](auto t) {
        with_type(a.draft_dtype, [&](auto d) {
            using TT = decltype(t);
            using TD = decltype(d);
            k_verify_stats<TT, TD>
                <<<row_grid(a.B * (2 * a.G + 1) * p.parts, kThreads), kThreads, 0, s>>>(a, p);
            k_verify_draw<TT, TD><<<row_grid(a.B * p.parts, kThreads), kThreads, 0, s>>>(a, p);
        });
    });
    return hipGetLastError();
}

}  // namespace tsc
