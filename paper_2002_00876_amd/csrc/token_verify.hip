// token_verify.hip -- verification of drafted tokens against the target's probabilities.
//
// Draft t is accepted while u_t q_t(z_t) < p_t(z_t); after a accepted drafts the next token is
// argmax_v r_v / e_v, r = max(p_a - q_a, 0) where draft a was refused and p_a otherwise, e_v the
// given exponentials: v's clock, of rate r_v, rings first with probability r_v / sum r.
//
// k_verify_stats sums rows in parts, one workgroup each (maximum and sum of the softmax).
// k_verify_draw runs the race over the one row of every sequence that its next token is drawn
// from, again in parts, whose winners meet in a maximum over (score, ~index) words, which no
// order of arrival changes.  Which row that is, each workgroup finds out by itself: the tests
// are a few numbers a draft.
//
// Both are bound by reading: 8 drafts of 256 sequences over 131072 bfloat16 tokens take 187 us, 1.2 GB
// at 6.4 TB/s, of which refused drafts save what follows them; of 1 sequence about 5 and 7 us, a few
// dependent loads and two atomics across the chip.
#include <hip/hip_runtime.h>

#include "token.h"

namespace tsc {
namespace {

constexpr int kStatThreads = 256;
constexpr int kDrawThreads = 512;
constexpr int kSmallThreads = 1024;
// Elements a wave, up to which one workgroup takes a sequence (us, 4 drafts: 4 sequences over 4096
// tokens 8.3 by one, over 6000 9.6 in parts; 128 sequences 8.8 and, over 5000, 15.4)
constexpr int kSmallElems = 4096;
constexpr int kMaxParts = kWave;   // parts of a row: one a lane when they are joined
constexpr int kMinPart = 2048;     // elements of a part: 8 a thread
constexpr int kMaxPart = 32768;
constexpr int kMaxGroups = 8;      // launches that the positions are divided among
constexpr int kAlive = 0x7fffffff;
// Elements of a position's rows from which the positions are divided among launches (us undivided /
// divided: 8 drafts of 128 sequences over 100003 tokens 96 / 103, of 256 over 65536 131 / 126, over
// 131072 244 / 187).
constexpr double kApartElems = 16e6;
constexpr int kStatParts = 2048, kDrawParts = 1024;   // workgroups that fill the chip

// Parts of a row: enough workgroups to fill the chip where the rows are few, and none so long that
// the chip waits for the last of them where sequences have unequal numbers of drafts (128
// sequences of up to 8 over 100003 tokens: both kernels take 83 us in whole rows, 75 in quarters)
inline int parts_of(int64_t rows, int64_t V, int64_t want) {
    int64_t p = (want + rows - 1) / rows;
    if (p < (V + kMaxPart - 1) / kMaxPart) p = (V + kMaxPart - 1) / kMaxPart;
    const int64_t most = (V + kMinPart - 1) / kMinPart;
    if (p > most) p = most;
    if (p > kMaxParts) p = kMaxParts;
    return p < 1 ? 1 : (int)p;
}
__device__ __forceinline__ void part_range(int V, int parts, int part, int* lo, int* hi) {
    // multiples of 64 elements, so that parts of an aligned row are aligned
    const int per = ((V + parts - 1) / parts + 63) / 64 * 64;
    *lo = min(part * per, V);
    *hi = min(*lo + per, V);
}

struct Plan {
    int parts, draw_parts;
    bool apart;       // the positions are divided among launches
    float2* stats;    // [B][2][G + 1][parts]: target's, draft's maximum and sum
    float* logit;     // [B][2][G + 1]: their logits of the draft
    uint64_t* best;   // [B] the race's largest word so far
    int32_t* left;    // [B] parts of the race that have not arrived
    int32_t* stop;    // [kMaxGroups][B] first draft refused before the group's, or kAlive
    size_t bytes;
};
inline Plan plan_of(int64_t B, int64_t G, int64_t V, void* ws) {
    Plan p;
    p.apart = (double)B * V >= kApartElems;
    p.parts = parts_of(p.apart ? 2 * B : B * (2 * G + 1), V, kStatParts);
    p.draw_parts = parts_of(B, V, kDrawParts);
    char* base = (char*)ws;
    size_t off = 0;
    auto take = [&](size_t bytes) {
        char* at = base + off;
        off += (bytes + 255) / 256 * 256;
        return at;
    };
    const size_t rows = (size_t)B * 2 * (G + 1);
    p.stats = (float2*)take(rows * p.parts * sizeof(float2));
    p.logit = (float*)take(rows * sizeof(float));
    p.best = (uint64_t*)take((size_t)B * sizeof(uint64_t));
    p.left = (int32_t*)take((size_t)B * sizeof(int32_t));
    p.stop = (int32_t*)take((size_t)B * kMaxGroups * sizeof(int32_t));
    p.bytes = off;
    return p;
}
__device__ __forceinline__ int64_t row_index(const VerifyArgs& a, int64_t b, int side, int64_t t) {
    return (b * 2 + side) * (a.G + 1) + t;
}

__device__ __forceinline__ float log_prob(float x, Soft s, const Scale& k) {
    return (x - s.m) * k.inv_t - logf(s.s);
}

// 2^((x - m) c - k), with the product's rounding made good: the hardware's exponential (2^-23) is
// what is left of the error, also far below the maximum.  0 from an exponent of -200 on, where the
// product may be infinite (tokens masked with the type's lowest value) and nothing can be made good.
__device__ __forceinline__ float numerator(float x, float m, float c, float k) {
    const float d = x - m, e = d * c;
    return e - k > -200.f ? exp2_(e - k) * fmaf(fmaf(d, c, -e), 0.69314718f, 1.f) : 0.f;
}

// Whether a draft of target's logit x and draft's y is accepted, and its log-probability.
// u q < p without a division: u e_q s_p < e_p s_q, the products in 64 bits.  Where both numerators
// are far below the 32-bit floats, both exponents are taken from the larger one's.  A p below the
// 64-bit floats (2^-1074) is 0, and refuses, as -inf does.
__device__ __forceinline__ bool accepts(const VerifyArgs& a, float x, float y, float u, float lse,
                                        Soft sp, Soft sq, float* logp) {
    *logp = 0.f;
    if (!(x > -INFINITY)) return false;
    *logp = log_prob(x, sp, a.scale);
    const float c = a.scale.c, cq = a.draft_scale.c, ep = (x - sp.m) * c;
    if (!(ep > -1074.f)) return false;
    if (y == -INFINITY || (a.draft_lse && lse == -INFINITY)) return true;
    const float mq = a.draft_lse ? lse / a.draft_scale.inv_t : sq.m;
    const float k = fminf(fmaxf(ep, (y - mq) * cq) + 100.f, 0.f);
    return (double)u * numerator(y, mq, cq, k) * (double)sp.s <
           (double)numerator(x, sp.m, c, k) * (a.draft_lse ? 1.0 : (double)sq.s);
}

struct Tests {
    Soft soft[2][kWave + 1];   // of the positions looked at: target, draft
    float logp[kWave];
    int stop;
};

// The first draft of [t0, t1), t1 - t0 <= 64, that is refused, or t1.  sh.soft then holds the
// rows' statistics, the target's of position t1 too, and sh.logp the drafts' log-probabilities.
template <int NT>
__device__ int test_drafts(const VerifyArgs& a, const Plan& p, int64_t b, int64_t t0, int64_t t1,
                           Tests& sh) {
    const int tid = threadIdx.x, lane = tid % kWave, m = (int)(t1 - t0);
    if (tid == 0) sh.stop = m;
    const bool sums = !a.draft_lse;
    float x = 0.f, y = 0.f, u = 0.f, l = 0.f;
    if (tid < m) {
        x = p.logit[row_index(a, b, 0, t0 + tid)];
        y = p.logit[row_index(a, b, 1, t0 + tid)];
        u = a.uniforms[b * a.G + t0 + tid];
        if (!sums) l = a.draft_lse[b * a.G + t0 + tid];
    }
    for (int r = tid / kWave; r < m + 1 + (sums ? m : 0); r += NT / kWave) {
        const int side = r > m, t = side ? r - m - 1 : r;
        const float2 q = lane < p.parts ? p.stats[row_index(a, b, side, t0 + t) * p.parts + lane]
                                        : make_float2(-FLT_MAX, 0.f);
        const Soft s = wave_soft({q.x, q.y}, side ? a.draft_scale.c : a.scale.c);
        if (lane == 0) sh.soft[side][t] = s;
    }
    __syncthreads();
    if (tid < m) {
        float lp;
        if (!accepts(a, x, y, u, l, sh.soft[0][tid], sh.soft[1][tid], &lp)) atomicMin(&sh.stop, tid);
        sh.logp[tid] = lp;
    }
    __syncthreads();
    return sh.stop;
}

// One workgroup per (sequence, position of [t0, t1) and side, part): maximum and sum of a part of
// a row.  The positions of a large call are divided among launches, of which `group` counts the
// earlier ones: the last of those began at position `before`, and sequences that have had a draft
// refused by then are done.
template <class TT, class TD>
__global__ __launch_bounds__(kStatThreads) void k_verify_stats(VerifyArgs a, Plan p, int64_t before,
                                                               int64_t t0, int64_t t1, int group) {
    __shared__ float2 red[kStatThreads / kWave];
    __shared__ Tests sh;
    const uint32_t width = 2 * (uint32_t)(t1 - t0);
    const uint64_t items = (uint64_t)p.parts * a.B * width;
    for (uint64_t i = blockIdx.x; i < items; i += gridDim.x) {
        const uint32_t row_at = item_row(i, p.parts, items);
        const uint32_t part = (uint32_t)(i - (uint64_t)row_at * p.parts);
        const int64_t b = row_at / width;
        const uint32_t r = row_at % width;
        const int64_t t = t0 + r / 2;
        const bool drafted = r & 1, first = r == 0 && part == 0;
        const int64_t n = clamp_rows(a.lengths, b, a.G);
        if (group == 0 && first && threadIdx.x == 0) {
            p.best[b] = 0;
            p.left[b] = p.draw_parts;
        }
        if (t >= n + (drafted ? 0 : 1)) continue;
        if (group > 0) {
            int stop = group > 1 ? p.stop[(group - 1) * a.B + b] : kAlive;
            if (stop == kAlive) {   // t0 <= n: all of the last launch's positions have drafts
                const int k = test_drafts<kStatThreads>(a, p, b, before, t0, sh);
                if (before + k < t0) stop = (int)(before + k);
                __syncthreads();
            }
            if (first && threadIdx.x == 0) p.stop[group * a.B + b] = stop;
            if (stop != kAlive) continue;
        }
        const TT* x = row_of<TT>(a.target, b, t);
        const TD* y = drafted ? row_of<TD>(a.draft, b, t) : nullptr;
        const int64_t row = row_index(a, b, drafted, t);
        if (part == 0 && threadIdx.x == 0 && t < n) {
            const int z = a.tokens[b * a.G + t];
            // (what is no token is refused: the target gives it nothing)
            p.logit[row] = z < 0 || z >= a.V ? -INFINITY : drafted ? to_f(y[z]) : to_f(x[z]);
        }
        if (drafted && a.draft_lse) continue;
        int lo, hi;
        part_range(a.V, p.parts, part, &lo, &hi);
        Soft s = soft_empty();
        const float c = drafted ? a.draft_scale.c : a.scale.c;
        if (drafted)
            walk_once<TD, kStatThreads, 4>(y, lo, hi, threadIdx.x,
                                          [&](const float (&v)[kVec<TD>], int, int) { soft_push(s, v, c); });
        else
            walk_once<TT, kStatThreads, 4>(x, lo, hi, threadIdx.x,
                                          [&](const float (&v)[kVec<TT>], int, int) { soft_push(s, v, c); });
        s = block_soft<kStatThreads>(s, c, red);
        if (threadIdx.x == 0) p.stats[row * p.parts + part] = make_float2(s.m, s.s);
    }
}

// Eight elements of a row
template <class T>
struct Eight {
    Raw<T> r[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T* at) {
#pragma unroll
        for (int h = 0; h < (int)sizeof(T) / 2; ++h) r[h] = load_raw<T, true>(at + h * kVec<T>);
    }
    __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
        for (int h = 0; h < (int)sizeof(T) / 2; ++h) {
            float u[kVec<T>];
            unpack<T>(r[h], u);
#pragma unroll
            for (int k = 0; k < kVec<T>; ++k) v[h * kVec<T> + k] = u[k];
        }
    }
};

// Rates of the race: p or max(p - q, 0) of a token from its logits
struct Race {
    float mp, ip, cp;   // target: p = 2^((x - mp) cp) ip
    float mq, iq, cq;   // draft
    bool refused;
};
__device__ __forceinline__ Race race_of(const VerifyArgs& a, int64_t b, int64_t at, bool refused,
                                        Soft sp, Soft sq) {
    Race r{sp.m, sp.s > 0.f ? 1.f / sp.s : 0.f, a.scale.c, 0.f, 0.f, a.draft_scale.c, refused};
    if (refused && a.draft_lse) {
        // (a log-sum-exp of -inf says q = 0: no difference of infinities, no power above the floats)
        const float lse = a.draft_lse[b * a.G + at];
        r.mq = lse > -INFINITY ? lse / a.draft_scale.inv_t : FLT_MAX;
        r.iq = lse > -INFINITY ? 1.f : 0.f;
    } else if (refused) {
        r.mq = sq.m;
        r.iq = sq.s > 0.f ? 1.f / sq.s : 0.f;
    }
    return r;
}
__device__ __forceinline__ uint64_t race_word(const Race& r, float x, float y, float e, int v) {
#pragma clang fp contract(off)   // where p and q are the same number their difference is 0
    const float p = exp2_((x - r.mp) * r.cp) * r.ip;
    const float d = r.refused ? p - exp2_((y - r.mq) * r.cq) * r.iq : p;
    // a token of positive d stands above all others, which run by their p
    const float score = (d > 0.f ? d : p) / fmaxf(e, FLT_MIN);
    const uint32_t key = (__float_as_uint(score) & 0x7fffffffu) | (d > 0.f ? 0x80000000u : 0u);
    return (uint64_t)key << 32 | (uint32_t)~v;
}

__device__ __forceinline__ uint64_t wave_max64(uint64_t x) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const uint64_t y = __shfl_xor((unsigned long long)x, o, kWave);
        x = x > y ? x : y;
    }
    return x;
}

// One workgroup per (sequence, part of the race).  Eight waves a SIMD are asked for: of the 80 VGPRs
// that it would take (5 to 6 waves) 64 are left and 3 or 4 go to scratch, outside the race's loop.
// What it gains where rows are many it loses in part where they are few (us for both kernels, without /
// with: 128 sequences of 8 drafts over 100003 bfloat16 77 / 75, over 100096 76.6 / 74.2, over 50000
// float32 69.3 / 68.7; 1 of 5 over 131072 bfloat16 11.7 / 12.2, float32 12.7 / 13.3; 8 of 5 23.4 / 24.3).
template <class TT, class TD>
__global__ __launch_bounds__(kDrawThreads, 8) void k_verify_draw(VerifyArgs a, Plan p) {
    __shared__ Tests sh;
    __shared__ uint64_t words[kDrawThreads / kWave];
    const int tid = threadIdx.x;
    const uint64_t items = (uint64_t)p.draw_parts * a.B;
    for (uint64_t i = blockIdx.x; i < items; i += gridDim.x) {
        const int64_t b = item_row(i, p.draw_parts, items);
        const int part = (int)(i - (uint64_t)b * p.draw_parts);
        const int64_t n = clamp_rows(a.lengths, b, a.G);
        int32_t* out = a.out + b * (a.G + 1);
        float* logp = a.logp ? a.logp + b * (a.G + 1) : nullptr;
        // the first draft that is refused; the sequence's first workgroup writes what is accepted
        int64_t t0 = 0, at;
        for (;; t0 += kWave) {
            const int64_t t1 = min(t0 + kWave, n);
            const int stop = test_drafts<kDrawThreads>(a, p, b, t0, t1, sh);
            at = t0 + stop;
            if (part == 0 && tid < stop) {
                out[t0 + tid] = a.tokens[b * a.G + t0 + tid];
                if (logp) logp[t0 + tid] = sh.logp[tid];
            }
            if (at < t1 || t1 == n) break;
            __syncthreads();
        }
        const bool refused = at < n;
        if (part == 0) {
            for (int64_t t = at + 1 + tid; t <= a.G; t += kDrawThreads) {
                out[t] = -1;
                if (logp) logp[t] = 0.f;
            }
            if (tid == 0) a.accepted[b] = (int32_t)at;
        }
        // the race over the row that the next token is drawn from
        const TT* x = row_of<TT>(a.target, b, at);
        const TD* y = refused ? row_of<TD>(a.draft, b, at) : nullptr;
        const float* e = a.noise + b * a.V;
        const Soft sp = sh.soft[0][at - t0];
        const Race race = race_of(a, b, at, refused, sp, sh.soft[1][refused ? at - t0 : 0]);
        int lo, hi;
        part_range(a.V, p.draw_parts, part, &lo, &hi);
        uint64_t best = 0;
        int v = lo + tid * 8;
        for (; v + 8 <= hi; v += kDrawThreads * 8) {
            Eight<TT> rx;
            Eight<TD> ry{};
            Eight<float> re;
            rx.load(x + v);
            if (refused) ry.load(y + v);
            re.load(e + v);
            float xv[8], yv[8], ev[8];
            rx.get(xv);
            ry.get(yv);
            re.get(ev);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const uint64_t word = race_word(race, xv[k], yv[k], ev[k], v + k);
                best = best > word ? best : word;
            }
        }
        for (; v < hi; ++v) {   // the thread that holds the part's last few
            const uint64_t word =
                race_word(race, to_f(x[v]), refused ? to_f(y[v]) : 0.f, e[v], v);
            best = best > word ? best : word;
        }
        best = wave_max64(best);
        if (tid % kWave == 0) words[tid / kWave] = best;
        __syncthreads();
        if (tid == 0) {
            for (int w = 1; w < kDrawThreads / kWave; ++w) best = best > words[w] ? best : words[w];
            bool mine = true;
            if (p.draw_parts > 1) {
                // The last part to arrive writes the winner.  All that the parts share are these
                // two words, both touched by atomics alone, so no fence (which would write back
                // and drop a whole L2) is needed: the count goes down once the maximum's old
                // value is here, that is, once the maximum is done.
                const unsigned long long old =
                    atomicMax((unsigned long long*)&p.best[b], (unsigned long long)best);
                asm volatile("" ::"v"(old) : "memory");
                mine = atomicSub(&p.left[b], 1) == 1;
                if (mine) best = atomicMax((unsigned long long*)&p.best[b], 0ull);
            }
            if (mine) {
                const int token = (int)~(uint32_t)best;
                out[at] = token;
                if (logp)
                    logp[at] = sp.s > 0.f ? log_prob(to_f(x[token]), sp, a.scale) : -INFINITY;
            }
        }
        __syncthreads();   // sh and words are free for the next part
    }
}

// A whole sequence by one workgroup, its rows by a wave each: vocabularies so small that a
// second launch and the joining of parts would take longer than the rows do
template <class TT, class TD>
__global__ __launch_bounds__(kSmallThreads) void k_verify_small(VerifyArgs a) {
    constexpr int kWaves = kSmallThreads / kWave;
    __shared__ Tests sh;
    __shared__ float logit[2][kWave];
    __shared__ uint64_t words[kWaves];
    const int tid = threadIdx.x, lane = tid % kWave;
    for (int64_t b = blockIdx.x; b < a.B; b += gridDim.x) {
        const int64_t n = clamp_rows(a.lengths, b, a.G);
        int32_t* out = a.out + b * (a.G + 1);
        float* logp = a.logp ? a.logp + b * (a.G + 1) : nullptr;
        int64_t t0 = 0, at;
        for (;; t0 += kWave) {
            const int64_t t1 = min(t0 + kWave, n);
            const int m = (int)(t1 - t0);
            if (tid == 0) sh.stop = m;
            for (int r = tid / kWave; r < 2 * m + 1; r += kWaves) {
                const int side = r & 1, k = r / 2;
                const int64_t t = t0 + k;
                const TT* x = row_of<TT>(a.target, b, t);
                const TD* y = side ? row_of<TD>(a.draft, b, t) : nullptr;
                if (lane == 0 && k < m) {
                    const int z = a.tokens[b * a.G + t];
                    logit[side][k] = z < 0 || z >= a.V ? -INFINITY : side ? to_f(y[z]) : to_f(x[z]);
                }
                if (side && a.draft_lse) continue;
                const float c = side ? a.draft_scale.c : a.scale.c;
                Soft s = soft_empty();
                if (side)
                    walk_row<TD, kWave, 4>(y, 0, a.V, lane,
                                           [&](const float (&v)[kVec<TD>], int, int) { soft_push(s, v, c); });
                else
                    walk_row<TT, kWave, 4>(x, 0, a.V, lane,
                                           [&](const float (&v)[kVec<TT>], int, int) { soft_push(s, v, c); });
                s = wave_soft(s, c);
                if (lane == 0) sh.soft[side][k] = s;
            }
            __syncthreads();
            if (tid < m) {
                float lp;
                const int64_t t = b * a.G + t0 + tid;
                if (!accepts(a, logit[0][tid], logit[1][tid], a.uniforms[t],
                             a.draft_lse ? a.draft_lse[t] : 0.f, sh.soft[0][tid], sh.soft[1][tid], &lp))
                    atomicMin(&sh.stop, tid);
                sh.logp[tid] = lp;
            }
            __syncthreads();
            const int stop = sh.stop;
            at = t0 + stop;
            if (tid < stop) {
                out[t0 + tid] = a.tokens[b * a.G + t0 + tid];
                if (logp) logp[t0 + tid] = sh.logp[tid];
            }
            if (at < t1 || t1 == n) break;
            __syncthreads();
        }
        for (int64_t t = at + 1 + tid; t <= a.G; t += kSmallThreads) {
            out[t] = -1;
            if (logp) logp[t] = 0.f;
        }
        const bool refused = at < n;
        const TT* x = row_of<TT>(a.target, b, at);
        const TD* y = refused ? row_of<TD>(a.draft, b, at) : nullptr;
        const float* e = a.noise + b * a.V;
        const Soft sp = sh.soft[0][at - t0];
        const Race race = race_of(a, b, at, refused, sp, sh.soft[1][refused ? at - t0 : 0]);
        uint64_t best = 0;
        for (int v = tid; v < a.V; v += kSmallThreads) {
            const uint64_t word = race_word(race, to_f(x[v]), refused ? to_f(y[v]) : 0.f, e[v], v);
            best = best > word ? best : word;
        }
        best = wave_max64(best);
        if (lane == 0) words[tid / kWave] = best;
        __syncthreads();
        if (tid == 0) {
#pragma unroll
            for (int w = 1; w < kWaves; ++w) best = best > words[w] ? best : words[w];
            const int token = (int)~(uint32_t)best;
            out[at] = token;
            a.accepted[b] = (int32_t)at;
            if (logp)
                logp[at] = sp.s > 0.f ? log_prob(to_f(x[token]), sp, a.scale) : -INFINITY;
        }
        __syncthreads();   // sh and words are free for the next sequence
    }
}

bool small(int64_t G, int64_t V) {
    constexpr int kWaves = kSmallThreads / kWave;
    return (2 * G + kWaves) / kWaves * V <= kSmallElems;
}

}  // namespace

size_t verify_workspace(int64_t B, int64_t G, int64_t V) {
    return small(G, V) ? 0 : plan_of(B, G, V, nullptr).bytes;
}

hipError_t launch_verify(const VerifyArgs& a, hipStream_t s) {
    hipError_t e = hipSuccess;
    with_type(a.target_dtype, [&](auto t) {
        with_type(a.draft_dtype, [&](auto d) {
            using TT = decltype(t);
            using TD = decltype(d);
            if (small(a.G, a.V)) {
                k_verify_small<TT, TD><<<row_grid(a.B, kSmallThreads), kSmallThreads, 0, s>>>(a);
                e = hipGetLastError();
                return;
            }
            const Plan p = plan_of(a.B, a.G, a.V, a.ws);
            // positions [0, 2), [2, 5), [5, 11) ... where they are worth a launch, 64 at most for
            // the tests of the next
            int64_t before = 0, t0 = 0;
            for (int group = 0; t0 <= a.G; ++group) {
                int64_t t1 = a.G + 1;
                if (p.apart && group < kMaxGroups - 1) t1 = min(t1, t0 + (t0 < 1 ? 2 : t0 < 63 ? t0 + 1 : 64));
                k_verify_stats<TT, TD>
                    <<<row_grid(a.B * 2 * (t1 - t0) * p.parts, kStatThreads), kStatThreads, 0, s>>>(
                        a, p, before, t0, t1, group);
                if ((e = hipGetLastError()) != hipSuccess) return;
                before = t0;
                t0 = t1;
            }
            k_verify_draw<TT, TD>
                <<<row_grid(a.B * p.draw_parts, kDrawThreads), kDrawThreads, 0, s>>>(a, p);
            e = hipGetLastError();
        });
    });
    return e;
}

}  // namespace tsc
