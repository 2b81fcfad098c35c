// token_distill.hip -- the divergence of a student's rows from a teacher's top logits, and its
// gradient.
//
// With q = softmax(s / T) and the teacher's p_k at the tokens i_k,
//   loss = sum_k p_k (log p_k - log q[i_k]),      d loss / d s_v = (q_v sum p - p_v) / T,
// and where the teacher's rest p_r = 1 - sum p is a class of its own, q_r = sum of q outside the
// slots,
//   loss += p_r (log p_r - log q_r),              d loss / d s_v = (q_v - p_v) / T at the slots,
//                                                 d loss / d s_v = q_v (1 - p_r / q_r) / T
// elsewhere.  q_r is summed by itself (a bit for every token of the vocabulary marks the slots):
// 1 - sum of the slots' q would lose it where the student puts nearly all on the slots.  Both
// gradients are  scale * exp(s_v / T - low)  outside the slots, low the log-sum-exp of what was
// walked over, so one walk over the row gives its sums and a second one writes the gradient,
// after which the K slots' values are written over it.
//
// The loss is bound by its read (3072 rows of 32000 float32 58 to 62 us, 6.4 to 6.8 TB/s), the
// gradient by what crosses the fabric: two reads and a write (8192 rows of 131072 bfloat16 900 us,
// 7.1 TB/s).
//
// One workgroup takes a row (k_distill).  For the gradient it reads it again backwards: what was
// read last is still in the L2, the rest in the memory-side cache.  Where the rows are few each is
// divided among workgroups, with a launch for the sums (k_distill_sums) and one for what follows.
#include <hip/hip_runtime.h>

#include "token.h"

namespace tsc {
namespace {

// What the slots leave, 1 - sum p with p_k = exp(t_k / T - lse), is known to about 2^-23 (|lse| + 8):
// t_k / T and lse are each rounded by 2^-24 of themselves and t_k / T = lse + log p_k, of which the p
// take |lse| + log K on the average; the 8 stands for that, exp and the sum.  Less than twice this is
// no rest: where the student gives nothing outside the slots, its loss would be infinite.
constexpr float kMinRest = 2.38418579e-7f;   // 2^-22
__device__ __forceinline__ float min_rest(float lse) { return kMinRest * (8.f + fabsf(lse)); }
constexpr int kPartThreads = 256;
constexpr int kWantParts = 1024;   // workgroups that fill the chip
constexpr int kMinPart = 4096;     // tokens of a part
constexpr int kMaxPart = 262144;   // whose marks take half of a workgroup's 64 KiB of LDS

// Slots of a row: a thread has kMaxTop / NT of them, or the first kMaxTop threads one each
struct Slot {
    int at;    // token, -1: empty
    float t;   // teacher's logit, -inf: empty
};

__device__ __forceinline__ float top_value(const void* p, int dtype, int64_t i) {
    return dtype == TS_FLOAT32    ? ((const float*)p)[i]
           : dtype == TS_BFLOAT16 ? to_f(((const Bf16*)p)[i])
                                  : to_f(((const F16*)p)[i]);
}

// What a row's loss and gradient are made of, the same in every thread
struct Row {
    float loss;
    float low, gain;   // outside the slots: gain * 2^((s_v - low) c)
    float high, part;  // at slot k: w * (2^((s_k - high) c) * part - p_k)
    float w;
};

template <int NT>
constexpr int kSlots = kMaxTop > NT ? kMaxTop / NT : 1;

template <class T, int NT>
struct Slots {
    Slot slot[kSlots<NT>];
    float xs[kSlots<NT>], p[kSlots<NT>];

    __device__ __forceinline__ void load(const DistillArgs& a, uint32_t row, const T* x, float tl) {
#pragma unroll
        for (int q = 0; q < kSlots<NT>; ++q) {
            const int k = q * NT + (int)threadIdx.x;
            slot[q] = {-1, -INFINITY};
            xs[q] = -INFINITY;
            // a teacher's row without a finite logit says nothing: its slots are empty
            if (k < a.K && tl != -INFINITY) {
                const int64_t i = (int64_t)row * a.K + k;
                const int at = a.top_indices[i];
                if (at >= 0 && at < (int)a.V) {
                    slot[q] = {at, top_value(a.top_values, a.top_dtype, i)};
                    xs[q] = to_f(x[at]);
                }
            }
        }
    }
    // Marks the slots of tokens [lo, hi) in bits; every thread calls it, and may read them after
    __device__ __forceinline__ void mark(uint32_t* bits, int lo, int hi) {
        for (int w = threadIdx.x; w < (hi - lo + 31) / 32; w += NT) bits[w] = 0;
        __syncthreads();
#pragma unroll
        for (int q = 0; q < kSlots<NT>; ++q) {
            const int at = slot[q].at - lo;
            if (at >= 0 && at < hi - lo) atomicOr(&bits[at >> 5], 1u << (at & 31));
        }
        __syncthreads();
    }
    // soft: of the tokens walked over (all, or with a rest those outside the slots)
    template <bool kRest>
    __device__ Row finish(const DistillArgs& a, uint32_t row, Soft soft, float tl, float2* red) {
#pragma clang fp contract(off)   // the loss is the same with the gradient and without, to the bit
        const float c = a.scale.c, inv_t = a.scale.inv_t;
        float* redf = (float*)red;
        Soft all = soft;
        if constexpr (kRest) {
            Soft own = soft_empty();
#pragma unroll
            for (int q = 0; q < kSlots<NT>; ++q) own.m = fmaxf(own.m, xs[q]);
#pragma unroll
            for (int q = 0; q < kSlots<NT>; ++q) own.s += exp2_((xs[q] - own.m) * c);
            all = soft_merge(soft, block_soft<NT>(own, c, red), c);
        }
        float norm = 1.f;
        if (kRest) {
#pragma unroll
            for (int q = 0; q < kSlots<NT>; ++q)
                p[q] = slot[q].at >= 0 ? exp_(slot[q].t * inv_t - tl) : 0.f;
        } else {
            float tm = -FLT_MAX, s = 0.f;
#pragma unroll
            for (int q = 0; q < kSlots<NT>; ++q) tm = fmaxf(tm, slot[q].t);
            tm = block_max<NT>(tm, redf);
#pragma unroll
            for (int q = 0; q < kSlots<NT>; ++q) s += p[q] = exp2_((slot[q].t - tm) * c);
            s = block_sum<NT>(s, redf);
            norm = s > 0.f ? 1.f / s : 0.f;
        }
        float mass = 0.f, kl = 0.f;
        const float ls = all.s > 0.f ? logf(all.s) : 0.f;
#pragma unroll
        for (int q = 0; q < kSlots<NT>; ++q) {
            p[q] *= norm;
            if (p[q] > 0.f) {
                mass += p[q];
                kl += p[q] * (logf(p[q]) - ((xs[q] - all.m) * inv_t - ls));
            }
        }
        mass = block_sum<NT>(mass, redf);
        kl = block_sum<NT>(kl, redf);
        float keep = mass > 0.f ? 1.f : 0.f;
        if constexpr (kRest) {
            float rest = 1.f - mass;
            if (!(rest > min_rest(tl))) rest = 0.f;
            if (a.K == (int)a.V) {   // (and where no token is outside the slots)
                float filled = 0.f;
#pragma unroll
                for (int q = 0; q < kSlots<NT>; ++q) filled += slot[q].at >= 0 ? 1.f : 0.f;
                if (block_sum<NT>(filled, redf) == (float)a.K) rest = 0.f;
            }
            const float low =
                soft.s > 0.f ? (soft.m - all.m) * inv_t + logf(soft.s) - ls : -INFINITY;
            if (rest > 0.f) kl += rest * (logf(rest) - low);
            keep = exp_(low) - rest;
            if (tl == -INFINITY) kl = keep = 0.f;   // no teacher, whatever the student's row
        }
        Row r;
        r.loss = kl;
        r.w = all.s > 0.f ? (a.weights ? a.weights[row] : 1.f) * inv_t : 0.f;
        r.low = soft.m;
        r.gain = soft.s > 0.f ? r.w * keep / soft.s : 0.f;
        r.high = all.m;
        r.part = all.s > 0.f && (kRest || keep > 0.f) ? 1.f / all.s : 0.f;
        return r;
    }
    // The gradient at the slots of tokens [lo, hi); the walk's values there are written before
    __device__ __forceinline__ void write(const Row& r, float c, T* grad, int lo, int hi) {
        __syncthreads();
#pragma unroll
        for (int q = 0; q < kSlots<NT>; ++q)
            if (slot[q].at >= lo && slot[q].at < hi)
                grad[slot[q].at] = from_f<T>(r.w * (exp2_((xs[q] - r.high) * c) * r.part - p[q]));
    }
};

// A vector's logits, -inf at the slots
template <class T, bool kRest>
__device__ __forceinline__ void unslotted(const Raw<T>& r, const uint32_t* bits, int at,
                                          float (&v)[kVec<T>]) {
    unpack<T>(r, v);
    if constexpr (kRest) {
        const uint32_t m = bits[at >> 5] >> (at & 31) & ((1u << kVec<T>) - 1);
        if (m)
#pragma unroll
            for (int k = 0; k < kVec<T>; ++k) v[k] = m >> k & 1 ? -INFINITY : v[k];
    }
}

template <class T>
__device__ __forceinline__ void store_grad(T* grad, const Raw<T>& r, const Row& row, float c) {
    float v[kVec<T>];
    unpack<T>(r, v);
#pragma unroll
    for (int k = 0; k < kVec<T>; ++k) v[k] = row.gain * exp2_((v[k] - row.low) * c);
    store_raw<T>(grad, pack<T>(v));
}

template <class T, int NT>
__device__ __forceinline__ void write_zeros(T* grad, int lo, int hi) {
    const int nv = (hi - lo) / kVec<T>;
    for (int i = threadIdx.x; i < nv; i += NT) store_raw<T>(grad + lo + (size_t)i * kVec<T>, Raw<T>{});
    const int e = lo + nv * kVec<T> + (int)threadIdx.x;
    if (e < hi) grad[e] = from_f<T>(0.f);
}

// Maximum and sum of tokens [lo, hi) outside the slots, the slow way that any logits allow
template <class T, int NT, bool kRest>
__device__ Soft sums_again(const T* x, const uint32_t* bits, int lo, int hi, float c, float2* red) {
    constexpr int W = kVec<T>;
    Soft s = soft_empty();
    walk_row<T, NT, 1>(x, lo, hi, threadIdx.x, [&](float (&v)[W], int at, int) {
        if constexpr (kRest) {
#pragma unroll
            for (int k = 0; k < W; ++k) {
                const int e = min(at + k, hi - 1) - lo;
                v[k] = bits[e >> 5] >> (e & 31) & 1 ? -INFINITY : v[k];
            }
        }
        soft_push(s, v, c);
    });
    return block_soft<NT>(s, c, red);
}

template <class T, int NT, bool kRest, bool kGrad>
__global__ __launch_bounds__(NT) void k_distill(DistillArgs a) {
    extern __shared__ uint32_t bits[];   // kRest: a bit for every token
    __shared__ float2 red[8];
    constexpr int W = kVec<T>, kU = kGrad ? 2 : 4;   // vectors asked for at once
    const int tid = threadIdx.x, V = (int)a.V, nv = V / W;
    const float c = a.scale.c;
    const uint32_t rows = (uint32_t)(a.B * a.N), N = (uint32_t)a.N;
    for (uint32_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const uint32_t b = row / N, n = row % N;
        T* grad = (T*)a.grad + (size_t)row * V;
        if (n >= clamp_rows(a.lengths, b, N)) {
            if (a.loss && tid == 0) a.loss[row] = 0.f;
            if constexpr (kGrad) write_zeros<T, NT>(grad, 0, V);
            continue;
        }
        const T* x = row_of<T>(a.logits, b, n);
        // (a vector's place as a 32-bit offset from the row's: one register and not two)
        auto from = [&](int i) { return (const T*)((const char*)x + (uint32_t)i * 16u); };
        auto to = [&](int i) { return (T*)((char*)grad + (uint32_t)i * 16u); };
        const float tl = kRest ? a.top_lse[row] : 0.f;
        Slots<T, NT> slots;
        slots.load(a, row, x, tl);
        if constexpr (kRest) slots.mark(bits, 0, V);
        ChunkSoft soft;
        soft.init(a.scale);
        float most = -INFINITY;
        auto push = [&](const Raw<T>& r, int i) {
            float v[W];
            unslotted<T, kRest>(r, bits, i * W, v);
            const float t = max_of(v);
            most = fmaxf(most, t);
            soft.raise(t, c);
            soft.push(v, c);
        };
        int i = tid;
        for (; i + (kU - 1) * NT < nv; i += kU * NT) {
            Raw<T> r[kU];
#pragma unroll
            for (int u = 0; u < kU; ++u) r[u] = load_raw<T, !kGrad>(from(i + u * NT));
#pragma unroll
            for (int u = 0; u < kU; ++u) push(r[u], i + u * NT);
        }
        for (; i < nv; i += NT) push(load_raw<T, !kGrad>(from(i)), i);
        const int e = nv * W + tid;   // the row's last few tokens
        if (e < V) {
            float one[1] = {kRest && bits[e >> 5] >> (e & 31) & 1 ? -INFINITY : to_f(x[e])};
            most = fmaxf(most, one[0]);
            soft.raise(one[0], c);
            soft.push(one, c);
        }
        Soft all = block_soft<NT>(soft.value(c), c, red);
        if (far(block_max<NT>(most, (float*)red), a.scale))
            all = sums_again<T, NT, kRest>(x, bits, 0, V, c, red);
        const Row r = slots.template finish<kRest>(a, row, all, tl, red);
        if (a.loss && tid == 0) a.loss[row] = r.loss;
        if constexpr (kGrad) {
            if (e < V) grad[e] = from_f<T>(r.gain * exp2_((to_f(x[e]) - r.low) * c));
            // backwards: what was read last is nearest
            i = tid + (nv > tid ? (nv - 1 - tid) / NT * NT : -NT);
            for (; i - (kU - 1) * NT >= 0; i -= kU * NT) {
                Raw<T> q[kU];
#pragma unroll
                for (int u = 0; u < kU; ++u) q[u] = load_raw<T, true>(from(i - u * NT));
#pragma unroll
                for (int u = 0; u < kU; ++u) store_grad<T>(to(i - u * NT), q[u], r, c);
            }
            for (; i >= 0; i -= NT)
                store_grad<T>(to(i), load_raw<T, true>(from(i)), r, c);
            slots.write(r, c, grad, 0, V);
        }
        __syncthreads();   // bits are free for the next row
    }
}

// ---- few rows ----

struct DistillPlan {
    int parts;
    float4* sums;   // [rows][parts]: maximum and sum, largest logit
    size_t bytes;
};
DistillPlan distill_plan(int64_t rows, int64_t V, void* ws) {
    DistillPlan p;
    int64_t parts = (kWantParts + rows - 1) / rows;
    const int64_t most = (V + kMinPart - 1) / kMinPart;
    if (parts > most) parts = most;
    if (parts > kWave) parts = kWave;
    if (parts < (V + kMaxPart - 1) / kMaxPart) parts = (V + kMaxPart - 1) / kMaxPart;
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

template <class T, bool kRest>
__global__ __launch_bounds__(kPartThreads) void k_distill_sums(DistillArgs a, DistillPlan p) {
    extern __shared__ uint32_t bits[];
    __shared__ float2 red[kPartThreads / kWave];
    constexpr int NT = kPartThreads, W = kVec<T>;
    const uint64_t items = (uint64_t)(a.B * a.N) * p.parts;
    for (uint64_t i = blockIdx.x; i < items; i += gridDim.x) {
        const uint32_t row = item_row(i, p.parts, items);
        const int part = (int)(i - (uint64_t)row * p.parts);
        const uint32_t b = row / (uint32_t)a.N, n = row % (uint32_t)a.N;
        if (n >= clamp_rows(a.lengths, b, a.N)) continue;
        const T* x = row_of<T>(a.logits, b, n);
        const float c = a.scale.c;
        int lo, hi;
        part_range((int)a.V, p.parts, part, &lo, &hi);
        if constexpr (kRest) {
            Slots<T, NT> slots;
            slots.load(a, row, x, a.top_lse[row]);
            slots.mark(bits, lo, hi);
        }
        ChunkSoft soft;
        soft.init(a.scale);
        float most = -INFINITY;
        walk_row<T, NT, 4>(x, lo, hi, threadIdx.x, [&](float (&v)[W], int at, int num) {
            if constexpr (kRest) {
                const uint32_t m = bits[(at - lo) >> 5] >> ((at - lo) & 31) & ((1u << W) - 1);
                if (m)
#pragma unroll
                    for (int k = 0; k < W; ++k) v[k] = m >> k & 1 ? -INFINITY : v[k];
            }
            const float t = max_of(v);
            most = fmaxf(most, t);
            soft.raise(t, c);
            soft.push(v, c);
        });
        Soft s = block_soft<NT>(soft.value(c), c, red);
        most = block_max<NT>(most, (float*)red);
        if (most != -INFINITY && far(most, a.scale)) s = sums_again<T, NT, kRest>(x, bits, lo, hi, c, red);
        if (threadIdx.x == 0) p.sums[i] = make_float4(s.m, s.s, most, 0.f);
        __syncthreads();   // bits are free for the next part
    }
}

template <class T, bool kRest, bool kGrad>
__global__ __launch_bounds__(kPartThreads) void k_distill_parts(DistillArgs a, DistillPlan p) {
    __shared__ float2 red[kPartThreads / kWave];
    constexpr int NT = kPartThreads, W = kVec<T>;
    const int parts = kGrad ? p.parts : 1;
    const uint64_t items = (uint64_t)(a.B * a.N) * parts;
    for (uint64_t i = blockIdx.x; i < items; i += gridDim.x) {
        const uint32_t row = item_row(i, parts, items);
        const int part = (int)(i - (uint64_t)row * parts);
        const uint32_t b = row / (uint32_t)a.N, n = row % (uint32_t)a.N;
        T* grad = (T*)a.grad + (size_t)row * a.V;
        int lo, hi;
        part_range((int)a.V, p.parts, part, &lo, &hi);
        if (n >= clamp_rows(a.lengths, b, a.N)) {
            if (a.loss && part == 0 && threadIdx.x == 0) a.loss[row] = 0.f;
            if constexpr (kGrad) write_zeros<T, NT>(grad, lo, hi);
            continue;
        }
        const T* x = row_of<T>(a.logits, b, n);
        const float c = a.scale.c, tl = kRest ? a.top_lse[row] : 0.f;
        Slots<T, NT> slots;
        slots.load(a, row, x, tl);
        const int lane = threadIdx.x % kWave;
        const float4 s = lane < p.parts ? p.sums[(size_t)row * p.parts + lane]
                                        : make_float4(-FLT_MAX, 0.f, 0.f, 0.f);
        const Row r = slots.template finish<kRest>(a, row, wave_soft({s.x, s.y}, c), tl, red);
        if (a.loss && part == 0 && threadIdx.x == 0) a.loss[row] = r.loss;
        if constexpr (kGrad) {
            walk_row<T, NT, 4, true>(x, lo, hi, threadIdx.x, [&](const float (&v)[W], int at, int num) {
                float y[W];
#pragma unroll
                for (int k = 0; k < W; ++k) y[k] = r.gain * exp2_((v[k] - r.low) * c);
                if (num == W)
                    store_raw<T>(grad + at, pack<T>(y));
                else
                    grad[at] = from_f<T>(y[0]);
            });
            slots.write(r, c, grad, lo, hi);
        }
    }
}

}  // namespace

size_t distill_workspace(int, int64_t B, int64_t N, int64_t V, int64_t) {
    return distill_plan(B * N, V, nullptr).bytes;
}

hipError_t launch_distill(const DistillArgs& a, hipStream_t s) {
    hipError_t e = hipSuccess;
    with_type(a.dtype, [&](auto t) {
        using T = decltype(t);
        const int64_t rows = a.B * a.N;
        const int V = (int)a.V;
        const DistillPlan p = distill_plan(rows, V, a.ws);
        if (p.parts > 1) {
            const unsigned grid = row_grid(rows * p.parts, kPartThreads);
            const unsigned one = row_grid(rows, kPartThreads);
            // bits of a part's tokens
            const size_t lds = ((size_t)(V + p.parts - 1) / p.parts + 63) / 64 * 64 / 8;
            if (a.top_lse) {
                k_distill_sums<T, true><<<grid, kPartThreads, lds, s>>>(a, p);
                if ((e = hipGetLastError()) != hipSuccess) return;
                if (a.grad)
                    k_distill_parts<T, true, true><<<grid, kPartThreads, 0, s>>>(a, p);
                else
                    k_distill_parts<T, true, false><<<one, kPartThreads, 0, s>>>(a, p);
            } else {
                k_distill_sums<T, false><<<grid, kPartThreads, 0, s>>>(a, p);
                if ((e = hipGetLastError()) != hipSuccess) return;
                if (a.grad)
                    k_distill_parts<T, false, true><<<grid, kPartThreads, 0, s>>>(a, p);
                else
                    k_distill_parts<T, false, false><<<one, kPartThreads, 0, s>>>(a, p);
            }
            return;
        }
        const size_t lds = a.top_lse ? (size_t)(V + 31) / 32 * 4 : 0;
        auto go = [&](auto nt) {
            constexpr int NT = decltype(nt)::value;
            const unsigned g = row_grid(rows, NT);
            if (a.top_lse && a.grad)
                k_distill<T, NT, true, true><<<g, NT, lds, s>>>(a);
            else if (a.top_lse)
                k_distill<T, NT, true, false><<<g, NT, lds, s>>>(a);
            else if (a.grad)
                k_distill<T, NT, false, true><<<g, NT, 0, s>>>(a);
            else
                k_distill<T, NT, false, false><<<g, NT, 0, s>>>(a);
        };
        // A wave a row while the rows fill the chip so: its sums need no barrier.  Gradients of 64
        // slots, us a call by 64 / 256 / 512 threads: 16384 rows of 1100 33 / 75 / 136, 8192 of 8000
        // 77 / 80 / 96, 4096 of 16000 71 / 66 / 72, 2048 of 32000 75 / 66 / 63.
        if (V <= 1024 || (V <= 8192 && rows >= 2048))
            go(std::integral_constant<int, 64>{});
        else if (V <= 24576)
            go(std::integral_constant<int, 256>{});
        else
            go(std::integral_constant<int, 512>{});
    });
    return e == hipSuccess ? hipGetLastError() : e;
}

}  // namespace tsc
