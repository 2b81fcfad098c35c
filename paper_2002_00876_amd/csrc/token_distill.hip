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
#include <hip/hip_runtime.h>

#include "token.h"

namespace tsc {
namespace {

constexpr float kMinRest = 9.5367431640625e-7f;   // 2^-20

// Slots of a row, held by the workgroup's first kMaxTop threads (a thread has kMaxTop / NT)
struct Slot {
    int at;    // token, -1: empty
    float t;   // teacher's logit, -inf: empty
};

__device__ __forceinline__ float top_value(const void* p, int dtype, int64_t i) {
    return dtype == TS_FLOAT32    ? ((const float*)p)[i]
           : dtype == TS_BFLOAT16 ? to_f(((const Bf16*)p)[i])
                                  : to_f(((const F16*)p)[i]);
}

template <class T, int NT, bool kRest, bool kGrad>
__global__ __launch_bounds__(NT) void k_distill(DistillArgs a) {
    extern __shared__ uint32_t marks[];   // kRest: a bit for every token
    __shared__ float2 red2[16];
    __shared__ float red[16];
    constexpr int W = kVec<T>, kSlots = kMaxTop > NT ? kMaxTop / NT : 1;
    const int tid = threadIdx.x, V = (int)a.V;
    const float c = a.scale.c, inv_t = a.scale.inv_t;
    for (int64_t row = blockIdx.x; row < a.B * a.N; row += gridDim.x) {
        const int64_t b = row / a.N, n = row % a.N;
        T* grad = (T*)a.grad + row * V;
        if (n >= clamp_rows(a.lengths, b, a.N)) {
            if (a.loss && tid == 0) a.loss[row] = 0.f;
            if constexpr (kGrad)
                for (int v = tid; v < V; v += NT) grad[v] = from_f<T>(0.f);
            continue;
        }
        const T* x = row_of<T>(a.logits, b, n);
        // a teacher's row without a finite logit says nothing: its slots are empty
        const float tl = a.top_lse ? a.top_lse[row] : 0.f;
        Slot slot[kSlots];
        float tm = -FLT_MAX;
#pragma unroll
        for (int q = 0; q < kSlots; ++q) {
            const int k = q * NT + tid;
            slot[q] = {-1, -INFINITY};
            if (k < a.K && tl != -INFINITY) {
                const int at = a.top_indices[row * a.K + k];
                if (at >= 0 && at < V)
                    slot[q] = {at, top_value(a.top_values, a.top_dtype, row * a.K + k)};
            }
            tm = fmaxf(tm, slot[q].t);
        }
        if constexpr (kRest) {
            for (int w = tid; w < (V + 31) / 32; w += NT) marks[w] = 0;
            __syncthreads();
#pragma unroll
            for (int q = 0; q < kSlots; ++q)
                if (slot[q].at >= 0) atomicOr(&marks[slot[q].at >> 5], 1u << (slot[q].at & 31));
            __syncthreads();
        }
        Soft soft = soft_empty();
        walk_row<T, NT, 4>(x, 0, V, tid, [&](const float (&v)[W], int at, int) {
            if constexpr (kRest) {
                const uint32_t bits = marks[at >> 5] >> (at & 31);   // at is a multiple of W
                float u[W];
#pragma unroll
                for (int k = 0; k < W; ++k) u[k] = bits >> k & 1 ? -INFINITY : v[k];
                soft_push(soft, u, c);
            } else {
                soft_push(soft, v, c);
            }
        });
        soft = block_soft<NT>(soft, c, red2);
        // the slots: teacher's p, student's numerators at the common maximum
        float xs[kSlots], p[kSlots];
        Soft own = soft_empty();
#pragma unroll
        for (int q = 0; q < kSlots; ++q) {
            xs[q] = slot[q].at >= 0 ? to_f(x[slot[q].at]) : -INFINITY;
            own.m = fmaxf(own.m, xs[q]);
        }
        Soft all = soft;
        if constexpr (kRest) {
#pragma unroll
            for (int q = 0; q < kSlots; ++q) own.s += exp2_((xs[q] - own.m) * c);
            all = soft_merge(soft, block_soft<NT>(own, c, red2), c);
        }
        float norm;
        if (a.top_lse) {
#pragma unroll
            for (int q = 0; q < kSlots; ++q)
                p[q] = slot[q].at >= 0 ? exp_(slot[q].t * inv_t - tl) : 0.f;
            norm = 1.f;
        } else {
            tm = block_max<NT>(tm, red);
            float s = 0.f;
#pragma unroll
            for (int q = 0; q < kSlots; ++q) s += p[q] = exp2_((slot[q].t - tm) * c);
            s = block_sum<NT>(s, red);
            norm = s > 0.f ? 1.f / s : 0.f;
        }
        float mass = 0.f, kl = 0.f;
        const float ls = all.s > 0.f ? logf(all.s) : 0.f;
#pragma unroll
        for (int q = 0; q < kSlots; ++q) {
            p[q] *= norm;
            if (p[q] > 0.f) {
                mass += p[q];
                kl += p[q] * (logf(p[q]) - ((xs[q] - all.m) * inv_t - ls));
            }
        }
        mass = block_sum<NT>(mass, red);
        kl = block_sum<NT>(kl, red);
        float keep = mass > 0.f ? 1.f : 0.f;   // outside the slots: keep * exp(s_v / T - low)
        if constexpr (kRest) {
            float rest = 1.f - mass;
            if (!(rest > kMinRest)) rest = 0.f;
            const float low = soft.s > 0.f ? (soft.m - all.m) * inv_t + logf(soft.s) - ls : -INFINITY;
            if (rest > 0.f) kl += rest * (logf(rest) - low);
            keep = exp_(low) - rest;
        }
        if (a.loss && tid == 0) a.loss[row] = kl;
        if constexpr (kGrad) {
            const float w = (a.weights ? a.weights[row] : 1.f) * inv_t;
            const float g = soft.s > 0.f ? w * keep / soft.s : 0.f;
            const float m = soft.m;
            walk_row<T, NT, 4>(x, 0, V, tid, [&](const float (&v)[W], int at, int num) {
                float y[W];
#pragma unroll
                for (int k = 0; k < W; ++k) y[k] = g * exp2_((v[k] - m) * c);
                if (num == W)
                    *(Raw<T>*)(grad + at) = pack<T>(y);
                else
                    grad[at] = from_f<T>(y[0]);
            });
            __syncthreads();   // the slots' values come after the walk's
#pragma unroll
            for (int q = 0; q < kSlots; ++q)
                if (slot[q].at >= 0) {
                    const float qk =
                        all.s > 0.f ? exp2_((xs[q] - all.m) * c) / all.s * (kRest || keep > 0.f) : 0.f;
                    grad[slot[q].at] = from_f<T>(w * (qk - (all.s > 0.f ? p[q] : 0.f)));
                }
        }
        __syncthreads();   // marks are free for the next row
    }
}

}  // namespace

size_t distill_workspace(int, int64_t, int64_t, int64_t, int64_t) { return 0; }

hipError_t launch_distill(const DistillArgs& a, hipStream_t s) {
    with_type(a.dtype, [&](auto t) {
        using T = decltype(t);
        const int64_t rows = a.B * a.N;
        const size_t lds = a.top_lse ? (size_t)(a.V + 31) / 32 * 4 : 0;
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
        if (a.V <= 1024)
            go(std::integral_constant<int, 64>{});
        else if (a.V <= 8192)
            go(std::integral_constant<int, 256>{});
        else
            go(std::integral_constant<int, 1024>{});
    });
    return hipGetLastError();
}

}  // namespace tsc
