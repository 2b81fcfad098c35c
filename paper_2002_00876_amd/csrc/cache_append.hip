// cache_append.hip -- new keys and values into a paged cache, keys and queries rotated on the way.
//
// A pair (x, y) of a head becomes (x cos a - y sin a, y cos a + x sin a), a = position * freq.  The
// angle is formed in 64 bits and reduced to a part of a turn there: at position 10^6 a 32-bit angle
// would be off by 2^-5.  Sine and cosine of what is left, and the rotation, are 32-bit, rounded once.
#include "cache.h"

namespace tsc {
namespace {

constexpr int kAppendThreads = 256;
constexpr double kTurn = 0.15915494309189533577;   // 1 / (2 pi)

typedef uint32_t Quad __attribute__((ext_vector_type(4)));   // 8 elements of 16 bits

__device__ __forceinline__ float2 cos_sin(int position, float freq) {
    const double t = (double)position * (double)freq * kTurn;
    float2 r;
    sincospif(2.f * (float)(t - rint(t)), &r.y, &r.x);
    return r;
}

template <class T>
__device__ __forceinline__ void unpack8(Quad r, float (&v)[8]) {
    unpack<T>({{r.x, r.y, r.z, r.w}}, v);
}
template <class T>
__device__ __forceinline__ Quad pack8(const float (&v)[8]) {
    const Raw<T> r = pack<T>(v);
    return {r.w[0], r.w[1], r.w[2], r.w[3]};
}

// One workgroup a token
template <class T, bool kNeighbours>
__global__ __launch_bounds__(kAppendThreads) void k_append(AppendArgs a) {
    __shared__ float2 cs[kMaxHead / 2];
    const int tid = threadIdx.x, D8 = a.D / 8, h = a.R / 2;
    const uint32_t tokens = (uint32_t)(a.B * a.N), N = (uint32_t)a.N;
    for (uint32_t token = blockIdx.x; token < tokens; token += gridDim.x) {
        const uint32_t b = token / N;
        const int n = (int)(token % N);
        Quad* q_out = (Quad*)((T*)a.q_out + (size_t)token * a.Hq * a.D);
        if (n >= new_tokens(a.c, b, (int)N)) {
            if (a.q_out)
                for (int i = tid; i < a.Hq * D8; i += kAppendThreads) q_out[i] = Quad{0, 0, 0, 0};
            continue;
        }
        const int slot = slots_before(a.c, b) + n;
        int64_t off = -1;
        if (slot < a.c.M * a.c.S) {
            int at;
            const int page = page_of(a.c, slot, &at);
            off = token_offset(a.c, a.c.pages[(int64_t)b * a.c.M + page], at);
        }
        if (tid < h) cs[tid] = cos_sin(a.positions ? a.positions[token] : slot, a.freqs[tid]);
        __syncthreads();
        // vectors of a head: its pairs (of two vectors each, or one), and what is not rotated
        const int pairs = kNeighbours ? a.R / 8 : a.R / 16, each = pairs + (a.D - a.R) / 8;
        const int step = kAppendThreads / each, c = tid % each;
        const T* k = (const T*)a.k.p + b * a.k.sb + n * a.k.sn;
        const T* q = (const T*)a.q.p + b * a.q.sb + n * a.q.sn;
        T* kc = (T*)a.c.k + off;
        for (int i = tid / each; i < a.Hk + a.Hq; i += step) {
            if (tid >= step * each) break;
            const bool is_k = i < a.Hk;
            if (is_k ? off < 0 : !a.q_out) continue;
            const Quad* x = (const Quad*)(is_k ? k + i * a.k.sh : q + (i - a.Hk) * a.q.sh);
            Quad* y = is_k ? (Quad*)(kc + i * a.c.sh) : q_out + (size_t)(i - a.Hk) * D8;
            if (c >= pairs) {
                const int e = a.R / 8 + c - pairs;
                y[e] = x[e];
            } else if (kNeighbours) {
                float v[8], w[8];
                unpack8<T>(x[c], v);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 t = cs[c * 4 + j];
                    w[2 * j] = v[2 * j] * t.x - v[2 * j + 1] * t.y;
                    w[2 * j + 1] = v[2 * j + 1] * t.x + v[2 * j] * t.y;
                }
                y[c] = pack8<T>(w);
            } else {
                float u[8], v[8], w[8], z[8];
                unpack8<T>(x[c], u);
                unpack8<T>(x[c + pairs], v);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float2 t = cs[c * 8 + j];
                    w[j] = u[j] * t.x - v[j] * t.y;
                    z[j] = v[j] * t.x + u[j] * t.y;
                }
                y[c] = pack8<T>(w);
                y[c + pairs] = pack8<T>(z);
            }
        }
        if (off >= 0) {
            const T* v = (const T*)a.v.p + b * a.v.sb + n * a.v.sn;
            for (int i = tid; i < a.Hk * D8; i += kAppendThreads) {
                const int head = i / D8, e = i % D8;
                ((Quad*)((T*)a.c.v + off + head * a.c.sh))[e] = ((const Quad*)(v + head * a.v.sh))[e];
            }
        }
        __syncthreads();   // cs is free for the next token
    }
}

}  // namespace

hipError_t launch_append(const AppendArgs& a, hipStream_t s) {
    const unsigned grid = row_grid(a.B * a.N, kAppendThreads);
    auto go = [&](auto t) {
        using T = decltype(t);
        if (a.neighbours)
            k_append<T, true><<<grid, kAppendThreads, 0, s>>>(a);
        else
            k_append<T, false><<<grid, kAppendThreads, 0, s>>>(a);
    };
    if (a.dtype == TS_BFLOAT16)
        go(Bf16{});
    else
        go(F16{});
    return hipGetLastError();
}

}  // namespace tsc
