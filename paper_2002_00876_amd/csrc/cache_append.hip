// cache_append.hip -- new keys and values into a paged cache, keys and queries rotated on the way.
//
// A pair (x, y) of a head becomes (x cos a - y sin a, y cos a + x sin a), a = position * freq.  The
// angle is formed in 64 bits and reduced to a part of a turn there: at position 10^6 a 32-bit angle
// would be off by 2^-5.  Sine and cosine of what is left, and the rotation, are 32-bit, rounded once.
//
// Bound by what it reads and writes: 12000 tokens of 32 + 8 + 8 heads of 128 in 65 us, 5.0 TB/s (88 us by a
// workgroup a token, which waits for the page and the angles before it asks for the vectors).
#include "cache.h"

namespace tsc {
namespace {

constexpr int kAppendThreads = 256;
constexpr int kAppendWaves = kAppendThreads / kWave;
// Up to so many tokens the waves of a workgroup share one's heads.  32 + 8 heads of 128, a wave a token and four,
// us a call: 16 tokens 13.2 and 12.8, 512 13.1 and 12.9, 1024 13.1 and 13.2, 2048 16.1 and 18.2, 8192 39 and 55.
constexpr int64_t kFewTokens = 1024;
constexpr double kTurn = 0.15915494309189533577;   // 1 / (2 pi)

typedef uint32_t Quad __attribute__((ext_vector_type(4)));   // 8 elements of 16 bits

__device__ __forceinline__ float2 cos_sin(int position, float freq) {
    const double t = (double)position * (double)freq * kTurn;
    const float half = 2.f * (float)(t - rint(t));   // in half turns, in [-1, 1]
    return make_float2(cospif(half), sinpif(half));
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

// What a token's vectors need: each lane has one chunk of a head (a pair of vectors to rotate, one of
// neighbours, or one that is not rotated) and takes that of every so many heads.  `parts` waves share a
// token's heads where tokens are few.  The first heads' vectors are asked for before the angles are formed
// and the page is looked up: the three latencies pass together.  (112 VGPRs: three heads' pairs of vectors, the
// 32-bit parts of a rotation, scalars kept in lanes.  No instruction touches the 20 bytes of scratch that the
// compiler reports.)
template <class T, bool kNeighbours>
__global__ __launch_bounds__(kAppendThreads) void k_append(AppendArgs a, int parts) {
    constexpr int kU = 3;   // heads asked for at once
    __shared__ float2 turns[kAppendWaves][kMaxHead / 2];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, D8 = a.D / 8;
    float2* cs = turns[wave];
    const int pairs = kNeighbours ? a.R / 8 : a.R / 16, each = pairs + (a.D - a.R) / 8;
    const int c = lane % each, step = kWave / each, heads = a.Hk + a.Hq;
    const bool works = lane < step * each;
    const uint32_t N = (uint32_t)a.N;
    const uint64_t items = (uint64_t)(a.B * a.N) * parts;
    for (uint64_t item = (uint64_t)blockIdx.x * kAppendWaves + wave; item < items;
         item += (uint64_t)gridDim.x * kAppendWaves) {
        const uint32_t token = item_row(item, parts, items), b = token / N;
        const int part = (int)(item - (uint64_t)token * parts), n = (int)(token % N);
        Quad* q_out = (Quad*)((T*)a.q_out + (size_t)token * a.Hq * a.D);
        if (n >= new_tokens(a.c, b, (int)N)) {
            for (int i = part * kWave + lane; i < a.Hq * D8; i += parts * kWave) q_out[i] = Quad{0, 0, 0, 0};
            continue;
        }
        const T* k = (const T*)a.k.p + b * a.k.sb + n * a.k.sn;
        const T* q = (const T*)a.q.p + b * a.q.sb + n * a.q.sn;
        const int e = c < pairs ? c : a.R / 8 + c - pairs;   // the lane's vector of a head
        Quad x[kU], y[kU];
        auto load = [&](int i0) {
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                const int i = i0 + u * step * parts;
                if (!works || i >= heads) break;
                const Quad* from = (const Quad*)(i < a.Hk ? k + i * a.k.sh : q + (i - a.Hk) * a.q.sh);
                x[u] = __builtin_nontemporal_load(from + e);
                if (!kNeighbours && c < pairs) y[u] = __builtin_nontemporal_load(from + e + pairs);
            }
        };
        const int begin = part * step + lane / each;
        load(begin);
        const int slot = slots_before(a.c, b) + n;
        int64_t off = -1;
        if (slot < a.c.M * a.c.S) {
            int at;
            const int page = page_of(a.c, slot, &at);
            off = token_offset(a.c, a.c.pages[(int64_t)b * a.c.M + page], at);
        }
        const int position = a.positions ? a.positions[token] : slot;
        for (int i = lane; i < a.R / 2; i += kWave) cs[i] = cos_sin(position, a.freqs[i]);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // a wave's own: no barrier
        for (int i0 = begin; i0 < heads; i0 += kU * step * parts) {
            if (i0 != begin) load(i0);
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                const int i = i0 + u * step * parts;
                if (!works || i >= heads) break;
                if (i < a.Hk && off < 0) continue;
                Quad* to = i < a.Hk ? (Quad*)((T*)a.c.k + off + i * a.c.sh) : q_out + (size_t)(i - a.Hk) * D8;
                if (c >= pairs) {
                    to[e] = x[u];
                } else if (kNeighbours) {
                    float v[8], w[8];
                    unpack8<T>(x[u], v);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float2 t = cs[c * 4 + j];
                        w[2 * j] = v[2 * j] * t.x - v[2 * j + 1] * t.y;
                        w[2 * j + 1] = v[2 * j + 1] * t.x + v[2 * j] * t.y;
                    }
                    to[e] = pack8<T>(w);
                } else {
                    float v[8], w[8], r[8], z[8];
                    unpack8<T>(x[u], v);
                    unpack8<T>(y[u], w);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float2 t = cs[c * 8 + j];
                        r[j] = v[j] * t.x - w[j] * t.y;
                        z[j] = w[j] * t.x + v[j] * t.y;
                    }
                    to[e] = pack8<T>(r);
                    to[e + pairs] = pack8<T>(z);
                }
            }
        }
        if (off >= 0) {
            const T* v = (const T*)a.v.p + b * a.v.sb + n * a.v.sn;
            for (int i = part * kWave + lane; i < a.Hk * D8; i += parts * kWave) {
                const int head = i / D8, at = i % D8;
                ((Quad*)((T*)a.c.v + off + head * a.c.sh))[at] =
                    __builtin_nontemporal_load((const Quad*)(v + head * a.v.sh) + at);
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // cs is free for the next token
    }
}

}  // namespace

hipError_t launch_append(const AppendArgs& a, hipStream_t s) {
    const int64_t tokens = a.B * a.N;
    const int parts = tokens < kFewTokens ? kAppendWaves : 1;
    const unsigned grid = row_grid((tokens * parts + kAppendWaves - 1) / kAppendWaves, kAppendThreads);
    auto go = [&](auto t) {
        using T = decltype(t);
        if (a.neighbours)
            k_append<T, true><<<grid, kAppendThreads, 0, s>>>(a, parts);
        else
            k_append<T, false><<<grid, kAppendThreads, 0, s>>>(a, parts);
    };
    if (a.dtype == TS_BFLOAT16)
        go(Bf16{});
    else
        go(F16{});
    return hipGetLastError();
}

}  // namespace tsc
