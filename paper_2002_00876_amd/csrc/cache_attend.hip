// cache_attend.hip -- attention of drafted tokens over a paged cache.
//
// The G = Hq / Hk query heads of a key head and a sequence's drafts make the rows of one product:
// row r = i G + g is draft i, head g.  Keys and values are read once for all of a tile's rows, with the
// running maximum and sum of each row's softmax.
//
// On the matrix cores the scores are formed transposed, S^T = K Q^T: a lane then holds the scores of
// one row (its column, lane % 16) at four slots a tile, so that maxima and sums are the lane's own but
// for two exchanges, and the numerators are at once the right operand of O^T = V^T P^T.  The contraction
// over slots may run in any order: operand element (quarter q, j) stands for slot 16 (j / 4) + 4 q + j % 4
// of 32, which is where the two score tiles left it.  V^T is read from LDS, where V lies as it does in
// the cache, by the transposing read, four slots of one element a lane.
//
// Numerators are rounded to the cache's type for the product (their sum is not): each is off by half a
// step at most, as the values are themselves, and the products are summed in 32 bits.
#include "cache.h"
#include "internal.h"

namespace tsc {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kWords = kMaxNodes / 32;
constexpr int kSplitBatch = 512;      // most sequences whose slots are divided among workgroups
constexpr int kWant = 512;            // workgroups that fill the chip
constexpr float kLow = -1e30f;        // below every score
constexpr float kNone = -1e36f;       // where a running maximum begins: below kLow * scale, the floats far

// Numerators are at most 2^kUp: float16's smallest normal number would otherwise be 2^-14 of the
// largest, and a long context's many small ones would lose their digits or vanish.
template <class T>
constexpr float kUp = std::is_same_v<T, F16> ? 14.f : 0.f;

typedef float F4 __attribute__((ext_vector_type(4)));
typedef uint32_t Quad __attribute__((ext_vector_type(4)));
typedef short S4 __attribute__((ext_vector_type(4)));
typedef short S8 __attribute__((ext_vector_type(8)));
typedef __bf16 B8 __attribute__((ext_vector_type(8)));
typedef _Float16 H8 __attribute__((ext_vector_type(8)));

template <class T>
__device__ __forceinline__ F4 mma(S8 a, S8 b, F4 c) {
    if constexpr (std::is_same_v<T, Bf16>)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(B8, a),
                                                       __builtin_bit_cast(B8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(H8, a),
                                                      __builtin_bit_cast(H8, b), c, 0, 0, 0);
}

// Four rows of 16 elements, 8 bytes a lane of each 16, turned: a lane gets its column's four
__device__ __forceinline__ S4 read_turned(const short* at) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) S4*)at);
}

// ---- how the slots are divided ----
//
// A unit is a tile's walk over KU slots.  All units of the call are cut into pieces of `per` units, so
// that about kWant pieces make up the call whatever the lengths; a workgroup takes one piece.
struct AttendPlan {
    int tiles;        // row tiles of a key head, of N drafts
    int least;        // units of a piece, at least
    bool split;
    unsigned grid;
    int* per;         // workspace: units of a piece
    int* base;        // [B]: first part of each sequence
    float2* ml;       // [parts][rows of a tile]: maximum (of exponents to base 2) and sum
    float* o;         // [parts][rows of a tile][D]
    size_t bytes;
};

struct Shape {
    int rows, units, tiles, pieces;   // of a sequence: rows, units of a row tile, its row tiles, pieces
};

__device__ __forceinline__ int slots_seen(const AttendArgs& a, int64_t b, int n) {
    return min(slots_before(a.c, b) + n, a.c.M * a.c.S);
}

template <int TR, int KU>
__device__ __forceinline__ Shape shape_of(const AttendArgs& a, int64_t b, int per) {
    const int n = new_tokens(a.c, b, a.N), G = a.Hq / a.Hk;
    Shape s;
    s.rows = n * G;
    s.tiles = (s.rows + TR - 1) / TR;
    s.units = n ? (slots_seen(a, b, n) + KU - 1) / KU : 0;
    s.pieces = max(1, (s.units + per - 1) / per);
    return s;
}

struct Piece {
    int64_t b;
    int head, tile, piece, per, part;   // part < 0: the whole row
    Shape s;
};

struct PlanShared {
    uint64_t units[kWaves];
    int sum[2][kWaves];
    int found[3];
};

// Which piece this workgroup takes; false: none
template <int TR, int KU>
__device__ bool find_piece(const AttendArgs& a, const AttendPlan& p, PlanShared& sh, Piece* w) {
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    int id;
    if (!p.split) {
        const int each = a.Hk * p.tiles;
        const int total = (int)a.B * each, many = (total + 7) / 8;
        id = (int)(blockIdx.x % 8) * many + (int)(blockIdx.x / 8);
        if ((int)(blockIdx.x / 8) >= many || id >= total) return false;
        w->b = id / each;
        w->per = 1 << 30;
        w->s = shape_of<TR, KU>(a, w->b, w->per);
        id -= (int)w->b * each;
        w->head = id / p.tiles;
        w->tile = id % p.tiles;
        w->piece = 0;
        w->part = -1;
        return true;
    }
    constexpr int kEach = kSplitBatch / kThreads;
    uint64_t units = 0;
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const int b = tid * kEach + k;
        if (b < a.B) {
            const Shape s = shape_of<TR, KU>(a, b, 1);
            units += (uint64_t)s.units * s.tiles;
        }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) units += __shfl_xor(units, o, kWave);
    if (lane == 0) sh.units[wave] = units;
    __syncthreads();
    units = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) units += sh.units[i];
    units *= a.Hk;
    const int per = max(p.least, (int)min((units + kWant - 1) / kWant, (uint64_t)1 << 30));
    // workgroups and parts of the sequences before a thread's own
    int mine[kEach], parts[kEach], all = 0, all_parts = 0;
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const int b = tid * kEach + k;
        mine[k] = parts[k] = 0;
        if (b < a.B) {
            const Shape s = shape_of<TR, KU>(a, b, per);
            mine[k] = a.Hk * (s.tiles * s.pieces + p.tiles - s.tiles);
            parts[k] = s.pieces > 1 ? a.Hk * s.tiles * s.pieces : 0;
        }
        all += mine[k];
        all_parts += parts[k];
    }
    int before = all, before_parts = all_parts;
#pragma unroll
    for (int o = 1; o < kWave; o *= 2) {
        const int x = __shfl_up(before, o, kWave), y = __shfl_up(before_parts, o, kWave);
        if (lane >= o) before += x, before_parts += y;
    }
    if (lane == kWave - 1) sh.sum[0][wave] = before, sh.sum[1][wave] = before_parts;
    __syncthreads();
    before -= all;
    before_parts -= all_parts;
    int total = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
        if (i < wave) before += sh.sum[0][i], before_parts += sh.sum[1][i];
        total += sh.sum[0][i];
    }
    // workgroups of an XCD take neighbouring pieces: row tiles of the same slots share its L2
    const int many = (total + 7) / 8;
    id = (int)(blockIdx.x % 8) * many + (int)(blockIdx.x / 8);
    const bool any = (int)(blockIdx.x / 8) < many && id < total;
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const int b = tid * kEach + k;
        if (blockIdx.x == 0 && b < a.B) p.base[b] = before_parts;
        if (any && id >= before && id < before + mine[k])
            sh.found[0] = b, sh.found[1] = before, sh.found[2] = before_parts;
        before += mine[k];
        before_parts += parts[k];
    }
    if (blockIdx.x == 0 && tid == 0) *p.per = per;
    __syncthreads();
    if (!any) return false;
    w->b = sh.found[0];
    id -= sh.found[1];
    w->per = per;
    w->s = shape_of<TR, KU>(a, w->b, per);
    const int working = a.Hk * w->s.tiles * w->s.pieces;
    if (id < working) {
        w->tile = id % w->s.tiles;
        id /= w->s.tiles;
        w->head = id % a.Hk;
        w->piece = id / a.Hk;
        w->part = w->s.pieces > 1 ? sh.found[2] + (w->head * w->s.tiles + w->tile) * w->s.pieces + w->piece
                                  : -1;
    } else {
        id -= working;
        const int rest = p.tiles - w->s.tiles;
        w->head = id / rest;
        w->tile = w->s.tiles + id % rest;
        w->piece = 0;
        w->part = -1;
    }
    return true;
}

// ---- who sees whom ----

// Bit j of node i's words: draft i follows draft j, or is j.  Steps of 1, 2, 4, ... drafts towards the
// text: after as many as N has bits every one is known.  Every thread calls it.
__device__ void find_ancestors(const AttendArgs& a, int64_t b, int n, uint32_t* words, short* up) {
    const int i = threadIdx.x, W = (a.N + 31) / 32;   // kThreads >= kMaxNodes
    uint32_t mine[kWords];
    int parent = -1;
    if (i < n) {
        parent = a.parents[b * a.N + i];
        if (parent >= i) parent = -1;
        if (parent < 0) parent = -1;
    }
#pragma unroll
    for (int w = 0; w < kWords; ++w) mine[w] = i / 32 == w ? 1u << (i % 32) : 0u;
    for (int reach = 1; reach < n; reach *= 2) {
        if (i < n) {
#pragma unroll
            for (int w = 0; w < kWords; ++w)
                if (w < W) words[i * W + w] = mine[w];
            up[i] = (short)parent;
        }
        __syncthreads();
        if (i < n && parent >= 0) {
#pragma unroll
            for (int w = 0; w < kWords; ++w)
                if (w < W) mine[w] |= words[parent * W + w];
            parent = up[parent];
        }
        __syncthreads();
    }
    if (i < n)
#pragma unroll
        for (int w = 0; w < kWords; ++w)
            if (w < W) words[i * W + w] = mine[w];
    __syncthreads();
}

// The slots from `at` on, 32 of them, that draft i sees: bit t stands for slot at + t.  `start`: slots
// before the drafts, `end`: all slots
__device__ __forceinline__ uint32_t seen(const AttendArgs& a, const uint32_t* words, int i, int at,
                                         int start, int end) {
    if (at + 32 <= start) return ~0u;
    const int from = at - start;   // first draft of these; negative: so many slots lie before them
    uint32_t bits;
    if (!a.parents) {
        const int k = i + 1 - from;   // of these, those of drafts up to i
        bits = k >= 32 ? ~0u : k <= 0 ? 0u : (1u << k) - 1;
    } else {
        const int W = (a.N + 31) / 32;
        const uint32_t* own = words + i * W;
        if (from >= 0) {
            const int w = from / 32, s = from % 32;
            const uint32_t lo = w < W ? own[w] : 0u, hi = w + 1 < W ? own[w + 1] : 0u;
            bits = (uint32_t)(((uint64_t)hi << 32 | lo) >> s);
        } else {
            bits = own[0] << -from | ((1u << -from) - 1);
        }
    }
    const int left = end - at;
    return left >= 32 ? bits : left <= 0 ? 0u : bits & ((1u << left) - 1);
}

// ---- a tile of slots against a wave's rows ----

template <class T, int DP, int M, int KT>
struct RowsOf {
    static constexpr int KS = DP + 8, VS = DP + 16;   // row strides in LDS: no bank twice
    static constexpr int kPairs = KT / 32;
    S8 q[M][DP / 32];
    F4 o[M][DP / 16];
    float m[M], l[M];

    // first: the wave's first row of the tile's
    __device__ __forceinline__ void load(const AttendArgs& a, const Piece& w, int first) {
        const int lane = threadIdx.x % kWave, G = a.Hq / a.Hk;
#pragma unroll
        for (int x = 0; x < M; ++x) {
            const int r = first + x * 16 + lane % 16, i = r / G, g = r % G;
            const short* at = (const short*)a.q.p + w.b * a.q.sb + i * a.q.sn +
                              (int64_t)(w.head * G + g) * a.q.sh;
#pragma unroll
            for (int s = 0; s < DP / 32; ++s) {
                const int d = s * 32 + lane / 16 * 8;
                q[x][s] = r < w.s.rows && d < a.D ? *(const S8*)(at + d) : S8{};
            }
#pragma unroll
            for (int t = 0; t < DP / 16; ++t) o[x][t] = F4{0.f, 0.f, 0.f, 0.f};
            m[x] = kNone;
            l[x] = 0.f;
        }
    }

    // bits[x][k]: the slots k * 32 + (0..31) that the lane's row x sees
    template <bool kMasked>
    __device__ __forceinline__ void step(const short* K, const short* V, float c2,
                                         const uint32_t (&bits)[M][kPairs]) {
        const int lane = threadIdx.x % kWave, row = lane % 16, quarter = lane / 16;
        F4 s[M][KT / 16];
#pragma unroll
        for (int t = 0; t < KT / 16; ++t) {
#pragma unroll
            for (int x = 0; x < M; ++x) s[x][t] = F4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < DP / 32; ++k) {
                const S8 f = *(const S8*)(K + (t * 16 + row) * KS + k * 32 + quarter * 8);
#pragma unroll
                for (int x = 0; x < M; ++x) s[x][t] = mma<T>(f, q[x][k], s[x][t]);
            }
        }
        S8 p[M][kPairs];
#pragma unroll
        for (int x = 0; x < M; ++x) {
            float most = kLow;
#pragma unroll
            for (int t = 0; t < KT / 16; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if constexpr (kMasked)
                        s[x][t][e] = bits[x][t / 2] >> (t % 2 * 16 + quarter * 4 + e) & 1
                                         ? s[x][t][e] : -INFINITY;
                    most = fmaxf(most, s[x][t][e]);
                }
            most = fmaxf(most, __shfl_xor(most, 16, kWave));
            most = fmaxf(most, __shfl_xor(most, 32, kWave)) * c2 - kUp<T>;
            if (__any(most > m[x])) {
                const float to = fmaxf(most, m[x]), f = exp2_(m[x] - to);
                m[x] = to;
                l[x] *= f;
#pragma unroll
                for (int t = 0; t < DP / 16; ++t) o[x][t] *= f;
            }
            float sum = 0.f;
#pragma unroll
            for (int t = 0; t < KT / 16; ++t) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float y = exp2_(fmaf(s[x][t][e], c2, -m[x]));
                    sum += y;
                    p[x][t / 2][t % 2 * 4 + e] = (short)from_f<T>(y).u;
                }
            }
            l[x] += sum;
        }
#pragma unroll
        for (int t = 0; t < DP / 16; ++t)
#pragma unroll
            for (int k = 0; k < kPairs; ++k) {
                const short* at = V + (k * 32 + quarter * 4 + row / 4) * VS + t * 16 + row % 4 * 4;
                const S4 lo = read_turned(at), hi = read_turned(at + 16 * VS);
                const S8 f = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
                for (int x = 0; x < M; ++x) o[x][t] = mma<T>(f, p[x][k], o[x][t]);
            }
    }

    // The sums of a row's four lanes
    __device__ __forceinline__ void finish() {
#pragma unroll
        for (int x = 0; x < M; ++x) {
            l[x] += __shfl_xor(l[x], 16, kWave);
            l[x] += __shfl_xor(l[x], 32, kWave);
        }
    }
};

__device__ __forceinline__ float lse_of(float m, float l) {
    return l > 0.f ? (m + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
}

template <class T>
__device__ __forceinline__ void store4(T* at, F4 v) {
    uint32_t w[2];
    w[0] = (uint32_t)from_f<T>(v[0]).u | (uint32_t)from_f<T>(v[1]).u << 16;
    w[1] = (uint32_t)from_f<T>(v[2]).u | (uint32_t)from_f<T>(v[3]).u << 16;
    *(uint2*)at = make_uint2(w[0], w[1]);
}

// A tile's rows: element d of row r to `out`, or to a part
template <class T, int TR>
__device__ __forceinline__ void store_row(const AttendArgs& a, const AttendPlan& p, const Piece& w, int r,
                                          int d, F4 o, float m, float l) {
    const int G = a.Hq / a.Hk, at = w.tile * TR + r;
    if (w.part >= 0) {
        if (at >= w.s.rows) return;
        const int64_t row = (int64_t)w.part * TR + r;
        *(F4*)(p.o + row * a.D + d) = o;
        if (d == 0) p.ml[row] = make_float2(m, l);
        return;
    }
    if (at >= a.N * G) return;
    const int64_t row = (w.b * a.N + at / G) * a.Hq + w.head * G + at % G;
    const float f = l > 0.f ? 1.f / l : 0.f;
    store4<T>((T*)a.out + row * a.D + d, o * f);
    if (d == 0 && a.lse) a.lse[row] = lse_of(m, l);
}

// Rows of a tile that are all padding
template <class T, int TR>
__device__ void store_padding(const AttendArgs& a, const Piece& w) {
    const int each = a.D / 4;
    for (int i = threadIdx.x; i < TR * each; i += kThreads)
        store_row<T, TR>(a, AttendPlan{}, w, i / each, i % each * 4, F4{0.f, 0.f, 0.f, 0.f}, 0.f, 0.f);
}

// ---- many rows: a wave takes M * 16 of them, all share the tile of slots ----

template <int DP>
constexpr int kTile = DP > 128 ? 32 : 64;

template <class T, int DP, int M>
struct ManyShared {
    static constexpr int KT = kTile<DP>;
    using R = RowsOf<T, DP, M, KT>;
    short k[2][KT * R::KS];
    short v[2][KT * R::VS];
    int64_t off[3][KT];
    PlanShared plan;
    short up[kMaxNodes];
    uint32_t words[];   // [N][ceil(N / 32)], where there are parents
};

template <class T, int DP, int M>
__global__ __launch_bounds__(kThreads) void k_attend_many(AttendArgs a, AttendPlan p) {
    using Shared = ManyShared<T, DP, M>;
    using R = typename Shared::R;
    constexpr int KT = Shared::KT, TR = 16 * M * kWaves, kRow = DP / 8, kPass = KT * kRow / kThreads;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    Shared& sh = *(Shared*)lds;
    Piece w;
    if (!find_piece<TR, KT>(a, p, sh.plan, &w)) return;
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    if (w.tile >= w.s.tiles) {
        store_padding<T, TR>(a, w);
        return;
    }
    const int n = w.s.rows / (a.Hq / a.Hk), start = slots_before(a.c, w.b), end = slots_seen(a, w.b, n);
    const int lo = w.piece * w.per, hi = min(lo + w.per, w.s.units);
    if (a.parents && (int64_t)hi * KT > start) find_ancestors(a, w.b, n, sh.words, sh.up);
    const int32_t* pages = a.c.pages + w.b * a.c.M;
    const int first = w.tile * TR + wave * 16 * M;
    R rows;
    rows.load(a, w, first);
    auto offset = [&](int u) -> int64_t {
        const int j = u * KT + tid;
        return u < hi && j < end ? slot_offset(a.c, pages, j) : -1;
    };
    Quad k[kPass], v[kPass];
    auto fetch = [&](int u) {
#pragma unroll
        for (int i = 0; i < kPass; ++i) {
            const int x = i * kThreads + tid, slot = x / kRow, d = x % kRow * 8;
            const int64_t off = sh.off[u % 3][slot] + (int64_t)w.head * a.c.sh + d;
            const bool there = sh.off[u % 3][slot] >= 0 && d < a.D;
            k[i] = there ? *(const Quad*)((const short*)a.c.k + off) : Quad{};
            v[i] = there ? *(const Quad*)((const short*)a.c.v + off) : Quad{};
        }
    };
    if (tid < KT) {
        sh.off[lo % 3][tid] = offset(lo);
        sh.off[(lo + 1) % 3][tid] = offset(lo + 1);
    }
    __syncthreads();
    fetch(lo);
    for (int u = lo; u < hi; ++u) {
        short *ks = sh.k[u % 2], *vs = sh.v[u % 2];
#pragma unroll
        for (int i = 0; i < kPass; ++i) {
            const int x = i * kThreads + tid, slot = x / kRow, d = x % kRow * 8;
            *(Quad*)(ks + slot * R::KS + d) = k[i];
            *(Quad*)(vs + slot * R::VS + d) = v[i];
        }
        __syncthreads();
        if (u + 1 < hi) fetch(u + 1);
        int64_t next = -1;
        if (tid < KT) next = offset(u + 2);
        uint32_t bits[M][R::kPairs];
        if ((int64_t)(u + 1) * KT > start) {
#pragma unroll
            for (int x = 0; x < M; ++x)
#pragma unroll
                for (int y = 0; y < R::kPairs; ++y) {
                    const int r = min(first + x * 16 + lane % 16, w.s.rows - 1);
                    bits[x][y] = seen(a, sh.words, r / (a.Hq / a.Hk), u * KT + y * 32, start, end);
                }
            rows.template step<true>(ks, vs, a.c2, bits);
        } else {
            rows.template step<false>(ks, vs, a.c2, bits);
        }
        if (tid < KT) sh.off[(u + 2) % 3][tid] = next;
    }
    rows.finish();
#pragma unroll
    for (int x = 0; x < M; ++x) {
        const int r = wave * 16 * M + x * 16 + lane % 16;
        const bool on = w.tile * TR + r < w.s.rows;
#pragma unroll
        for (int t = 0; t < DP / 16; ++t) {
            const int d = t * 16 + lane / 16 * 4;
            if (d < a.D)
                store_row<T, TR>(a, p, w, r, d, on ? rows.o[x][t] : F4{0.f, 0.f, 0.f, 0.f}, rows.m[x],
                                 on ? rows.l[x] : 0.f);
        }
    }
}

// ---- few rows: every wave takes all of them, and slots of its own ----

template <class T, int DP, int M>
struct FewShared {
    static constexpr int KT = 32;
    using R = RowsOf<T, DP, M, KT>;
    struct Wave {
        short k[KT * R::KS];
        short v[KT * R::VS];
    };
    union {
        Wave wave[kWaves];
        float o[kWaves][M * 16][DP];
    };
    float2 ml[kWaves][M * 16];
    PlanShared plan;
    short up[kMaxNodes];
    uint32_t words[];
};

template <class T, int DP, int M>
__global__ __launch_bounds__(kThreads) void k_attend_few(AttendArgs a, AttendPlan p) {
    using Shared = FewShared<T, DP, M>;
    using R = typename Shared::R;
    constexpr int KT = Shared::KT, KU = KT * kWaves, TR = 16 * M, kRow = DP / 8, kPass = KT * kRow / kWave;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    Shared& sh = *(Shared*)lds;
    Piece w;
    if (!find_piece<TR, KU>(a, p, sh.plan, &w)) return;
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    if (w.tile >= w.s.tiles) {
        store_padding<T, TR>(a, w);
        return;
    }
    const int n = w.s.rows / (a.Hq / a.Hk), start = slots_before(a.c, w.b), end = slots_seen(a, w.b, n);
    const int lo = w.piece * w.per, hi = min(lo + w.per, w.s.units);
    if (a.parents && (int64_t)hi * KU > start) find_ancestors(a, w.b, n, sh.words, sh.up);
    const int32_t* pages = a.c.pages + w.b * a.c.M;
    R rows;
    rows.load(a, w, w.tile * TR);
    short *ks = sh.wave[wave].k, *vs = sh.wave[wave].v;
    // a lane's slot of the wave's tile of unit u (its lanes' first half has one each)
    auto offset = [&](int u) -> int64_t {
        const int j = u * KU + wave * KT + lane % KT;
        return u < hi && j < end ? slot_offset(a.c, pages, j) : -1;
    };
    Quad k[kPass], v[kPass];
    auto fetch = [&](int64_t own) {
#pragma unroll
        for (int i = 0; i < kPass; ++i) {
            const int x = i * kWave + lane, slot = x / kRow, d = x % kRow * 8;
            const int64_t at = __shfl(own, slot, kWave), off = at + (int64_t)w.head * a.c.sh + d;
            const bool there = at >= 0 && d < a.D;
            k[i] = there ? *(const Quad*)((const short*)a.c.k + off) : Quad{};
            v[i] = there ? *(const Quad*)((const short*)a.c.v + off) : Quad{};
        }
    };
    fetch(offset(lo));
    int64_t next = offset(lo + 1);
    for (int u = lo; u < hi; ++u) {
#pragma unroll
        for (int i = 0; i < kPass; ++i) {
            const int x = i * kWave + lane, slot = x / kRow, d = x % kRow * 8;
            *(Quad*)(ks + slot * R::KS + d) = k[i];
            *(Quad*)(vs + slot * R::VS + d) = v[i];
        }
        // the wave's own tile: its stores come before its reads without a barrier
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (u + 1 < hi) {
            fetch(next);
            next = offset(u + 2);
        }
        const int at = u * KU + wave * KT;
        uint32_t bits[M][1];
        if (at < end) {
            if (at + KT > start) {
#pragma unroll
                for (int x = 0; x < M; ++x) {
                    const int r = min(w.tile * TR + x * 16 + lane % 16, w.s.rows - 1);
                    bits[x][0] = seen(a, sh.words, r / (a.Hq / a.Hk), at, start, end);
                }
                rows.template step<true>(ks, vs, a.c2, bits);
            } else {
                rows.template step<false>(ks, vs, a.c2, bits);
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    rows.finish();
    __syncthreads();   // the tiles make room for the waves' sums
#pragma unroll
    for (int x = 0; x < M; ++x) {
        const int r = x * 16 + lane % 16;
#pragma unroll
        for (int t = 0; t < DP / 16; ++t) *(F4*)&sh.o[wave][r][t * 16 + lane / 16 * 4] = rows.o[x][t];
        if (lane < 16) sh.ml[wave][r] = make_float2(rows.m[x], rows.l[x]);
    }
    __syncthreads();
    const int each = a.D / 4;
    for (int i = tid; i < TR * each; i += kThreads) {
        const int r = i / each, d = i % each * 4;
        const bool on = w.tile * TR + r < w.s.rows;
        float m = kNone, l = 0.f;
        F4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int y = 0; y < kWaves; ++y) m = fmaxf(m, sh.ml[y][r].x);
#pragma unroll
        for (int y = 0; y < kWaves; ++y) {
            const float f = exp2_(sh.ml[y][r].x - m);
            l += f * sh.ml[y][r].y;
            o += f * *(const F4*)&sh.o[y][r][d];
        }
        store_row<T, TR>(a, p, w, r, d, on ? o : F4{0.f, 0.f, 0.f, 0.f}, m, on ? l : 0.f);
    }
}

// ---- the parts of a row together ----

// A wave a row
template <class T, int TR, int KU>
__global__ __launch_bounds__(kThreads) void k_attend_join(AttendArgs a, AttendPlan p) {
    const int lane = threadIdx.x % kWave, G = a.Hq / a.Hk;
    const int64_t rows = a.B * a.N * a.Hq, step = (int64_t)gridDim.x * kWaves;
    for (int64_t row = (int64_t)blockIdx.x * kWaves + threadIdx.x / kWave; row < rows; row += step) {
        const int64_t b = row / ((int64_t)a.N * a.Hq);
        const int rest = (int)(row - b * a.N * a.Hq), i = rest / a.Hq, h = rest % a.Hq;
        const Shape s = shape_of<TR, KU>(a, b, *p.per);
        const int at = i * G + h % G, tile = at / TR;
        if (s.pieces < 2 || tile >= s.tiles) continue;   // written as a whole
        float m = kNone, l = 0.f;
        F4 o = {0.f, 0.f, 0.f, 0.f};
        if (at < s.rows) {
            const int64_t first = ((int64_t)p.base[b] + ((h / G) * s.tiles + tile) * s.pieces) * TR + at % TR;
            for (int y = lane; y < s.pieces; y += kWave) m = fmaxf(m, p.ml[first + (int64_t)y * TR].x);
            m = wave_max_fast(m);
            for (int y = 0; y < s.pieces; ++y) {
                const int64_t part = first + (int64_t)y * TR;
                const float2 ml = p.ml[part];
                const float f = exp2_(ml.x - m);
                l += f * ml.y;
                if (lane * 4 < a.D) o += f * *(const F4*)(p.o + part * a.D + lane * 4);
            }
        }
        const float f = l > 0.f ? 1.f / l : 0.f;
        if (lane * 4 < a.D) store4<T>((T*)a.out + row * a.D + lane * 4, o * f);
        if (lane == 0 && a.lse) a.lse[row] = lse_of(m, l);
    }
}

// ---- launches ----

// Rows of a tile and slots of a unit of the kernel that a call takes
struct Choice {
    int few, m;
    int rows() const { return 16 * m * (few ? 1 : kWaves); }
};
Choice choose(int64_t N, int64_t Hq, int64_t Hk) {
    const int64_t rows = N * (Hq / Hk);
    if (rows <= 16) return {1, 1};
    if (rows <= 32) return {1, 2};
    if (rows <= 64) return {0, 1};
    return {0, 2};
}

AttendPlan attend_plan(int64_t B, int64_t N, int64_t Hq, int64_t Hk, int64_t D, void* ws) {
    const Choice c = choose(N, Hq, Hk);
    const int64_t TR = c.rows();
    AttendPlan p{};
    p.tiles = (int)((N * (Hq / Hk) + TR - 1) / TR);
    p.split = B <= kSplitBatch;
    p.least = c.few ? 1 : 2;
    const int64_t items = B * Hk * p.tiles;
    p.grid = (unsigned)((items + (p.split ? kWant : 0) + 7) / 8 * 8);
    size_t off = 0;
    auto take = [&](size_t bytes) {
        char* at = (char*)ws + off;
        off += (bytes + 255) / 256 * 256;
        return at;
    };
    if (p.split) {
        // a row tile of several pieces has at most twice the full ones, of which there are kWant at most
        const size_t parts = 2 * kWant;
        p.per = (int*)take(sizeof(int));
        p.base = (int*)take(sizeof(int) * B);
        p.ml = (float2*)take(sizeof(float2) * parts * TR);
        p.o = (float*)take(sizeof(float) * parts * TR * D);
    }
    p.bytes = off;
    return p;
}

template <class K, class... A>
hipError_t launch_lds(AllowLds& allow, size_t most, K kernel, unsigned grid, size_t lds, hipStream_t s,
                      const A&... args) {
    const hipError_t e = allow(most, kernel);
    if (e != hipSuccess) return e;
    kernel<<<grid, kThreads, lds, s>>>(args...);
    return hipGetLastError();
}

template <class T, int DP, int M, bool kFew>
hipError_t attend_as(const AttendArgs& a, const AttendPlan& p, hipStream_t s) {
    using Shared = std::conditional_t<kFew, FewShared<T, DP, M>, ManyShared<T, DP, M>>;
    constexpr int TR = 16 * M * (kFew ? 1 : kWaves), KU = kFew ? 32 * kWaves : kTile<DP>;
    static AllowLds allow;
    const size_t words = a.parents ? (size_t)a.N * ((a.N + 31) / 32) * sizeof(uint32_t) : 0;
    const size_t most = sizeof(Shared) + (size_t)kMaxNodes * kWords * sizeof(uint32_t);
    hipError_t e;
    if constexpr (kFew)
        e = launch_lds(allow, most, k_attend_few<T, DP, M>, p.grid, sizeof(Shared) + words, s, a, p);
    else
        e = launch_lds(allow, most, k_attend_many<T, DP, M>, p.grid, sizeof(Shared) + words, s, a, p);
    if (e != hipSuccess || !p.split) return e;
    const int64_t rows = a.B * a.N * a.Hq;
    k_attend_join<T, TR, KU><<<row_grid((rows + kWaves - 1) / kWaves, kThreads), kThreads, 0, s>>>(a, p);
    return hipGetLastError();
}

template <class T, int DP>
hipError_t attend_rows(const AttendArgs& a, const AttendPlan& p, hipStream_t s) {
    const Choice c = choose(a.N, a.Hq, a.Hk);
    if (c.few)
        return c.m == 1 ? attend_as<T, DP, 1, true>(a, p, s) : attend_as<T, DP, 2, true>(a, p, s);
    return c.m == 1 ? attend_as<T, DP, 1, false>(a, p, s) : attend_as<T, DP, 2, false>(a, p, s);
}

template <class T>
hipError_t attend_type(const AttendArgs& a, const AttendPlan& p, hipStream_t s) {
    if (a.D <= 64) return attend_rows<T, 64>(a, p, s);
    if (a.D <= 96) return attend_rows<T, 96>(a, p, s);
    if (a.D <= 128) return attend_rows<T, 128>(a, p, s);
    return attend_rows<T, 256>(a, p, s);
}

}  // namespace

size_t attend_workspace(int64_t B, int64_t N, int64_t Hq, int64_t Hk, int64_t D) {
    return attend_plan(B, N, Hq, Hk, D, nullptr).bytes;
}
int64_t attend_grid(int64_t B, int64_t N, int64_t Hq, int64_t Hk, int64_t) {
    const int64_t TR = choose(N, Hq, Hk).rows();
    return B * Hk * ((N * (Hq / Hk) + TR - 1) / TR) + kWant + 8;
}
hipError_t launch_attend(const AttendArgs& a, hipStream_t s) {
    const AttendPlan p = attend_plan(a.B, a.N, a.Hq, a.Hk, a.D, a.ws);
    return a.dtype == TS_BFLOAT16 ? attend_type<Bf16>(a, p, s) : attend_type<F16>(a, p, s);
}

}  // namespace tsc
