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
// Products take 16-bit numerators.  Where a lane has one row (tiles of 64 rows), a numerator is two of them, a
// cut one and its rest, whose product costs little beside the read: outputs are as good as with 32-bit numerators
// (off by 2^-15 of a bfloat16's, 2^-21 of a float16's).  Where it has two, numerators are rounded to the cache's
// type (their sum is not): each is off by half a step at most, as the values are themselves, which makes the error
// of an output 1.4 times that of its own rounding.  Calls with both products and with one, us: 64 contexts of
// up to 8000 slots (8 heads of 128, up to 5 drafts of 32 heads) 176 and 174; one of 131072 (4 heads of 64, 7 drafts
// of 28) 38 and 37; 8 trees of 64 drafts of 64 heads over 4500 slots 135 and 113.
//
// Few rows are bound by the read: the first of these calls has 0.96 GB, 5.5 TB/s.  Many are bound by the products
// and the exponentials beside them, which two waves a SIMD do not hide of each other: the last one 640 TFLOP/s.
#include <algorithm>

#include "cache.h"
#include "internal.h"

namespace tsc {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kWords = kMaxNodes / 32;
// Most sequences whose slots are divided among workgroups, a thread each.  One more, of 1000 slots each, us a call:
// 8 heads of 128 180 and 197, one 33 and 31; with one of 32000 slots among others of 200 88 and 690.
constexpr int kSplitBatch = 256;
constexpr int kWant = 512;            // workgroups that fill the chip
// Most rows whose parts are joined by a workgroup each.  So and by tiles, us a call: 256 rows over 16000 slots 25
// and 58, 2048 over 4 x 8000 43 and 50, 4096 over 8 x 4000 47.1 and 45.5, 8192 over 16 x 2000 52 and 43.
constexpr int kWideRows = 2048;
constexpr float kLow = -1e30f;        // below every score
constexpr float kNone = -1e37f;       // where a running maximum begins: below kLow times the largest c2, 1.44e6

// A row's numerators are 2^(exponent - m + kUp), m its maximum so far: float16's smallest normal number
// would otherwise be 2^-14 of the largest, and a long context's many small ones would lose their digits or
// vanish.  m may lag behind by kLag before what was summed is brought up to it (8 rows of 64 by 64 heads
// over 4500 slots: 121 us with no lag, 117 so); float16's largest numerators stay below 2^15.5.
template <class T>
constexpr float kUp = std::is_same_v<T, F16> ? 14.f : 0.f;
template <class T>
constexpr float kLag = std::is_same_v<T, F16> ? 1.f : 8.f;

// An exponent is s c2 - m, whose product is exact (an fma): it is rounded once, after the difference.  m is a
// rounded product, so numerators of a row share a factor of up to 2^(half of m's last place), which the sums share
// too.  Past kFarOut that could leave the types' range: the products are rounded as m is (what they lose is
// what the scores themselves were rounded by), and the largest one's numerator is 2^kUp again.
constexpr float kFarOut = 1 << 20;
// What is taken from exponents of which `most` is the largest
template <class T>
__device__ __forceinline__ float base_of(float most) {
    const float m = most - kUp<T>;
    return most - m > kUp<T> + 0.5f ? most : m;   // floats that far out may lie further apart than kUp
}
__device__ __forceinline__ float rounded_product(float a, float b) {
#pragma clang fp contract(off)
    return a * b;
}

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

// Two numerators, cut to T, and what was cut off, rounded to T.  minus is -1, which the compiler does not know: a
// conversion from float16, a product and a sum are one instruction, a conversion and a difference two.
typedef short S2 __attribute__((ext_vector_type(2)));
struct Split {
    S2 whole, rest;
};
template <class T>
__device__ __forceinline__ Split split(float a, float b, float minus) {
    float u, v;
    S2 whole;
    if constexpr (std::is_same_v<T, Bf16>) {
        const uint32_t x = __float_as_uint(a), y = __float_as_uint(b);
        whole = __builtin_bit_cast(S2, __builtin_amdgcn_perm(y, x, 0x07060302u));
        u = a - __uint_as_float(x & 0xffff0000u);
        v = b - __uint_as_float(y & 0xffff0000u);
    } else {
        const auto h = __builtin_amdgcn_cvt_pkrtz(a, b);
        whole = __builtin_bit_cast(S2, h);
        u = fmaf((float)h[0], minus, a);
        v = fmaf((float)h[1], minus, b);
    }
    return {whole, S2{(short)from_f<T>(u).u, (short)from_f<T>(v).u}};
}

// Four rows of 16 elements, 8 bytes a lane of each 16, turned: a lane gets its column's four
__device__ __forceinline__ S4 read_turned(const short* at) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) S4*)at);
}

// ---- how the slots are divided ----
//
// A unit is a row tile's walk over KU slots of a key head.  A head's units of all row tiles, one tile after
// the other, make a line that is cut into equal stretches, one a workgroup, whatever the lengths: none of
// them waits for a longer one.  All heads' lines are cut alike and their stretches lie side by side, so that
// the heads of a slot, which lie one behind the other in most caches, are read at about the same time (a
// context of 131072 slots, 4 heads of 64: 31 us where each head had stretches of its own, 28 so; no difference
// to 64 contexts of up to 8000 slots with 8 heads of 128).
// What a workgroup has of a row tile is written as a part where the tile goes on elsewhere; a stretch has two
// such ends at most.
struct AttendPlan {
    int tiles;          // row tiles of a key head, of N drafts
    int chunks;         // of kJoinRows rows of a tile that have rows
    int least;          // units of a stretch, at least
    bool split;         // otherwise a workgroup takes one row tile
    unsigned grid;
    int* per;           // workspace: units of a stretch
    uint64_t* before;   // [B]: units of a head's sequences before
    float2* ml;         // [2 * grid][rows of a tile]: maximum (of exponents to base 2) and sum
    float* o;           // [2 * grid][rows of a tile][D]
    size_t bytes;
};

// (Values from LDS and of other lanes that are the same in all lanes, which the compiler cannot know: what
// follows from them is scalar.)
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ uint64_t uniform(uint64_t x) {
    return (uint64_t)(uint32_t)uniform((int)(x >> 32)) << 32 | (uint32_t)uniform((int)(uint32_t)x);
}

// x, of which the compiler keeps nothing ready across the loops before: their registers are needed there
__device__ __forceinline__ int afresh(int x) {
    asm volatile("" : "+v"(x));
    return x;
}

struct Shape {
    int rows, units, tiles;   // of a sequence: rows, units of a row tile, row tiles of a key head
};

__device__ __forceinline__ int2 size_of(const AttendArgs& a, int64_t b) {   // drafts, slots before them
    return make_int2(new_tokens(a.c, b, a.N), slots_before(a.c, b));
}

template <int TR, int KU>
__device__ __forceinline__ Shape shape_of(const AttendArgs& a, int2 size) {
    Shape s;
    s.rows = size.x * (a.Hq / a.Hk);
    s.tiles = (s.rows + TR - 1) / TR;
    s.units = size.x ? (min(size.y + size.x, a.c.M * a.c.S) + KU - 1) / KU : 0;
    return s;
}

// Units [lo, hi) of a row tile, all the same in all lanes
struct Work {
    int64_t b;
    Shape s;
    int n, start, end;              // drafts, slots before them, all slots
    int head, tile, lo, hi, part;   // part < 0: all of its units

    template <int TR, int KU>
    __device__ __forceinline__ void of(const AttendArgs& a, int b_, int2 size) {
        b = b_;
        n = uniform(size.x);
        start = uniform(size.y);
        s = shape_of<TR, KU>(a, make_int2(n, start));
        end = min(start + n, a.c.M * a.c.S);
    }
};

struct WalkShared {
    uint64_t before[kSplitBatch];
    int2 size[kSplitBatch];   // drafts, slots before them
    uint64_t sum[kWaves];
};

template <int TR, int KU>
struct Walk {
    const AttendArgs& a;
    const AttendPlan& p;
    WalkShared& sh;
    uint64_t begin, at, end;   // of the workgroup's stretch
    int per, stretch, head;

    // The stretch; every thread calls it
    __device__ __forceinline__ Walk(const AttendArgs& a_, const AttendPlan& p_, WalkShared& sh_)
        : a(a_), p(p_), sh(sh_) {
        const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
        if (!p.split) {
            const int total = (int)a.B * a.Hk * p.tiles, many = (total + 7) / 8;
            stretch = (int)(blockIdx.x % 8) * many + (int)(blockIdx.x / 8);
            begin = at = 0;
            end = (int)(blockIdx.x / 8) < many && stretch < total;
            per = 1;
            return;
        }
        constexpr int kEach = kSplitBatch / kThreads;
        uint64_t mine[kEach], all = 0;
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            const int b = tid * kEach + k;
            mine[k] = 0;
            if (b < a.B) {
                const int2 size = size_of(a, b);
                const Shape s = shape_of<TR, KU>(a, size);
                mine[k] = (uint64_t)s.units * s.tiles;
                sh.size[b] = size;
            }
            all += mine[k];
        }
        uint64_t upto = all;
#pragma unroll
        for (int o = 1; o < kWave; o *= 2) {
            const uint64_t x = __shfl_up(upto, o, kWave);
            if (lane >= o) upto += x;
        }
        if (lane == kWave - 1) sh.sum[wave] = upto;
        __syncthreads();
        uint64_t start = upto - all, total = 0;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) {
            if (i < wave) start += sh.sum[i];
            total += sh.sum[i];
        }
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            const int b = tid * kEach + k;
            if (b < a.B) sh.before[b] = start;
            if (blockIdx.x == 0 && b < a.B) p.before[b] = start;
            start += mine[k];
        }
        total = uniform(total);
        const int most = (int)(gridDim.x / (unsigned)a.Hk);
        per = uniform(max(p.least, (int)min((total + most - 1) / most, (uint64_t)INT32_MAX)));
        if (blockIdx.x == 0 && tid == 0) *p.per = per;
        // workgroups of an XCD take neighbouring stretches: row tiles of the same slots share its L2
        const int used = (int)((total + per - 1) / per) * a.Hk, many = (used + 7) / 8;
        const int g = (int)(blockIdx.x % 8) * many + (int)(blockIdx.x / 8);
        stretch = g / a.Hk;
        head = g % a.Hk;
        begin = at = uniform(min((uint64_t)stretch * per, total));
        end = (int)(blockIdx.x / 8) < many ? uniform(min(at + per, total)) : at;
        __syncthreads();
    }

    __device__ __forceinline__ bool next(Work* w) {
        if (at >= end) return false;
        if (!p.split) {
            const int each = a.Hk * p.tiles, b = stretch / each, rest = stretch - b * each;
            w->template of<TR, KU>(a, b, size_of(a, b));
            w->head = rest / p.tiles;
            w->tile = rest % p.tiles;
            w->lo = 0;
            w->hi = w->s.units;
            w->part = -1;
            at = end;
            return true;
        }
        int b = 0;
        for (int more = (int)a.B; more - b > 1;) {   // the last sequence that begins here or before
            const int mid = (b + more) / 2;
            if (uniform(sh.before[mid]) <= at)
                b = mid;
            else
                more = mid;
        }
        w->template of<TR, KU>(a, b, sh.size[b]);
        const uint64_t in = at - uniform(sh.before[b]);
        const int tile = uniform((int)(in >> 32 ? in / (uint32_t)w->s.units : (uint32_t)in / (uint32_t)w->s.units));
        w->lo = (int)(in - (uint64_t)tile * w->s.units);
        w->hi = uniform((int)min((uint64_t)w->s.units, w->lo + (end - at)));
        w->head = head;
        w->tile = tile;
        w->part = w->lo == 0 && w->hi == w->s.units ? -1 : 2 * (stretch * a.Hk + head) + (at != begin);
        at += w->hi - w->lo;
        return true;
    }
};

// ---- who sees whom ----

// Bit j of node i's words: draft i follows draft j, or is j.  Steps of 1, 2, 4, ... drafts towards the
// text: after as many as N has bits every one is known.  Every thread calls it, with draft threadIdx.x's
// parent as it was given.
__device__ void find_ancestors(const AttendArgs& a, int n, int parent, uint32_t* words, short* up) {
    const int i = threadIdx.x, W = (a.N + 31) / 32;   // kThreads >= kMaxNodes
    uint32_t mine[kWords];
    if (parent >= i || parent < 0) parent = -1;
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

// ---- a tile of slots in LDS ----
//
// Tiles go from the cache to LDS directly (a wave's load puts its lanes' 16 bytes one behind the other), so
// rows of DP elements are not padded; instead the 16-byte chunks of a row are exchanged by its slot, so that
// neither the sixteen rows of a score operand nor the eight of a turned read meet in a bank.
template <int DP>
struct Tile {
    static constexpr int kRow = DP / 8;   // chunks of a row
    static __device__ __forceinline__ int k_swap(int slot) { return kRow == 8 ? slot >> 1 & 7 : slot & 15; }
    static __device__ __forceinline__ int v_swap(int slot) {
        return kRow == 8 ? (slot >> 1 & 3) * 2 : (slot & 7) * 2;
    }
    // First element of a chunk.  Behind a head's end, where queries are 0 and no output is, any of the
    // head's own will do.
    static __device__ __forceinline__ int element(int chunk, int D) { return chunk * 8 < D ? chunk * 8 : 0; }
};

// What is read for a slot that is not there
__device__ const Quad kZeros[kMaxHead / 8] = {};

// Where a slot's keys and values of a head lie
struct __attribute__((aligned(16))) Place {
    const short* k;
    const short* v;
};
__device__ __forceinline__ Place place_of(const AttendArgs& a, int head, int id, int token, bool there) {
    const int64_t off = there ? token_offset(a.c, id, token) : -1, at = off + (int64_t)head * a.c.sh;
    return off < 0 ? Place{(const short*)kZeros, (const short*)kZeros}
                   : Place{(const short*)a.c.k + at, (const short*)a.c.v + at};
}

// 16 bytes a lane from `from` to LDS: those of the wave's lane l to `to` + 16 l, `to` the same in all.  once:
// nothing else will read them, so they are not kept in the caches.  The load has no result that the compiler
// would wait for, which its builtin makes it do at the next read of any LDS: loads_done() waits.  (M0 holds
// the LDS address and is read one state after it is written.)
__device__ __forceinline__ uint32_t lds_address(const void* at) {
    return (uint32_t)uniform((int)(uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)at);
}
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"   // M0 is reserved: the compiler has to be told all the same
__device__ __forceinline__ void load_to_lds(const short* from, short* to, bool once) {
    const uint32_t at = lds_address(to);
    if (once)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off nt" ::"s"(at), "v"(from)
                     : "memory", "m0");
    else
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(at), "v"(from)
                     : "memory", "m0");
}
// 4 bytes a lane, likewise
__device__ __forceinline__ void load_id_to_lds(const int32_t* from, int32_t* to) {
    const uint32_t at = lds_address(to);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(at), "v"(from)
                 : "memory", "m0");
}
#pragma clang diagnostic pop

// Waits until at most `left` of the wave's loads are on their way (a barrier does not)
template <int left>
__device__ __forceinline__ void loads_done() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0f70 | (left & 15) | (left >> 4) << 14);   // vmcnt
    asm volatile("" ::: "memory");
}

// Operands are read from LDS this many products ahead, and the scheduler keeps to it: without that it
// reads each where it is used, and its latency is all there is to see.
template <int M>
constexpr int kAheadOf = 8 / M;
#define in_step(products, reads)                                      \
    do {                                                              \
        if (products) __builtin_amdgcn_sched_group_barrier(0x008, products, 0); \
        __builtin_amdgcn_sched_group_barrier(0x100, reads, 0);        \
    } while (0)

// ---- a tile of slots against a wave's rows ----

// A lane's part of the queries' operand: row r's elements 32 s + 8 (lane / 16) + (0..7)
__device__ __forceinline__ S8 query(const AttendArgs& a, const Work& w, int r, int s) {
    const int G = a.Hq / a.Hk, i = r / G, g = r % G, d = s * 32 + (int)threadIdx.x % kWave / 16 * 8;
    const short* at = (const short*)a.q.p + w.b * a.q.sb + i * a.q.sn + (int64_t)(w.head * G + g) * a.q.sh;
    return r < w.s.rows && d < a.D ? *(const S8*)(at + d) : S8{};
}

template <class T, int DP, int M, int KT>
struct RowsOf {
    static constexpr int kPairs = KT / 32, kAhead = kAheadOf<M>;
    static constexpr bool kRest = M == 1;   // numerators of two parts
    F4 o[M][DP / 16];
    float m[M], l[M];

    __device__ __forceinline__ void init() {
#pragma unroll
        for (int x = 0; x < M; ++x) {
#pragma unroll
            for (int t = 0; t < DP / 16; ++t) o[x][t] = F4{0.f, 0.f, 0.f, 0.f};
            m[x] = kNone;
            l[x] = 0.f;
        }
    }

    // The scores of a tile in LDS
    __device__ __forceinline__ void scores(const short* K, const S8 (&q)[M][DP / 32], F4 (&s)[M][KT / 16]) {
        const int lane = threadIdx.x % kWave, row = lane % 16, quarter = lane / 16;
        const int swap = Tile<DP>::k_swap(row);   // (the same for row + 16)
        constexpr int kEach = DP / 32, kAll = KT / 16 * kEach;
        auto operand = [&](int i) {
            return *(const S8*)(K + (i / kEach * 16 + row) * DP + ((i % kEach * 4 + quarter) ^ swap) * 8);
        };
        S8 f[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) f[i] = operand(i);
        in_step(0, kAhead);
#pragma unroll
        for (int i = 0; i < kAll; ++i) {
            const int t = i / kEach;
#pragma unroll
            for (int x = 0; x < M; ++x)
                s[x][t] = mma<T>(f[i % kAhead], q[x][i % kEach], i % kEach ? s[x][t] : F4{0.f, 0.f, 0.f, 0.f});
            if (i + kAhead < kAll) f[i % kAhead] = operand(i + kAhead);
            in_step(M, 1);
        }
    }

    // Takes the scores of slots that the lane's row x does not see out; bits: slots k * 32 + (0..31)
    static __device__ __forceinline__ void mask(F4 (&s)[KT / 16], int k, uint32_t bits) {
        const int quarter = threadIdx.x % kWave / 16;
#pragma unroll
        for (int t = 2 * k; t < 2 * k + 2; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                s[t][e] = bits >> (t % 2 * 16 + quarter * 4 + e) & 1 ? s[t][e] : -INFINITY;
    }

    // Scores to numerators
    __device__ __forceinline__ void numerators(F4 (&s)[M][KT / 16], S8 (&p)[M][kPairs], S8 (&rest)[M][kPairs], float c2) {
#pragma unroll
        for (int x = 0; x < M; ++x) {
            float most = kLow;
#pragma unroll
            for (int t = 0; t < KT / 16; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) most = fmaxf(most, s[x][t][e]);
            most = fmaxf(most, __shfl_xor(most, 16, kWave));
            most = base_of<T>(rounded_product(fmaxf(most, __shfl_xor(most, 32, kWave)), c2));
            if (__any(most - m[x] > kLag<T>)) {
                const float to = fmaxf(most, m[x]), f = exp2_(m[x] - to);
                m[x] = to;
                l[x] *= f;
#pragma unroll
                for (int t = 0; t < DP / 16; ++t) o[x][t] *= f;
            }
            float c = c2;
            if (__any(fabsf(m[x]) > kFarOut)) {
                c = 1.f;
#pragma unroll
                for (int t = 0; t < KT / 16; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[x][t][e] = rounded_product(s[x][t][e], c2);
            }
#pragma unroll
            for (int t = 0; t < KT / 16; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[x][t][e] = fmaf(s[x][t][e], c, -m[x]);
#pragma unroll
            for (int t = 0; t < KT / 16; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[x][t][e] = exp2_(s[x][t][e]);
            float sum = 0.f, minus = -1.f;
            asm("" : "+s"(minus));
#pragma unroll
            for (int t = 0; t < KT / 16; ++t) {
                sum += (s[x][t][0] + s[x][t][1]) + (s[x][t][2] + s[x][t][3]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if constexpr (!kRest) {
                        p[x][t / 2][t % 2 * 4 + e] = (short)from_f<T>(s[x][t][e]).u;
                    } else if (e % 2 == 0) {
                        const Split two = split<T>(s[x][t][e], s[x][t][e + 1], minus);
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            p[x][t / 2][t % 2 * 4 + e + i] = two.whole[i];
                            rest[x][t / 2][t % 2 * 4 + e + i] = two.rest[i];
                        }
                    }
                }
            }
            l[x] += sum;
        }
    }

    __device__ __forceinline__ void values(const short* V, const S8 (&p)[M][kPairs], const S8 (&rest)[M][kPairs]) {
        const int lane = threadIdx.x % kWave, row = lane % 16, quarter = lane / 16;
        const int slot = quarter * 4 + row / 4, swap = Tile<DP>::v_swap(slot);   // (the same for slot + 16)
        auto operand = [&](int i) {
            const int t = i / kPairs, k = i % kPairs;
            const short* at = V + (k * 32 + slot) * DP + ((t * 2 + row % 4 / 2) ^ swap) * 8 + row % 2 * 4;
            const S4 lo = read_turned(at), hi = read_turned(at + 16 * DP);
            return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        };
        constexpr int kAll = DP / 16 * kPairs;
        S8 f[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) f[i] = operand(i);
        in_step(0, 2 * kAhead);
#pragma unroll
        for (int i = 0; i < kAll; ++i) {
#pragma unroll
            for (int x = 0; x < M; ++x) {
                o[x][i / kPairs] = mma<T>(f[i % kAhead], p[x][i % kPairs], o[x][i / kPairs]);
                if constexpr (kRest) o[x][i / kPairs] = mma<T>(f[i % kAhead], rest[x][i % kPairs], o[x][i / kPairs]);
            }
            if (i + kAhead < kAll) f[i % kAhead] = operand(i + kAhead);
            in_step((kRest ? 2 : 1) * M, 2);
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

#undef in_step

// (2^kUp is taken out of both before they are added: in the logarithm it would cost four bits)
template <class T>
__device__ __forceinline__ float lse_of(float m, float l) {
    constexpr float one = 1.f / (1 << (int)kUp<T>);
    return l > 0.f ? (m + kUp<T> + __builtin_amdgcn_logf(l * one)) * kLn2 : -INFINITY;
}

template <class T>
__device__ __forceinline__ void store4(T* at, F4 v) {
    uint32_t w[2];
    w[0] = (uint32_t)from_f<T>(v[0]).u | (uint32_t)from_f<T>(v[1]).u << 16;
    w[1] = (uint32_t)from_f<T>(v[2]).u | (uint32_t)from_f<T>(v[3]).u << 16;
    *(uint2*)at = make_uint2(w[0], w[1]);
}

// Where row r of a tile goes: to `out`, or to a part
template <class T, int TR>
struct Target {
    float* part;   // its elements, or NULL
    T* out;        // likewise
    float f;       // what they are multiplied by

    __device__ __forceinline__ Target(const AttendArgs& a, const AttendPlan& p, const Work& w, int r, float m,
                                      float l, bool first) : part(nullptr), out(nullptr), f(1.f) {
        const int G = a.Hq / a.Hk, at = w.tile * TR + r;
        if (w.part >= 0) {
            if (at >= w.s.rows) return;
            const int64_t row = (int64_t)w.part * TR + r;
            part = p.o + row * a.D;
            if (first) p.ml[row] = make_float2(m, l);
        } else if (at < a.N * G) {
            const int64_t row = (w.b * a.N + at / G) * a.Hq + w.head * G + at % G;
            if (at >= w.s.rows) l = 0.f;   // padding
            f = l > 0.f ? 1.f / l : 0.f;
            out = (T*)a.out + row * a.D;
            if (first && a.lse) a.lse[row] = lse_of<T>(m, l);
        }
    }
    __device__ __forceinline__ void store(int d, F4 o) const {
        if (part)
            *(F4*)(part + d) = o;
        else if (out)
            store4<T>(out + d, o * f);
    }
};

// Rows of a tile that are all padding
template <class T, int TR>
__device__ void store_padding(const AttendArgs& a, const Work& w) {
    const int each = a.D / 4;
    for (int i = threadIdx.x; i < TR * each; i += kThreads)
        Target<T, TR>(a, AttendPlan{}, w, i / each, 0.f, 0.f, i % each == 0)
            .store(i % each * 4, F4{0.f, 0.f, 0.f, 0.f});
}

// ---- the kernel ----

// Slots of a unit, and tiles in LDS: one is worked on and the others are on their way.
template <int DP, int M>
constexpr int kSlots = DP == 256 ? 32 : 64;
template <int DP, int M>
constexpr int kStages = DP == 64 ? 4 : 2;

template <int DP, int KT, int NS>
struct AttendShared {
    static constexpr int kGroup = kThreads / KT;   // units whose places are looked up together
    short k[NS][KT * DP];
    short v[NS][KT * DP];
    Place place[kGroup + 1][KT];
    int32_t ids[kThreads];
    WalkShared walk;
    short up[kMaxNodes];
    uint32_t words[];   // [N][ceil(N / 32)], where there are parents
};

// A wave takes 16 * M of a tile's rows, and all take each tile of slots.
template <class T, int DP, int M>
__global__ __launch_bounds__(kThreads, 2) void k_attend(AttendArgs a, AttendPlan p) {
    constexpr int KT = kSlots<DP, M>, NS = kStages<DP, M>, kFar = NS - 1;
    constexpr int TR = 16 * M * kWaves, kRow = DP / 8, kPass = KT * kRow / kThreads;
    using Shared = AttendShared<DP, KT, NS>;
    using R = RowsOf<T, DP, M, KT>;
    constexpr int kGroup = Shared::kGroup, kRing = kGroup + 1;
    static_assert(kFar < kGroup, "the first group has what is fetched before the loop, and its first step's");
    extern __shared__ __attribute__((aligned(16))) char lds[];
    Shared& sh = *(Shared*)lds;
    const int tid = threadIdx.x, lane = tid % kWave, wave = uniform(tid / kWave);
    Walk<TR, KT> walk(a, p, sh.walk);
    Work w;
    while (walk.next(&w)) {
        if (w.tile >= w.s.tiles) {
            store_padding<T, TR>(a, w);
            return;   // there is nothing behind it
        }
        const int lo = w.lo, hi = w.hi, first = w.tile * TR + wave * 16 * M, G = a.Hq / a.Hk;
        const int32_t* pages = a.c.pages + w.b * a.c.M;
        // The places of kGroup units from x on, a thread a slot.  Page numbers go to LDS, too, a group ahead:
        // the compiler would wait for all loads before them if they had a result.
        auto page_at = [&](int x, int* at) { return page_of(a.c, min(x * KT + tid, w.end - 1), at); };
        auto ask = [&](int x) {
            int at;
            load_id_to_lds(pages + page_at(x, &at), sh.ids + wave * kWave);
        };
        auto keep = [&](int x, int id, int at) {
            sh.place[(x + tid / KT - lo) % kRing][tid % KT] = place_of(a, w.head, id, at, x * KT + tid < w.end);
        };
        auto find = [&](int x) {
            int at;
            page_at(x, &at);
            keep(x, sh.ids[tid], at);
        };
        auto fetch = [&](int u) {
            // (some of the places first: LDS would be waited for before each load)
            constexpr int kSome = DP == 256 ? 1 : M == 2 ? kPass / 2 : kPass;
#pragma unroll
            for (int i0 = 0; i0 < kPass; i0 += kSome) {
                Place from[kSome];
#pragma unroll
                for (int i = 0; i < kSome; ++i) from[i] = sh.place[(u - lo) % kRing][((i0 + i) * kThreads + tid) / kRow];
#pragma unroll
                for (int i = 0; i < kSome; ++i) {
                    const int x = (i0 + i) * kThreads + tid, slot = x / kRow, at = x % kRow;
                    const int to = ((i0 + i) * kThreads + wave * kWave) * 8;
                    const short* k = from[i].k + Tile<DP>::element(at ^ Tile<DP>::k_swap(slot), a.D);
                    const short* v = from[i].v + Tile<DP>::element(at ^ Tile<DP>::v_swap(slot), a.D);
                    load_to_lds(k, sh.k[u % NS] + to, p.tiles == 1);
                    load_to_lds(v, sh.v[u % NS] + to, p.tiles == 1);
                }
            }
        };
        // what has to be waited for is asked for at once: parents, queries, page numbers
        const bool forks = a.parents && hi * KT > w.start;
        const int parent = forks && tid < w.n ? a.parents[w.b * a.N + tid] : -1;
        S8 q[M][DP / 32];
#pragma unroll
        for (int x = 0; x < M; ++x)
#pragma unroll
            for (int y = 0; y < DP / 32; ++y) q[x][y] = query(a, w, first + x * 16 + lane % 16, y);
        int token;
        const int page = page_at(lo, &token);
        keep(lo, pages[page], token);
        if (forks) find_ancestors(a, w.n, parent, sh.words, sh.up);
        loads_done<0>();   // (what has results)
        __syncthreads();
        ask(lo + kGroup);
        for (int u = lo; u < min(lo + kFar, hi); ++u) fetch(u);
        R rows;
        rows.init();
        for (int u = lo; u < hi; ++u) {
            // loads come back in order: all but those of the units behind this one are there
            if (u + kFar <= hi)
                loads_done<(kFar - 1) * 2 * kPass>();
            else
                loads_done<0>();
            __syncthreads();
            if (u + kFar < hi) fetch(u + kFar);
            if ((u + kFar - lo) % kGroup == kGroup - 1 && u + kFar + 1 < hi) {
                find(u + kFar + 1);
                ask(u + kFar + 1 + kGroup);   // (its numbers are written where these have been read)
            }
            if (first >= w.s.rows) continue;
            F4 s[M][KT / 16];
            S8 n[M][R::kPairs], rest[M][R::kPairs];
            __builtin_amdgcn_s_setprio(1);   // (the other workgroup's wave then does its exponentials)
            rows.scores(sh.k[u % NS], q, s);
            __builtin_amdgcn_s_setprio(0);
            if ((u + 1) * KT > w.start) {
#pragma unroll
                for (int x = 0; x < M; ++x) {
                    const int i = min(first + x * 16 + lane % 16, w.s.rows - 1) / G;
#pragma unroll
                    for (int y = 0; y < R::kPairs; ++y)
                        R::mask(s[x], y, seen(a, sh.words, i, u * KT + y * 32, w.start, w.end));
                }
            }
            rows.numerators(s, n, rest, a.c2);
            __builtin_amdgcn_s_setprio(1);
            rows.values(sh.v[u % NS], n, rest);
            __builtin_amdgcn_s_setprio(0);
        }
        rows.finish();
        const int own = afresh(lane);
#pragma unroll
        for (int x = 0; x < M; ++x) {
            const Target<T, TR> to(a, p, w, wave * 16 * M + x * 16 + own % 16, rows.m[x], rows.l[x], own < 16);
#pragma unroll
            for (int t = 0; t < DP / 16; ++t) {
                const int d = t * 16 + own / 16 * 4;
                if (d < a.D) to.store(d, rows.o[x][t]);
            }
        }
        loads_done<0>();   // (page numbers)
        __syncthreads();   // LDS is free for the next row tile
    }
}

// ---- the parts of a row together ----

__device__ __forceinline__ uint32_t over(uint64_t x, int per) {   // (64-bit divisions take their time)
    return x >> 32 ? (uint32_t)(x / (uint32_t)per) : (uint32_t)x / (uint32_t)per;
}

// Which parts make up a row tile's rows; pieces = 1: none, it was written as a whole
template <int TR, int KU>
struct Parts {
    int pieces, first, begun, step, rows;

    __device__ __forceinline__ Parts(const AttendArgs& a, const AttendPlan& p, int64_t b, int head, int tile) {
        const int per = *p.per;
        const Shape s = shape_of<TR, KU>(a, size_of(a, b));
        pieces = first = begun = 0;
        step = 2 * a.Hk;
        rows = s.rows - tile * TR;
        if (tile >= s.tiles) return;   // padding
        const uint64_t from = p.before[b] + (uint64_t)tile * s.units;
        const uint32_t g = over(from, per);   // the first stretch that has some of the tile
        pieces = (int)(over(from + s.units - 1, per) - g) + 1;
        // the tile's part of the first stretch is that stretch's second, unless both begin together
        first = 2 * ((int)g * a.Hk + head);
        begun = (uint64_t)g * per != from;
    }
    // Row r of part y
    __device__ __forceinline__ int64_t row(int y, int r) const {
        return (int64_t)(first + step * y + (y == 0 ? begun : 0)) * TR + r;
    }
};

// Adds up a row's parts mine, mine + groups, ...: four elements a lane, from d on
template <class P>
__device__ __forceinline__ void add_parts(const AttendArgs& a, const AttendPlan& p, const P& parts, int r, int d,
                                          int mine, int groups, int pieces, float m, F4* o, float* l) {
    constexpr int kU = 4;   // parts asked for at once
    for (int y = mine; y < pieces; y += kU * groups) {
        float2 ml[kU];
        F4 x[kU];
#pragma unroll
        for (int k = 0; k < kU; ++k) {
            const int64_t z = parts.row(min(y + k * groups, pieces - 1), r);
            ml[k] = p.ml[z];
            x[k] = *(const F4*)(p.o + z * a.D + d);
        }
#pragma unroll
        for (int k = 0; k < kU; ++k) {
            const float f = y + k * groups < pieces ? exp2_(ml[k].x - m) : 0.f;
            *l += f * ml[k].y;
            *o += f * x[k];
        }
    }
}

// Lanes that have four elements of a row each
__device__ __forceinline__ int lanes_across(int D) { return D <= 64 ? 16 : D <= 128 ? 32 : 64; }

constexpr int kJoinRows = 16;

// Many rows, of few parts each: a workgroup takes kJoinRows rows of a tile, a group of lanes a row
template <class T, int TR, int KU>
__global__ __launch_bounds__(kThreads) void k_attend_join(AttendArgs a, AttendPlan p) {
    const int G = a.Hq / a.Hk, across = lanes_across(a.D), d = (int)threadIdx.x % across * 4;
    uint32_t at = blockIdx.x;
    const int chunk = (int)(at % (uint32_t)p.chunks);
    at /= (uint32_t)p.chunks;
    const int tile = (int)(at % (uint32_t)p.tiles);
    at /= (uint32_t)p.tiles;
    const int head = (int)(at % (uint32_t)a.Hk);
    const int64_t b = at / (uint32_t)a.Hk;
    const Parts<TR, KU> parts(a, p, b, head, tile);
    if (parts.pieces == 1) return;
    for (int r = chunk * kJoinRows + (int)threadIdx.x / across; r < (chunk + 1) * kJoinRows;
         r += kThreads / across) {
        const int in = tile * TR + r;
        if (in >= a.N * G) return;
        const int pieces = r < parts.rows ? parts.pieces : 0;
        float m = kNone, l = 0.f;
        for (int y = 0; y < pieces; ++y) m = fmaxf(m, p.ml[parts.row(y, r)].x);
        F4 o = {0.f, 0.f, 0.f, 0.f};
        add_parts(a, p, parts, r, d < a.D ? d : 0, 0, 1, pieces, m, &o, &l);
        const int64_t row = (b * a.N + in / G) * a.Hq + head * G + in % G;
        if (d < a.D) store4<T>((T*)a.out + row * a.D + d, o * (l > 0.f ? 1.f / l : 0.f));
        if (d == 0 && a.lse) a.lse[row] = lse_of<T>(m, l);
    }
}

// Few rows, which may be in many parts: a workgroup a row, whose groups of lanes take every so many parts
template <class T, int TR, int KU>
__global__ __launch_bounds__(kThreads) void k_attend_join_wide(AttendArgs a, AttendPlan p) {
    __shared__ float tops[kWaves];
    __shared__ F4 sums[kWaves][kWave];
    __shared__ float weights[kWaves][kWave];
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave, G = a.Hq / a.Hk;
    const int across = lanes_across(a.D), d = tid % across * 4;
    const uint32_t row = blockIdx.x, each = (uint32_t)(a.N * a.Hq);
    const int64_t b = row / each;
    const int rest = (int)(row % each), i = rest / a.Hq, h = rest % a.Hq;
    const int in = i * G + h % G, r = in % TR;
    const Parts<TR, KU> parts(a, p, b, h / G, in / TR);
    if (parts.pieces == 1) return;
    const int pieces = r < parts.rows ? parts.pieces : 0;
    float m = kNone, l = 0.f;
    for (int y = tid; y < pieces; y += kThreads) m = fmaxf(m, p.ml[parts.row(y, r)].x);
    m = wave_max_fast(m);
    if (lane == 0) tops[wave] = m;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kWaves; ++k) m = fmaxf(m, tops[k]);
    F4 o = {0.f, 0.f, 0.f, 0.f};
    add_parts(a, p, parts, r, d < a.D ? d : 0, tid / across, kThreads / across, pieces, m, &o, &l);
    for (int k = across; k < kWave; k *= 2) {
        l += __shfl_xor(l, k, kWave);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], k, kWave);
    }
    sums[wave][lane] = o;
    weights[wave][lane] = l;
    __syncthreads();
    if (tid >= across) return;
    o = F4{0.f, 0.f, 0.f, 0.f}, l = 0.f;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) o += sums[k][lane], l += weights[k][lane];
    if (d < a.D) store4<T>((T*)a.out + (int64_t)row * a.D + d, o * (l > 0.f ? 1.f / l : 0.f));
    if (d == 0 && a.lse) a.lse[row] = lse_of<T>(m, l);
}

// ---- launches ----

// Row tiles of 64 or 128 rows.  (Heads of more than 128 elements leave no registers for a second row a lane.)  With
// 64 and 128, rows of a key head and us a call: 64 contexts of 500 slots, 64 rows 38 and 42, 65 rows 65 and 44, 256
// rows 132 and 90; 8 of 4000, 64 rows 46 and 50, 65 rows 46.4 and 47.7, 192 rows 81 and 59; one of 8000, 64 rows 26
// and 27, 65 rows 30 and 27, 128 rows 30 and 35.
int sixteens(int64_t N, int64_t Hq, int64_t Hk, int64_t D) { return N * (Hq / Hk) > 64 && D <= 128 ? 2 : 1; }

AttendPlan attend_plan(int64_t B, int64_t N, int64_t Hq, int64_t Hk, int64_t D, void* ws) {
    const int64_t TR = 16 * kWaves * sixteens(N, Hq, Hk, D);
    AttendPlan p{};
    p.tiles = (int)((N * (Hq / Hk) + TR - 1) / TR);
    p.chunks = (int)((std::min(N * (Hq / Hk), TR) + kJoinRows - 1) / kJoinRows);
    p.split = B <= kSplitBatch;
    p.least = 1;
    const int64_t items = B * Hk * p.tiles;
    // (a multiple of 8 of them, as each XCD takes an eighth)
    p.grid = (unsigned)(p.split ? (std::max(kWant / Hk, (int64_t)1) * Hk + 7) / 8 * 8 : (items + 7) / 8 * 8);
    size_t off = 0;
    auto take = [&](size_t bytes) {
        char* at = (char*)ws + off;
        off += (bytes + 255) / 256 * 256;
        return at;
    };
    if (p.split) {
        const size_t parts = 2 * p.grid;
        p.per = (int*)take(sizeof(int));
        p.before = (uint64_t*)take(sizeof(uint64_t) * B);
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

template <class T, int DP, int M>
hipError_t attend_as(const AttendArgs& a, const AttendPlan& p, hipStream_t s) {
    constexpr int TR = 16 * M * kWaves, KT = kSlots<DP, M>;
    using Shared = AttendShared<DP, KT, kStages<DP, M>>;
    static AllowLds allow;
    const size_t words = a.parents ? (size_t)a.N * ((a.N + 31) / 32) * sizeof(uint32_t) : 0;
    const size_t most = sizeof(Shared) + (size_t)kMaxNodes * kWords * sizeof(uint32_t);
    const hipError_t e = launch_lds(allow, most, k_attend<T, DP, M>, p.grid, sizeof(Shared) + words, s, a, p);
    if (e != hipSuccess || !p.split) return e;
    const int64_t rows = a.B * a.N * a.Hq;
    if (rows <= kWideRows)
        k_attend_join_wide<T, TR, KT><<<(unsigned)rows, kThreads, 0, s>>>(a, p);
    else
        k_attend_join<T, TR, KT><<<(unsigned)(a.B * a.Hk * p.tiles * p.chunks), kThreads, 0, s>>>(a, p);
    return hipGetLastError();
}

template <class T, int DP>
hipError_t attend_rows(const AttendArgs& a, const AttendPlan& p, hipStream_t s) {
    if constexpr (DP <= 128)
        if (sixteens(a.N, a.Hq, a.Hk, a.D) == 2) return attend_as<T, DP, 2>(a, p, s);
    return attend_as<T, DP, 1>(a, p, s);
}

template <class T>
hipError_t attend_type(const AttendArgs& a, const AttendPlan& p, hipStream_t s) {
    if (a.D <= 64) return attend_rows<T, 64>(a, p, s);
    if (a.D <= 128) return attend_rows<T, 128>(a, p, s);
    return attend_rows<T, 256>(a, p, s);
}

}  // namespace

size_t attend_workspace(int64_t B, int64_t N, int64_t Hq, int64_t Hk, int64_t D) {
    return attend_plan(B, N, Hq, Hk, D, nullptr).bytes;
}
bool attend_fits(int64_t B, int64_t N, int64_t Hq, int64_t Hk, int64_t D, int64_t slots) {
    const AttendPlan p = attend_plan(B, N, Hq, Hk, D, nullptr);
    if (B * Hk * p.tiles > (int64_t)1 << 23) return false;   // 2^31 threads
    // units of a stretch are an int; 2^35 slots are 2^30 tiles of 32, and each of up to 2^20 row tiles begins another
    return !p.split || B * p.tiles * ((slots + 31) / 32) / (p.grid / Hk) < INT32_MAX;
}
hipError_t launch_attend(const AttendArgs& a, hipStream_t s) {
    const AttendPlan p = attend_plan(a.B, a.N, a.Hq, a.Hk, a.D, a.ws);
    return a.dtype == TS_BFLOAT16 ? attend_type<Bf16>(a, p, s) : attend_type<F16>(a, p, s);
}

}  // namespace tsc
