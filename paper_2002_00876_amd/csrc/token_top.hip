// token_top.hip -- the K largest logits of every row, in order, and the row's log-sum-exp.
//
// Logits are compared as 32-bit keys, a monotone image of the float (-0 counted as 0); a logit
// and its index make one 64-bit word (key, ~index), so that the words of a row are all
// different and their order is that of the result: larger logits first, equal ones by the
// lowest index.
//
// A threshold that K logits reach is found, the logits that reach it go into a list in LDS, and
// each of them finds its place there by counting the larger ones.
//   Rows of up to 1024 logits are held in a wave's registers: the threshold is found by bisection
// (k_top_short).
//   Longer rows take two launches.  k_top_scan guesses the threshold from a sample spread over the
// row: a sample that holds the part f of a row holds about K f of its K largest logits, and the
// logit of rank 1.5 K f + 4 sqrt(K f) + 4 in it lies below the row's K-th, unless the sample
// happens to hold more than half again its share.  Then it reads the row once, in parts where the
// rows are few, for the sums of its softmax, and keeps the vectors of logits that reach the guess;
// with the threshold known its waves never wait for each other.  k_top_pick makes the list from
// the kept vectors.  Where K logits do not reach the guess, or more vectors than are kept do, it
// reads the row again: maxima of groups of logits give a threshold that at least K reach.
//   The scan is bound by its reading: 2048 rows of 131072 bfloat16 98 us, 5.5 TB/s, of which the
// guess takes 10 and keeping vectors 8; the pick (21 us) by the latency of its steps.
//   Where more reach that than the list holds -- many equal logits, or the largest all in a few
// groups -- the threshold is raised by bisection over the whole row, and logits equal to the
// last threshold are taken in the order of their indices.
#include <hip/hip_runtime.h>

#include "token.h"

namespace tsc {
namespace {

constexpr int kCap = 1024;    // logits that the list holds
constexpr int kShort = 1024;  // longest rows that a wave holds in its registers
constexpr int kTopThreads = 256;

__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t u = __float_as_uint(x + 0.0f);   // -0 + 0 = 0
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float of_key(uint32_t k) {
    return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}
__device__ __forceinline__ uint64_t word_of(uint32_t key, int index) {
    return (uint64_t)key << 32 | (uint32_t)~index;
}

template <int kWords>
struct TopSharedOf {
    uint64_t list[kWords];
    float2 red[16];
    int redi[2][16];
    int n;   // words in the list, or vectors noted
};
using TopShared = TopSharedOf<kCap>;

// Number of the workgroup's keys that reach lo; `turn` alternates between calls, which makes
// one barrier enough
template <int NT, int J>
__device__ __forceinline__ int count_keys(const uint32_t (&key)[J], uint32_t lo, int turn,
                                          TopShared* sh) {
    int c = 0;
#pragma unroll
    for (int j = 0; j < J; ++j) c += __popcll(__ballot(key[j] >= lo));
    if constexpr (NT == kWave) return c;
    if (threadIdx.x % kWave == 0) sh->redi[turn & 1][threadIdx.x / kWave] = c;
    __syncthreads();
    c = 0;
#pragma unroll
    for (int w = 0; w < NT / kWave; ++w) c += sh->redi[turn & 1][w];
    return c;
}

// A threshold in [lo, hi) that at least K of the keys reach, K / 8 + 1 more at most where the
// keys allow it; lo where fewer than K reach any other.  hi: none reaches it.  count: how many
// reach the result, if it is not lo.
template <int NT, int J>
__device__ uint32_t threshold(const uint32_t (&key)[J], int K, uint32_t lo, uint32_t hi, int* count,
                              TopShared* sh = nullptr) {
    int turn = 0;
    while (hi - lo > 1) {
        const uint32_t mid = lo + (hi - lo) / 2;
        const int c = count_keys<NT, J>(key, mid, turn++, sh);
        if (c >= K) {
            lo = mid;
            *count = c;
            if (c <= K + K / 8 + 1) break;
        } else {
            hi = mid;
        }
    }
    if constexpr (NT > kWave) __syncthreads();   // redi is free for the next search
    return lo;
}

// The list's words, of logits x, each find their place among them
template <class T, int NT, class S>
__device__ __forceinline__ void write_places(const TopArgs& a, const T* x, uint32_t row, int n,
                                             const S& sh) {
    T* values = (T*)a.values + (size_t)row * a.K;
    int32_t* indices = a.indices + (size_t)row * a.K;
    for (int i = threadIdx.x; i < n; i += NT) {
        const uint64_t w = sh.list[i];
        int place = 0, j = 0;
        for (; j + 4 <= n; j += 4)
#pragma unroll
            for (int k = 0; k < 4; ++k) place += sh.list[j + k] > w;
        for (; j < n; ++j) place += sh.list[j] > w;
        if (place < a.K) {
            const int at = (int)~(uint32_t)w;
            const float v = of_key((uint32_t)(w >> 32));
            values[place] = v == 0.f ? x[at] : from_f<T>(v);   // a key does not know a zero's sign
            indices[place] = at;
        }
    }
}

template <class T, int NT>
__device__ __forceinline__ void write_padding(const TopArgs& a, uint32_t row) {
    for (int k = threadIdx.x; k < a.K; k += NT) {
        ((T*)a.values)[(size_t)row * a.K + k] = from_f<T>(-INFINITY);
        a.indices[(size_t)row * a.K + k] = -1;
    }
    if (a.lse && threadIdx.x == 0) a.lse[row] = -INFINITY;
}

// Puts the threads' hits into the list in the order of (call, thread); have: the words in it
template <int NT, class S>
__device__ __forceinline__ int append_ordered(bool hit, uint64_t word, int have, int most, S& sh) {
    const uint64_t votes = __ballot(hit);
    int before = 0, all = __popcll(votes);
    if constexpr (NT > kWave) {
        if (threadIdx.x % kWave == 0) sh.redi[0][threadIdx.x / kWave] = all;
        __syncthreads();
        all = 0;
#pragma unroll
        for (int w = 0; w < NT / kWave; ++w) {
            if (w < (int)threadIdx.x / kWave) before += sh.redi[0][w];
            all += sh.redi[0][w];
        }
        __syncthreads();
    }
    before += have + __popcll(votes & ((1ull << (threadIdx.x % kWave)) - 1));
    if (hit && before < most) sh.list[before] = word;
    return min(have + all, most);
}

// Rows of up to 64 * J logits, a wave each
template <class T, int J>
__global__ __launch_bounds__(kWave) void k_top_short(TopArgs a) {
    constexpr int NT = kWave;
    __shared__ TopSharedOf<kWave * J> sh;
    const int tid = threadIdx.x, K = a.K, V = a.V;
    const uint32_t rows = (uint32_t)(a.B * a.N), N = (uint32_t)a.N;
    for (uint32_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const uint32_t b = row / N, n = row % N;
        if (n >= clamp_rows(a.lengths, b, N)) {
            write_padding<T, NT>(a, row);
            continue;
        }
        const T* x = row_of<T>(a.logits, b, n);
        float v[J];
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int e = j * NT + tid;
            v[j] = e < V ? to_f(x[e]) : -INFINITY;
        }
        Soft soft = soft_empty();
        uint32_t key[J], mine = 0;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            soft.m = fmaxf(soft.m, v[j]);
            key[j] = j * NT + tid < V ? key_of(v[j]) : 0u;   // 0: below every logit's
            mine = max(mine, key[j]);
        }
#pragma unroll
        for (int j = 0; j < J; ++j) soft.s += exp2_((v[j] - soft.m) * a.scale.c);
        soft = block_soft<NT>(soft, a.scale.c, sh.red);
        if (a.lse && tid == 0) a.lse[row] = soft_lse(soft, a.scale.inv_t);
        const int enough = 2 * K + 64;   // words that are soon counted
        uint32_t lo = 1;                 // every logit's key reaches it
        int c = V;
        if (V > enough) {
            // lanes' largest logits first: what K of them reach, K logits reach
            const uint32_t hi = key_of(INFINITY) + 1;
            const uint32_t one[1] = {mine};
            if (K <= kWave / 2) lo = threshold<NT, 1>(one, K, lo, hi, &c);
            c = count_keys<NT, J>(key, lo, 0, nullptr);
            if (c > enough) lo = threshold<NT, J>(key, K, lo, hi, &c);
        }
        // too many that equal lo: those above it, and the first of these
        const uint32_t first = c > enough ? lo + 1 : lo;
        int have = 0;
#pragma unroll
        for (int j = 0; j < J; ++j)
            if (j * NT < V)
                have = append_ordered<NT>(key[j] >= first, word_of(key[j], j * NT + tid), have,
                                          kWave * J, sh);
        if (c > enough)
            for (int j = 0; j < J && have < K; ++j) {
                uint32_t kj = key[0];
#pragma unroll
                for (int i = 1; i < J; ++i) kj = i == j ? key[i] : kj;
                have = append_ordered<NT>(kj == lo, word_of(lo, j * NT + tid), have, K, sh);
            }
        __syncthreads();
        write_places<T, NT>(a, x, row, have, sh);
        __syncthreads();   // the list is free for the next row
    }
}

// ---- longer rows ----

// Appends the row's logits whose keys reach lo, that of a finite logit, to the list, as far as it
// holds them; sh.n is their number
template <class T, int NT>
__device__ void collect(const T* row, int V, uint32_t lo, TopShared& sh) {
    if (threadIdx.x == 0) sh.n = 0;
    __syncthreads();
    const float least = of_key(lo);
    walk_row<T, NT, 1>(row, 0, V, threadIdx.x, [&](const float (&v)[kVec<T>], int at, int num) {
#pragma unroll
        for (int k = 0; k < kVec<T>; ++k)
            if (k < num && v[k] >= least) {
                const int i = atomicAdd(&sh.n, 1);
                if (i < kCap) sh.list[i] = word_of(key_of(v[k]), at + k);
            }
    });
    __syncthreads();
}

template <class T, int NT>
__device__ int count_row(const T* row, int V, uint32_t lo, TopShared& sh) {
    int c = 0;
    const float least = of_key(lo);
    walk_row<T, NT, 1>(row, 0, V, threadIdx.x, [&](const float (&v)[kVec<T>], int, int num) {
#pragma unroll
        for (int k = 0; k < kVec<T>; ++k) c += k < num && v[k] >= least;
    });
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) c += __shfl_xor(c, o, kWave);
    if (threadIdx.x % kWave == 0) sh.redi[0][threadIdx.x / kWave] = c;
    __syncthreads();
    c = 0;
#pragma unroll
    for (int w = 0; w < NT / kWave; ++w) c += sh.redi[0][w];
    __syncthreads();
    return c;
}

// The logits equal to the one of key `tie`, in the order of their indices, until the list has
// K words
template <class T, int NT>
__device__ int append_equal(const T* row, int V, int K, uint32_t tie, int have, TopShared& sh) {
    for (int base = 0; base < V && have < K; base += NT) {
        const int e = base + (int)threadIdx.x;
        const bool hit = e < V && key_of(to_f(row[e])) == tie;
        have = append_ordered<NT>(hit, word_of(tie, e), have, K, sh);
    }
    __syncthreads();
    return have;
}

// The list from the row itself, where more logits than it holds reach lo.  Leaves the row's K
// largest words in it and perhaps others; returns their number.
template <class T, int NT>
__device__ int select_again(const T* row, int V, int K, uint32_t lo, TopShared& sh) {
    uint32_t hi = key_of(INFINITY) + 1;
    collect<T, NT>(row, V, lo, sh);
    int c = sh.n;
    __syncthreads();
    if (c <= kCap) return c;
    uint32_t mid = lo + 1;   // the usual reason: many that equal lo
    while (hi - lo > 1 && c > kCap) {
        const int m = count_row<T, NT>(row, V, mid, sh);
        if (m >= K) {
            lo = mid;
            c = m;
        } else {
            hi = mid;
        }
        mid = lo + (hi - lo) / 2;
    }
    collect<T, NT>(row, V, c <= kCap ? lo : hi, sh);
    const int have = sh.n;
    __syncthreads();
    return c <= kCap ? have : append_equal<T, NT>(row, V, K, lo, have, sh);
}

constexpr int kScanThreads = 256;
constexpr int kSample = 4;        // vectors a thread in the sample
constexpr int kKeep = 252;        // vectors that a wave keeps: 8 workgroups fill a CU's LDS
constexpr int kScanWaves = kScanThreads / kWave;
constexpr int kScanWant = 2048;   // workgroups that fill the chip
constexpr int kMinScan = 2048;    // elements of a part
// Parts of rows that the workspace holds at once, at 20 KB each (83 MB).  Larger calls take a pair of
// launches for each slab: 16384 rows of 8000 bfloat16 165 us, and 142 by 8192, 131 by 16384 parts; the
// workspace is what bounds it, and up to 4096 rows it makes no difference.
constexpr int64_t kSlab = 4096;

struct TopPlan {
    int parts;
    int64_t rows;     // of a slab
    float* least;     // [rows]
    float4* sums;     // [rows][parts]: maximum and sum of the softmax, largest logit
    int32_t* count;   // [rows][parts][kScanWaves]: vectors that reach the threshold
    int32_t* at;      // [rows][parts][kScanWaves][kKeep]: their numbers
    Vec4* kept;       // [rows][parts][kScanWaves][kKeep]: and what they hold
    size_t bytes;
};
TopPlan top_plan(int64_t rows, int64_t V, void* ws) {
    TopPlan p;
    int64_t parts = (kScanWant + rows - 1) / rows;
    const int64_t most = (V + kMinScan - 1) / kMinScan;
    if (parts > most) parts = most;
    if (parts > kTopThreads / kScanWaves) parts = kTopThreads / kScanWaves;
    p.parts = parts < 1 ? 1 : (int)parts;
    p.rows = rows < kSlab / p.parts ? rows : kSlab / p.parts;
    size_t off = 0;
    auto take = [&](size_t bytes) {
        char* at = (char*)ws + off;
        off += (bytes + 255) / 256 * 256;
        return at;
    };
    const size_t n = (size_t)p.rows * p.parts;
    p.least = (float*)take((size_t)p.rows * sizeof(float));
    p.sums = (float4*)take(n * sizeof(float4));
    p.count = (int32_t*)take(n * kScanWaves * sizeof(int32_t));
    p.at = (int32_t*)take(n * kScanWaves * kKeep * sizeof(int32_t));
    p.kept = (Vec4*)take(n * kScanWaves * kKeep * sizeof(Vec4));
    p.bytes = off;
    return p;
}

struct ScanShared {
    union {
        uint32_t key[kScanThreads * kSample];   // the sample's
        Vec4 kept[kScanWaves][kKeep];
    };
    int at[kScanWaves][kKeep];
    float2 red[kScanWaves];
    float least;
};

// The threshold guessed from the largest logits of a sample's vectors, by one wave
__device__ uint32_t guess(const uint32_t* keys, int K, float sampled) {
    constexpr int J = kScanThreads * kSample / kWave;
    uint32_t key[J], high = 0;
#pragma unroll
    for (int j = 0; j < J; ++j) {
        key[j] = keys[j * kWave + threadIdx.x];
        high = max(high, key[j]);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) high = max(high, __shfl_xor(high, o, kWave));
    const float part = K * fminf(sampled, 1.f);
    const float rank = fminf(K * 1.25f + 8.f, 1.5f * part + 4.f * sqrtf(part) + 4.f);
    // `rank` logits lie in about this many different ones of so many groups
    auto reach = [&](float groups) { return max(1, (int)(groups * (1.f - exp_(-rank / groups)))); };
    const uint32_t low = key_of(-FLT_MAX), top = __builtin_amdgcn_readfirstlane(high) + 1;
    int c;
    if (rank > 100.f) return threshold<kWave, J>(key, reach(J * kWave), low, top, &c);
    // (a step of the search takes the time of its keys)
    uint32_t of4[J / 4];
#pragma unroll
    for (int j = 0; j < J / 4; ++j)
        of4[j] = max(max(key[j], key[j + J / 4]), max(key[j + J / 2], key[j + J / 4 * 3]));
    return threshold<kWave, J / 4>(of4, reach(J / 4 * kWave), low, top, &c);
}

// One workgroup a part of a row: sums of its softmax, and the vectors that reach the threshold.
// They are kept in LDS until the end: the loads' waits would count their stores to memory.
template <class T>
__global__ __launch_bounds__(kScanThreads, 8) void k_top_scan(TopArgs a, TopPlan p, uint32_t first,
                                                              uint32_t rows) {
    __shared__ ScanShared sh;
    constexpr int NT = kScanThreads, W = kVec<T>;
    const uint32_t i = blockIdx.x / (uint32_t)p.parts, part = blockIdx.x % (uint32_t)p.parts;
    if (i >= rows) return;
    const uint32_t row = first + i, b = row / (uint32_t)a.N, n = row % (uint32_t)a.N;
    if (n >= clamp_rows(a.lengths, b, a.N)) return;
    const T* x = row_of<T>(a.logits, b, n);
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave, nv = a.V / W;
    {
        // a 16th of the row at least, an 8th where the list would be long: units of 64 vectors
        constexpr int kRound = kScanWaves * kSample, kOnce = NT * kSample * W;
        const int units = (nv + kWave - 1) / kWave;
        const int rounds = (a.V * (a.K > 128 ? 2 : 1) + 16 * kOnce - 1) / (16 * kOnce);
        float top[kSample];
        for (int q = 0; q < rounds; ++q) {
            Raw<T> r[kSample];
            bool there[kSample];
#pragma unroll
            for (int j = 0; j < kSample; ++j) {
                // (rows of no more units than the sample has are taken whole)
                const int at = (wave * kSample + j) * rounds + q;
                const int u = units <= kRound ? at : at * units / (kRound * rounds);
                r[j] = load_raw<T, false>(x + (size_t)min(u * kWave + lane, nv - 1) * W);
                there[j] = u * kWave + lane < nv;
            }
#pragma unroll
            for (int j = 0; j < kSample; ++j) {
                float v[W];
                unpack<T>(r[j], v);
                const float t = there[j] ? max_of(v) : -INFINITY;
                top[j] = q ? fmaxf(top[j], t) : t;
            }
        }
#pragma unroll
        for (int j = 0; j < kSample; ++j) sh.key[j * NT + tid] = key_of(top[j]);
        __syncthreads();
        if (tid < kWave) {
            const uint32_t lo = guess(sh.key, a.K, (float)(rounds * kOnce) / (float)a.V);
            if (tid == 0) {
                sh.least = of_key(lo);
                if (part == 0) p.least[i] = sh.least;
            }
        }
        __syncthreads();
    }
    const int per = ((nv + p.parts - 1) / p.parts + 7) / 8 * 8;   // whole cache lines
    const int lo = min((int)part * per, nv), hi = min(lo + per, nv);
    const float c = a.scale.c, least = sh.least;
    ChunkSoft soft;
    soft.init(a.scale);
    float most = -INFINITY;
    int found = 0;   // of this wave
    auto keep = [&](bool reaches, const Raw<T>& r, int v) {
        const uint64_t votes = __ballot(reaches);
        const int k = found + __builtin_amdgcn_mbcnt_hi((uint32_t)(votes >> 32),
                                                        __builtin_amdgcn_mbcnt_lo((uint32_t)votes, 0));
        if (reaches && k < kKeep) {
            sh.kept[wave][k] = {r.w[0], r.w[1], r.w[2], r.w[3]};
            sh.at[wave][k] = v;
        }
        found += __popcll(votes);
    };
    auto work = [&](const Raw<T> (&r)[2], int v0, int v1) {
        float v[2][W], top[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            unpack<T>(r[u], v[u]);
            top[u] = max_of(v[u]);
        }
        const float t = fmaxf(top[0], top[1]);
        most = fmaxf(most, t);
        soft.raise(t, c);
#pragma unroll
        for (int u = 0; u < 2; ++u) soft.push(v[u], c);
        if (__any(t >= least)) {
            keep(top[0] >= least, r[0], v0);
            keep(top[1] >= least, r[1], v1);
        }
    };
    const char* base = (const char*)x;
    auto load = [&](int v) { return load_raw<T, true>((const T*)(base + (uint32_t)v * 16u)); };
    // the loops go by the wave's first lane, so that all its lanes count the same vectors
    int v = __builtin_amdgcn_readfirstlane(lo + wave * kWave);
    for (; v + 3 * NT + kWave <= hi; v += 4 * NT) {
        const int i = v + lane;
        Raw<T> r[2], s[2];
        r[0] = load(i), r[1] = load(i + NT), s[0] = load(i + 2 * NT), s[1] = load(i + 3 * NT);
        work(r, i, i + NT);
        work(s, i + 2 * NT, i + 3 * NT);
    }
    for (; v < hi; v += NT) {
        const int i = v + lane;
        const Raw<T> r = load(min(i, hi - 1));
        float one[W];
        unpack<T>(r, one);
        const float t = i < hi ? max_of(one) : -INFINITY;
        most = fmaxf(most, t);
        soft.raise(t, c);
        if (i < hi) soft.push(one, c);
        keep(t >= least, r, i);
    }
    const int e = nv * W + tid;   // the row's last few logits; k_top_pick looks at all of them
    if (part == 0 && e < a.V) {
        float one[1] = {to_f(x[e])};
        most = fmaxf(most, one[0]);
        soft.raise(one[0], c);
        soft.push(one, c);
    }
    const Soft all = block_soft<NT>(soft.value(c), c, sh.red);
    most = block_max<NT>(most, (float*)sh.red);
    if (tid == 0) {
        p.sums[blockIdx.x] = make_float4(all.m, all.s, most, 0.f);
    }
    const size_t q = (size_t)blockIdx.x * kScanWaves + wave;
    if (lane == 0) p.count[q] = found;
    for (int k = lane; k < min(found, kKeep); k += kWave) {
        p.kept[q * kKeep + k] = sh.kept[wave][k];
        p.at[q * kKeep + k] = sh.at[wave][k];
    }
}

// A threshold that at least K of the row's logits reach, from the maxima of groups of them
template <class T, int NT>
__device__ uint32_t group_threshold(const T* row, int V, int K, TopShared& sh) {
    constexpr int kU = 4;
    float group[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u) group[u] = -INFINITY;
    int turn = 0;
    walk_row<T, NT, 1>(row, 0, V, threadIdx.x, [&](const float (&v)[kVec<T>], int, int) {
        const float t = max_of(v);
#pragma unroll
        for (int u = 0; u < kU; ++u)
            if ((turn & (kU - 1)) == u) group[u] = fmaxf(group[u], t);
        ++turn;
    });
    uint32_t key[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u) key[u] = key_of(group[u]);
    int c;
    return threshold<NT, kU>(key, K, key_of(-FLT_MAX), key_of(INFINITY) + 1, &c, &sh);
}

// One workgroup a row: the list from the kept vectors
template <class T>
__global__ __launch_bounds__(kTopThreads) void k_top_pick(TopArgs a, TopPlan p, uint32_t first,
                                                          uint32_t rows) {
    __shared__ TopShared sh;
    constexpr int NT = kTopThreads, W = kVec<T>, J = kCap / NT;
    const int tid = threadIdx.x, K = a.K, V = a.V;
    const uint32_t i = blockIdx.x;
    if (i >= rows) return;
    const uint32_t row = first + i, b = row / (uint32_t)a.N, n = row % (uint32_t)a.N;
    if (n >= clamp_rows(a.lengths, b, a.N)) {
        write_padding<T, NT>(a, row);
        return;
    }
    const T* x = row_of<T>(a.logits, b, n);
    const float c = a.scale.c, least = p.least[i];
    if (tid == 0) sh.n = 0;
    __syncthreads();
    auto append = [&](float v, int at) {
        const int k = atomicAdd(&sh.n, 1);
        if (k < kCap) sh.list[k] = word_of(key_of(v), at);
    };
    bool lost = false;
    Soft soft = soft_empty();
    float most;
    {
        const int lane = tid % kWave;
        const float4 s = lane < p.parts ? p.sums[(size_t)i * p.parts + lane]
                                        : make_float4(-FLT_MAX, 0.f, -INFINITY, 0.f);
        soft = wave_soft({s.x, s.y}, c);
        most = wave_max_fast(s.z);
    }
    // the scan's waves' vectors, `each` threads to a wave's
    const int lists = p.parts * kScanWaves, each = NT / lists;
    if (tid < lists * each) {
        const size_t q = (size_t)i * lists + tid / each;
        const int count = p.count[q];
        lost = count > kKeep;
        for (int k = tid % each; k < min(count, kKeep); k += each) {
            const Vec4 w = p.kept[q * kKeep + k];
            const int at = p.at[q * kKeep + k] * W;
            float v[W];
            unpack<T>({{w.x, w.y, w.z, w.w}}, v);
#pragma unroll
            for (int e = 0; e < W; ++e)
                if (v[e] >= least) append(v[e], at + e);
        }
    }
    const int e = V / W * W + tid;   // the row's last few logits
    if (e < V && to_f(x[e]) >= least) append(to_f(x[e]), e);
    if (a.lse) {
        if (far(most, a.scale)) {
            soft = soft_empty();
            walk_row<T, NT, 1>(x, 0, V, tid,
                               [&](const float (&v)[W], int, int) { soft_push(soft, v, c); });
            soft = block_soft<NT>(soft, c, sh.red);
        }
        if (tid == 0) a.lse[row] = soft_lse(soft, a.scale.inv_t);
    }
    lost = __syncthreads_or(lost);
    int have = sh.n;
    __syncthreads();
    if (lost || have > kCap || (have < K && least > -FLT_MAX)) {
        have = select_again<T, NT>(x, V, K, group_threshold<T, NT>(x, V, K, sh), sh);
    } else if (have > K + K / 4 + 32) {
        // counting takes the square of the list's length: what the K-th is above leaves it
        uint64_t w[J];
        uint32_t key[J];
#pragma unroll
        for (int j = 0; j < J; ++j) {
            w[j] = j * NT + tid < have ? sh.list[j * NT + tid] : 0;
            key[j] = (uint32_t)(w[j] >> 32);
        }
        int reach;
        const uint32_t lo = threshold<NT, J>(key, K, key_of(least), key_of(INFINITY) + 1, &reach, &sh);
        if (tid == 0) sh.n = 0;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < J; ++j)
            if (key[j] >= lo) sh.list[atomicAdd(&sh.n, 1)] = w[j];
        __syncthreads();
        have = sh.n;
    }
    // -inf is none of the K largest before every finite logit is
    if (have < K) have = append_equal<T, NT>(x, V, K, key_of(-INFINITY), have, sh);
    __syncthreads();
    write_places<T, NT>(a, x, row, have, sh);
}

}  // namespace

size_t top_workspace(int64_t B, int64_t N, int64_t V, int64_t) {
    return V <= kShort ? 0 : top_plan(B * N, V, nullptr).bytes;
}

hipError_t launch_top(const TopArgs& a, hipStream_t s) {
    hipError_t e = hipSuccess;
    with_type(a.dtype, [&](auto t) {
        using T = decltype(t);
        const int64_t rows = a.B * a.N;
        const unsigned grid = row_grid(rows, kWave);
        if (a.V <= 64)
            k_top_short<T, 1><<<grid, kWave, 0, s>>>(a);
        else if (a.V <= 256)
            k_top_short<T, 4><<<grid, kWave, 0, s>>>(a);
        else if (a.V <= kShort)
            k_top_short<T, 16><<<grid, kWave, 0, s>>>(a);
        else {
            const TopPlan p = top_plan(rows, a.V, a.ws);
            for (int64_t first = 0; first < rows && e == hipSuccess; first += p.rows) {
                const uint32_t n = (uint32_t)(rows - first < p.rows ? rows - first : p.rows);
                const uint32_t at = (uint32_t)first;
                k_top_scan<T><<<n * p.parts, kScanThreads, 0, s>>>(a, p, at, n);
                k_top_pick<T><<<n, kTopThreads, 0, s>>>(a, p, at, n);
                e = hipGetLastError();
            }
        }
    });
    return e == hipSuccess ? hipGetLastError() : e;
}

}  // namespace tsc
