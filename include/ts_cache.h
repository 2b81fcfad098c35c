/*
 * ts_cache.h -- C ABI of the calls on a larger model's paged cache of keys and values
 * (libtschain.so, MI355X / gfx950): what its pass over drafted tokens needs, before
 * ts_token_verify answers them.
 *   - new keys and values into the cache, keys and queries rotated by their positions on the way;
 *   - attention of drafted tokens, a tree or a path of them, over the cache.
 * Status codes, errors, ownership, streams and reproducibility are those of ts_chain.h: every
 * pointer is a device pointer owned by the caller, nothing is allocated, work is enqueued on
 * `stream`, and results are bitwise the same for the same inputs.
 *
 * Common arguments
 *   dtype    TS_BFLOAT16 or TS_FLOAT16, of all tensors of a call but those said to be float32.
 *   D        elements of a head: a multiple of 8 in [8, ts_cache_max_head()].
 *   Hq, Hk   heads of queries, and of keys and values: Hq a multiple of Hk, Hq <= 1024.  Query head h
 *            reads key head h / (Hq / Hk).
 *   k_cache, v_cache  [P, S, Hk, D]: P pages of S tokens, elements from a page, a token, a head
 *            to the next (ts_cache_layout: the same of both), those of a head contiguous.  Heads
 *            start at multiples of 16 bytes.
 *   pages    int32 [B, M]: the pages of each sequence; its token at slot j lies in page
 *            pages[b, j / S] at j % S.  A page outside [0, P) is not there: nothing is written to it, and
 *            its keys and values are read as zeros.  M * S <= 2^30.
 *   starts   int32 [B]: tokens of each sequence that the cache holds before the new ones, clamped
 *            to [0, M * S] on the device.  New token n lies at slot starts[b] + n; slots from M * S
 *            on do not exist: they are not written and not seen.
 *   lengths  int32 [B]: new tokens of each sequence, 0 <= lengths[b] <= N, or NULL (every length is
 *            N); clamped on the device.  Tokens from there on are padding and are never read.
 *   B, N     B >= 1, N >= 1, B * N * Hq <= 2^29.
 * With TS_CHECK=1 in the environment a call copies lengths, starts, pages and parents to the host and
 * returns TS_ERR_LENGTHS for a length or a start out of range (the last new slot included), and
 * TS_ERR_LABELS for a page that is needed and not there, and for a parent out of range.
 */
#ifndef TS_CACHE_H
#define TS_CACHE_H

#include "ts_token.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Largest D, and the most drafted tokens of a sequence. */
int ts_cache_max_head(void);
int ts_cache_max_nodes(void);

/* A paged cache: sizes, and strides in elements (each a multiple of 8). */
typedef struct ts_cache_layout {
    int64_t pages, page_size, heads, head_size;
    int64_t stride_page, stride_token, stride_head;
} ts_cache_layout;

/*
 * Appends keys and values, rotating keys (and queries) by their positions.
 *   k, v     [B, N, Hk, D], elements from a sequence, a token, a head to the next in strides[0..2] and
 *            strides[3..5]; q [B, N, Hq, D] in strides[6..8], or NULL.  All strides are multiples of 8
 *            and >= 0, and all heads start at multiples of 16 bytes.
 *   freqs    float32 [R / 2] or NULL (R = 0: nothing is rotated): what a position's angles are per
 *            position.  With angle a = position * freqs[i], formed in 64 bits, a pair (x, y) becomes
 *            (x cos a - y sin a, y cos a + x sin a), rounded once.
 *   R        rotated elements of a head, the first ones: a multiple of 16, at most D.
 *   neighbours  0: pair i is (i, i + R / 2); 1: it is (2 i, 2 i + 1).
 *   positions  int32 [B, N] or NULL: the position of each new token (a draft's depth in its tree counts,
 *            not its slot); NULL: its slot.
 *   q_out    [B, N, Hq, D], contiguous (may be q itself where q is); zeros for padding.
 * k, v and q do not overlap the caches, and no slot is written twice in a call (it would hold what one of
 * the two writes).
 */
ts_status ts_cache_append(const void* k, const void* v, const void* q, const int64_t strides[9],
                          int dtype, const float* freqs, int64_t R, int neighbours,
                          const int32_t* positions, void* k_cache, void* v_cache,
                          const ts_cache_layout* layout, const int32_t* pages, int64_t M,
                          const int32_t* starts, const int32_t* lengths, int64_t B, int64_t N,
                          int64_t Hq, void* q_out, void* stream);

/* Workspace bytes of ts_cache_attend; 0 for invalid arguments. */
size_t ts_cache_attend_workspace_bytes(int64_t B, int64_t N, int64_t Hq, int64_t Hk, int64_t D);

/*
 * Attention of drafted tokens over the cache that holds them and what was before.
 *   q        [B, N, Hq, D], elements from a sequence, a token, a head to the next in strides[0..2].
 *   parents  int32 [B, N] or NULL: the draft that draft i continues, below i; -1 (or anything outside
 *            [0, i)): it continues the text before the drafts.  NULL: a path, parents[i] = i - 1.
 *   N        at most ts_cache_max_nodes().  With up to 256 sequences B * ceil(N * Hq / (64 * Hk)) * M * S up to
 *            2^35 always fits; what the kernels' numbers do not hold is refused (TS_ERR_BAD_DIM).
 *   scale    in [1e-6, 1e6]: out_i = sum_j p_j v_j, p = softmax(scale * q_i . k_j) over the slots j
 *            before starts[b], the drafts that i follows, and i itself.
 *   out      [B, N, Hq, D], contiguous, not overlapping q; lse float32 [B, N, Hq] or NULL: log sum_j exp(scale q_i . k_j).
 *            Where no slot is seen out is 0 and lse -inf, and so they are for padding.
 *   ws       device workspace of at least ts_cache_attend_workspace_bytes(...), aligned to 256
 *            bytes.  Its contents on entry are ignored.
 * Queries, keys and values of slots before starts[b] + lengths[b] are finite, products q . k within 1e30
 * in size and values within 1e27 (sums of up to 2^30 of them, with numerators of up to 2^8, stay 32-bit
 * floats); what lies behind these slots is never used.
 */
ts_status ts_cache_attend(const void* q, const int64_t strides[3], int dtype, const void* k_cache,
                          const void* v_cache, const ts_cache_layout* layout,
                          const int32_t* pages, int64_t M, const int32_t* starts,
                          const int32_t* parents, const int32_t* lengths, int64_t B, int64_t N,
                          int64_t Hq, float scale, void* out, float* lse, void* ws,
                          size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* TS_CACHE_H */
