/*
 * A paged key / value cache held in 8 bits, for NVIDIA B200 (sm_100a): appending to it, attention over it, and
 * eviction from it by the attention weight its tokens received (csrc/kv8_append.cu, kv8_attend.cu, kv8_evict.cu).
 *
 * A value is stored as e4m3 (4 exponent, 3 mantissa bits) and stands for stored * 2^e, one e for each page, kind
 * (keys, values) and key head.  e is the smallest one in [-32, 31] with amax <= 448 * 2^e, amax being the largest
 * finite or infinite magnitude among the page's tokens (NaN do not count and stay NaN; what exceeds 448 * 2^e is cut to
 * that).  As the scales are powers of two, moving a stored value to a larger one is exact unless it becomes subnormal.
 *
 *   pool   uint8 [pages][2][n_kv][block][head_dim]: keys, then values (16-byte aligned)
 *   exps   int8  [pages][2][n_kv]
 *   block_table  int32 [B][max_blocks]: row b's page for its tokens block * i .. is block_table[b][i]
 *   ctx    int32 [B]: cached tokens of every row; 0 = padding row
 * Rows of one call do not share pages that the call writes.  A token whose page lies outside the pool is not written;
 * in attention it stands for zeros.  A row's results depend on that row alone: not on the other rows of the call and
 * not on where its pages lie.
 * Data pointers are DEVICE pointers of the current device; calls are asynchronous on the given stream, allocate nothing
 * and may be captured into a graph.  Status codes are those of corun.h.
 */
#ifndef CORUN_KV8_H
#define CORUN_KV8_H

#include <stdint.h>

#include "corun.h"
#include "corun_rope.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
  void *pool;
  int8_t *exps;
  int64_t pages;                 /* pages * 2 * n_kv * block < 2^31                     */
  int32_t block, n_kv, head_dim; /* block 16, 32 or 64; n_kv >= 1; head_dim 64 or 128   */
} corun_kv8_cache;

typedef struct {
  const int32_t *block_table;
  int32_t max_blocks;   /* max_blocks * block < 2^30                                            */
  const int32_t *ctx;   /* cached tokens of every row, the call's own tokens among them         */
  const int32_t *cu;    /* int32 [B + 1]: row b's tokens of this call are cu[b] .. cu[b + 1] - 1, its last ones in
                           the cache; NULL: one token per row, token b being row b's             */
  int32_t B;            /* 1..65535                                                             */
  int32_t T;            /* tokens there is room for (cu[B] <= T; NULL cu: B); 0: a call that reads and writes nothing,
                           whose data pointers may be NULL                                      */
} corun_kv8_rows;

/*
 * Appends the rows' new tokens: k, v [T, n_kv, head_dim] and, where q is given, q [T, n_q, head_dim] -> q_out, all of
 * type dtype.  With `rope` keys and queries are rotated on the way at positions[t] (int32 [T]; not the place in the
 * cache, which eviction changes), rot_dim <= head_dim; keys enter the cache from 32 bits, q_out is rounded to dtype
 * (q_out may be q).  A page that held tokens of its row before keeps max(its e, that of the new tokens), and its old
 * values move to it.  mass (float [B][n_kv][max_blocks * block] or NULL): the new tokens' entries become 0.
 * A row with ctx 0, with more new tokens than ctx, with ctx beyond its table or with tokens outside [0, T) is left out;
 * tokens of no row keep q_out as it was.  Errors: EINVAL, ECUDA.
 */
int corun_kv8_append(const corun_kv8_cache *cache, const corun_kv8_rows *rows, const corun_heads *k, const corun_heads *v,
                     int32_t dtype, const corun_rope *rope, const int32_t *positions, const corun_heads *q,
                     const corun_heads *q_out, int32_t n_q, float *mass, void *cuda_stream);

/*
 * out[t, h] = sum_j p_j v_j,  p = softmax_j(scale q[t, h] . k_j) over the cached tokens j of t's row with j <= i and, where
 * window > 0, j > i - window, i = ctx - (the row's new tokens) + (t's place among them) being t's own place; query head
 * h reads key head h / (n_q / n_kv).  A query that sees no token (i < 0) yields zeros; rows with ctx 0 or beyond
 * their table and tokens of no row keep `out` as it was.  What pages hold behind a row's last token is not read as numbers (it may be NaN).
 * mass (float [B][n_kv][max_blocks * block] or NULL): mass[b][g][j] += sum of p_j over the row's queries and the heads of g;
 * with mass, max_new * n_q / n_kv <= 32.
 *   dtype     of q and out: CORUN_BF16 or CORUN_F16; heads start on 16 bytes
 *   max_new   largest number of new tokens of a row (cu NULL: 1); a row with more is left out
 *   ws        corun_kv8_attend_bytes(...) bytes, 256-byte aligned, the call's own until it has run
 * A NaN among the values of a token reaches every query that sees the token, and may reach other queries of the same row and call.
 * n_q a multiple of n_kv, n_q / n_kv <= 32, B <= 512, scale > 0, T / (128 / (n_q / n_kv)) + B at most some 65000 (EINVAL beyond).  Queries and softmax weights enter the tensor cores as
 * sums of e4m3 values that hold 11 or more bits of them, but for what is below 2^-25 of the largest value of the query, or weight among 128
 * neighbouring tokens; scores, weights' sums and outputs are held in 32 bits
 * (scores beyond 2^20 in magnitude so lose bits of their differences, and mass of its weights; outputs stay means of the values).
 * A row with more than 32 columns (new tokens * n_q / n_kv) is not split over its cached tokens: one SM takes each of its tiles of 128
 * columns and key head through all of them.  That is for chunks of prompts; a few tokens more than 32 columns hold behind a very long cache
 * (100003 tokens, 8 heads a key head: 4 tokens 78 us, 5 tokens 2080) are faster in two calls.
 * Errors: EINVAL, ECUDA.  A bounded device-side wait that expires is recorded in the first 1024 bytes of ws: corun_kv8_sync waits for
 * the stream and returns ETIMEOUT in that case.  With T 0 corun_kv8_attend_bytes is 0 and ws may be NULL; where it has 1024 bytes or more,
 * those are cleared.  corun_kv8_sync is for a ws that has them.
 */
int64_t corun_kv8_attend_bytes(int32_t B, int32_t T, int32_t max_new, int32_t n_q, int32_t n_kv, int32_t head_dim, int32_t block,
                               int32_t max_blocks, int32_t with_mass);
int corun_kv8_attend(const corun_kv8_cache *cache, const corun_kv8_rows *rows, int32_t max_new, const corun_heads *q,
                     const corun_heads *out, int32_t dtype, int32_t n_q, float scale, int32_t window, float *mass, void *ws,
                     int64_t ws_bytes, void *cuda_stream);
int corun_kv8_sync(const void *ws, void *cuda_stream);

/*
 * Shortens every row b with 0 < keep'[b] < ctx[b] to keep'[b] tokens, keep' = keep[b] but at least sinks + recent and at most
 * max_keep (keep[b] <= 0: the row stays).  For every key head on its own stay the first `sinks` tokens, the last `recent` and, of the others, those
 * with the largest mass (ties: the lowest index; NaN counts as the smallest), in their order, moved to the front of the
 * row's pages; a block's e becomes the largest e that its tokens had.  mass moves along.  The pages behind the new end
 * are the caller's to free; mass behind it is left as it was.
 *   new_ctx   int32 [B]: the rows' tokens afterwards (may be ctx itself)
 *   kept      int32 [B][n_kv][max_keep]: the former places of the tokens that stayed, ascending, then -1; all -1 for a
 *             row that stays as it is
 *   ws        corun_kv8_evict_bytes(...) bytes, 256-byte aligned, the call's own until it has run
 * A row with ctx beyond its table or with a page outside the pool stays as it is.
 * sinks, recent >= 0, sinks + recent <= max_keep, 1 <= max_keep <= max_blocks * block, max_blocks <= 65536.  Errors: EINVAL, ECUDA.
 */
int64_t corun_kv8_evict_bytes(int32_t B, int32_t n_kv, int32_t max_keep);
int corun_kv8_evict(const corun_kv8_cache *cache, const int32_t *block_table, int32_t max_blocks, int32_t B, const int32_t *ctx,
                    int32_t *new_ctx, float *mass, const int32_t *keep, int32_t max_keep, int32_t sinks, int32_t recent,
                    int32_t *kept, void *ws, int64_t ws_bytes, void *cuda_stream);

#ifdef __cplusplus
}
#endif
#endif
