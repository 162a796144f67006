/*
 * harts_rollout.h -- C ABI of libharts for generation: a paged key/value cache,
 * attention of new rows over a forest of cached segments, and the recurrent
 * steps of the linear layers.  The calls follow the conventions of harts.h
 * (return values and messages, validation before anything is enqueued, the
 * caller's stream and buffers, no allocation on the device).
 */
#ifndef HARTS_ROLLOUT_H_
#define HARTS_ROLLOUT_H_

#include "harts.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { HARTS_E4M3 = 2 }; /* 8-bit cache storage, beside HARTS_BF16 */

/* ------------------------------------------------------------------------
 * Generation over a forest of cached segments: what one generated token (or a
 * few drafted ones, or the rows of a prompt) needs in the layers above.
 *
 * harts_cache -- a paged key/value cache, described to the calls below by
 * device pointers.  A segment is a run of consecutive rows of one branch of
 * the forest; its row p lies in slot p % 64 of page pages[seg][p / 64].
 *   k, v       [n_pages][H][64][d]: bf16 (kind HARTS_BF16) or e4m3 codes
 *              (HARTS_E4M3).  16-byte aligned.
 *   k_exp, v_exp  [n_pages][H][64] biased scale exponents of e4m3 rows: a
 *              stored code y with exponent b in [1, 254] stands for
 *              y * 2^(b - 127), for an infinity past what bf16 holds.
 *              4-byte aligned; NULL for bf16.
 *   pages      [n_seg][pitch] int32 page of every 64 rows, -1 for none.
 *   len        [n_seg] int32 rows of every segment, new rows included.
 * Lengths beyond pitch * 64 hold no further rows, and rows on a page outside
 * [0, n_pages) do not exist: they are neither read nor written.
 * d in {64, 128}; 1 <= H <= 65535.
 *
 * Row tables: int32 [n][2] of (segment, position); a negative position counts
 * from the segment's end (-1 its last row), so that a table stays valid while
 * the lengths grow.  An entry that names no existing row is skipped by a
 * write and read as zeros.
 *
 * harts_cache_write -- rows k_new, v_new [n][H][d] bf16 into the cache, as
 *   given or, for e4m3, each (row, head) with the smallest scale 2^e
 *   (e >= -126) that brings its largest finite magnitude to 448 or less,
 *   every x * 2^-e rounded once to nearest even (infinities and NaN are
 *   stored as NaN; where the nearest code stands for 2^128, which bf16 does
 *   not hold, from 248 * 2^120, the one below, 240 * 2^120, is taken).  A call
 *   may name a row only once; k_new, v_new and rows lie outside the cache,
 *   whose parts lie apart.
 * harts_cache_read -- k_out, v_out [n][H][d] bf16: the values that the rows
 *   stand for, exact (an e4m3 code has 4 significant bits).  They overlap
 *   no other argument.
 * ---------------------------------------------------------------------- */
typedef struct harts_cache {
  void *k, *v;
  uint8_t *k_exp, *v_exp;
  const int32_t* pages;
  const int32_t* len;
  int32_t n_pages, n_seg, pitch, H, d, kind;
} harts_cache;

int harts_cache_write(const harts_cache* cache, const int32_t* rows, int64_t n, const void* k_new,
                      const void* v_new, void* stream);

int harts_cache_read(const harts_cache* cache, const int32_t* rows, int64_t n, void* k_out, void* v_out,
                     void* stream);

/* ------------------------------------------------------------------------
 * harts_gen_attn -- attention of new rows over the forest.  Segment s has
 * n_new[s] query rows, its last rows; each sees every row of the segment's
 * ancestors and the segment's own rows up to itself:
 *     o = softmax(scale q K^T) V over the visible rows,  lse = its log-sum.
 * Every segment is read once for all query rows below it, so a prefix that
 * sequences share is read once, at any depth of sharing.
 *
 * harts_gen_layout / harts_gen_tables (host) -- sizes, then tables.
 *   parent   [n_seg] parent segment or -1, any order; n_new [n_seg] >= 0.
 *   cap      [n_seg] about how many rows the segment holds while the tables
 *            are in use: how finely they are split, by their shares of the
 *            whole.  Results differ by rounding only, but room that stays empty
 *            takes splits from the segments that all rows wait for.
 *   Hq, Hkv  query and key heads; Hq a multiple of Hkv, query head h reads
 *            key head h / (Hq / Hkv).
 *   rows     [n_rows][2] out: the row table of the query rows (for
 *            harts_cache_write): segments by ascending id, each one's new
 *            rows in order.  q, o and lse are in this order.
 *   order    [n_rows] out: the query rows in depth-first order (children by
 *            ascending id), in which the rows below a segment are contiguous.
 *   items    [n_items][12] out: work items (segment, first place in order,
 *            first stacked row, stacked rows, split, splits, new rows of the
 *            segment, part of a row's first part, 16-row tiles of a wave,
 *            waves along rows, multiplier and shift that divide by splits); a
 *            stacked row is one of the Hq/Hkv query heads of one query row.
 *   part_off [n_rows + 1] out: partial results of every row (in q's order).
 *   Errors: HARTS_EINVAL (NULL, sizes, a parent out of range or a cycle),
 *   HARTS_EUNSUPPORTED (table sizes beyond int32), HARTS_ENOMEM.
 *
 * harts_gen_attn (device) -- q, o [n_rows][Hq][d] bf16; lse [n_rows][Hq]
 *   float32 or NULL; sizes, items, order, part_off from the tables; ws of
 *   harts_gen_workspace_size bytes.  A row that sees no key, or only keys of
 *   score -infinity, gets zeros and lse = -infinity; a key that a row does
 *   not see has no influence on it, whatever its values.  Weights are summed
 *   up to 2^8 times too large before they are normalised: values that 2^8 and
 *   the number of keys bring past float32 may give infinities.  Deterministic.
 * All: HARTS_EINVAL (NULL, misaligned, small workspace), HARTS_EUNSUPPORTED
 * (d, heads, kind), HARTS_EHIP.  Device calls are asynchronous and can be
 * captured; o, lse and ws overlap no other argument.
 * ---------------------------------------------------------------------- */
typedef struct harts_gen_sizes {
  int64_t n_rows, n_items, n_parts, n_join; /* n_join: rows of several parts */
} harts_gen_sizes;

int harts_gen_layout(int32_t n_seg, const int32_t* parent, const int32_t* n_new, const int64_t* cap, int32_t Hq,
                     int32_t Hkv, harts_gen_sizes* out);

int harts_gen_tables(int32_t n_seg, const int32_t* parent, const int32_t* n_new, const int64_t* cap, int32_t Hq,
                     int32_t Hkv, int32_t* rows, int32_t* order, int32_t* items, int32_t* part_off);

int harts_gen_workspace_size(const harts_gen_sizes* sizes, int32_t Hq, int32_t d, size_t* bytes);

int harts_gen_attn(const harts_cache* cache, const harts_gen_sizes* sizes, const int32_t* items, const int32_t* order,
                   const int32_t* part_off, int32_t Hq, float scale, const void* q, void* o, float* lse, void* ws,
                   size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------------
 * Recurrent steps of the linear layers, states kept in pools.  Sequence i
 * takes rows [row_off[i], row_off[i + 1]) one after the other (row_off NULL:
 * row i alone), starting from state idx_in[i] of S_in and leaving its last
 * state in entry idx_out[i] of S_out:
 *   harts_la_step   S_t = e^{g_t} S_{t-1} + k_t v_t^T,  o_t = scale S_t^T q_t;
 *   harts_kda_step  D = Diag(e^{g_t}) S_{t-1},
 *                   S_t = D + beta_t k_t (v_t - D^T k_t)^T, o_t the same.
 *   q, k, v, o  [n_rows][H][d] (dtype); g float32 [n_rows][H] (la) or
 *               [n_rows][H][d] (kda); beta float32 [n_rows][H].  16-byte
 *               aligned, as the states are; la's g and beta 4-byte aligned.
 *   S_in        float32 [n_in][H][d][d]; idx_in int32 [n_seq] or NULL (entry
 *               i).  Several sequences may start from one entry.  An index
 *               outside [0, n_in) starts from zeros.
 *   S_out       float32 [n_out][H][d][d]; idx_out likewise; outside
 *               [0, n_out) the last state is not kept.  Where an index of
 *               idx_out repeats an earlier one, that sequence writes no
 *               state and its outputs are NaN (found by reading the earlier
 *               ones: free up to thousands of sequences, quadratic beyond).
 *   S_out may be S_in itself if idx_out is idx_in and n_out = n_in, for an
 *   update in place; otherwise the two must not overlap.
 * Rows behind the last sequence, entries that no index names and outputs of
 * sequences without rows stay as they are; a sequence without rows hands its
 * state on.  dtype HARTS_BF16 or HARTS_F32, d in {64, 128}.  Row offsets are
 * clamped to [0, n_rows] and must not decrease.  o and S_out overlap no other
 * argument, except S_out and S_in as above.  Deterministic.  Errors as above.
 * ---------------------------------------------------------------------- */
int harts_la_step(int32_t dtype, int64_t n_seq, int64_t n_rows, int32_t H, int32_t d, float scale, const void* q,
                  const void* k, const void* v, const float* g, const int32_t* row_off, const float* S_in,
                  const int32_t* idx_in, int64_t n_in, float* S_out, const int32_t* idx_out, int64_t n_out, void* o,
                  void* stream);

int harts_kda_step(int32_t dtype, int64_t n_seq, int64_t n_rows, int32_t H, int32_t d, float scale, const void* q,
                   const void* k, const void* v, const float* g, const float* beta, const int32_t* row_off,
                   const float* S_in, const int32_t* idx_in, int64_t n_in, float* S_out, const int32_t* idx_out,
                   int64_t n_out, void* o, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* HARTS_ROLLOUT_H_ */
