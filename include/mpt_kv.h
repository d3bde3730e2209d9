/*
 * mpt_kv.h -- C ABI of the paged key/value cache operators (sm_103a).
 *
 * mpt.h lays prompts out so that an exact-prefix cache is hit most; these
 * calls serve the laid-out prompts: a cache of pages, table rows forked from a
 * cached prefix, new keys and values written into their pages, attention of
 * the new tokens over the cache, and the merge of attention over parts of the
 * keys (a prefix attended once for all requests under it, then each request's
 * own suffix).
 *
 * Conventions shared by every call:
 *   - All tensors are device memory owned by the caller; the calls copy
 *     nothing to the host, do not synchronise and allocate nothing, so they
 *     can be captured in a CUDA graph.  Work is enqueued on `stream` (a
 *     cudaStream_t, NULL = the legacy default stream).
 *   - The host checks what it can see (types, sizes, strides, alignment) and
 *     returns INVALID_ARG or TOO_LARGE before anything is enqueued.  What only
 *     the device sees (page ids, lengths, row numbers) is bounded by the
 *     kernels, as stated at each call: no value of them makes a kernel read or
 *     write outside the tensors.
 *   - A cache page holds page_size tokens (a power of two, 8 to 256) of every
 *     KV head.  Keys and values are addressed as
 *       k + page * k_stride[0] + slot * k_stride[1] + head * k_stride[2],
 *     the head_dim elements of one head contiguous; strides count elements and
 *     are multiples of 8, pointers are 16-byte aligned.
 *   - Request i owns the new tokens q_offsets[i] .. q_offsets[i+1] - 1 of the
 *     packed token axis and kv_lens[i] tokens of the cache, the new ones the
 *     last among them; its token at position p lies on page
 *     page_table[i * table_stride + p / page_size], slot p % page_size.
 *   - Attention clamps lengths to what the table and the token axis hold
 *     (0 <= kv_lens[i] <= table_width * page_size, offsets from 0 to tokens) and
 *     takes positions from the clamped ones.  Writes, and codes read back, take
 *     lengths as they are: token t of request i stands at kv_lens[i] -
 *     (q_offsets[i+1] - q_offsets[i]) + t - q_offsets[i], and one whose position
 *     the table does not have is dropped.  The two differ only where a length
 *     or an offset reaches past the tensors.
 *   - A page id outside [0, n_pages) is a page that the cache does not hold
 *     (-1 by convention): its keys are masked, writes to it are dropped.
 */
#ifndef MPT_KV_H
#define MPT_KV_H

#include "mpt.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types. */
#define MPT_KV_BF16 0
#define MPT_KV_F16 1
#define MPT_KV_F32 2 /* mpt_kv_merge and mpt_kv4_read only */

/* One layer's cache and the requests of one step. */
typedef struct mpt_kv_cache {
  void* k; /* device, `type` */
  void* v;
  int64_t k_stride[3]; /* elements between pages, slots, KV heads */
  int64_t v_stride[3];
  int32_t type; /* MPT_KV_BF16 or MPT_KV_F16 */
  int32_t n_pages;
  int32_t page_size;  /* power of two, 8 to 256 */
  int32_t kv_heads;   /* 1 to 1024 */
  int32_t head_dim;   /* multiple of 8, 8 to 256 */
  int32_t batch;      /* requests, 0 to 2^20 */
  const int32_t* page_table; /* [batch][table_stride] */
  int64_t table_stride;
  int32_t table_width; /* entries of a row, >= 1; table_width * page_size < 2^31 */
  const int32_t* q_offsets; /* [batch + 1], from 0, not decreasing (or attention does nothing, and writes drop tokens) */
  const int32_t* kv_lens;   /* [batch] */
} mpt_kv_cache;

/* Bytes of workspace mpt_kv_attend needs on the current device (it depends on
 * the device only, not on the lengths).  Errors: INVALID_ARG, CUDA. */
mpt_status mpt_kv_attend_workspace_bytes(int32_t head_dim, size_t* bytes);

/* Attention of new tokens over a paged cache (the new tokens' keys and values
 * already written to it).  Token t of request i (q_i new tokens, L_i keys)
 * stands at position p = L_i - q_i + t and sees the keys j <= p (causal != 0)
 * or every j < L_i (causal == 0), less the masked ones:
 *     out = sum_j softmax_j(scale q.k_j) v_j,   lse = ln sum_j exp(scale q.k_j).
 * A row that sees no key gives out = 0, lse = -inf.  A masked key has no part
 * in the result whatever its key and value hold (NaN and infinities among it).
 * Query head h reads KV head h / (heads / kv_heads).
 *   q, out: device, `type`, [tokens][heads][head_dim] with element strides
 *     q_stride[2] / out_stride[2] between tokens and heads (multiples of 8);
 *     16-byte aligned; out must not overlap q or the cache;
 *   heads: a multiple of kv_heads, heads / kv_heads <= 128, tokens times that
 *     < 2^31;
 *   lse: device float[tokens][heads], or NULL;
 *   max_q_len: the most new tokens of one request if the caller knows it, else
 *     0.  It only chooses the kernel; any value gives the same function.
 *   scale: finite, > 0.
 *   workspace: device, 256-byte aligned, at least
 *     mpt_kv_attend_workspace_bytes(); not shared with another call in flight.
 * Scores, maxima, sums and the accumulated output are 32-bit; probabilities
 * are rounded to `type` for the product with the values (f16: at 2^11 times
 * their size at least, so that many small ones keep their weight), the output
 * once at the end.  The same call gives the same bits.
 * A bounded wait inside a kernel that gives up shows in mpt_kv_check.
 * Errors: INVALID_ARG, TOO_LARGE, WORKSPACE_TOO_SMALL, CUDA. */
mpt_status mpt_kv_attend(const mpt_kv_cache* cache, const void* q, const int64_t* q_stride, int64_t tokens,
                         int32_t heads, int32_t max_q_len, int32_t causal, float scale, void* out,
                         const int64_t* out_stride, float* lse, void* workspace, size_t workspace_bytes,
                         void* stream);

/* Merge attention results over disjoint sets of keys: with
 * lse = ln sum_p exp(lse_p), out = sum_p exp(lse_p - lse) out_p.  A part with
 * lse_p = -inf has no part in the row whatever out_p holds; where every part
 * is empty, out = 0 and lse = -inf.
 *   outs: host array of n_parts device pointers, each `type`
 *     [rows][head_dim] contiguous, 16-byte aligned; lses: likewise float[rows];
 *   type: BF16, F16 or F32; out the same type; lse may be NULL;
 *   out may be one of the outs; no other overlap of out or lse with one another,
 *   an out or an lse of a part (INVALID_ARG).
 * Limits: 1 <= n_parts <= 16, rows >= 0, head_dim a multiple of 8 in 8..1024.
 * Errors: INVALID_ARG, TOO_LARGE, CUDA. */
mpt_status mpt_kv_merge(const void* const* outs, const float* const* lses, int32_t n_parts, int64_t rows,
                        int32_t head_dim, int32_t type, void* out, float* lse, void* stream);

/* Write the new tokens' keys and values (device, the cache's type,
 * [tokens][kv_heads][head_dim], element strides k_stride[2] / v_stride[2]
 * between tokens and heads, multiples of 8) into their pages.  Tokens whose
 * position is negative, beyond the table, or on a page that the cache does not
 * hold are dropped.  Errors: INVALID_ARG, TOO_LARGE, CUDA. */
mpt_status mpt_kv_write(const mpt_kv_cache* cache, const void* k_new, const int64_t* k_stride, const void* v_new,
                        const int64_t* v_stride, int64_t tokens, void* stream);

/* How positions turn new keys and queries: elements x_i and x_{i + rot/2}
 * (adjacent == 0), or x_{2i} and x_{2i+1}, i < rot / 2, of each head become
 *     x c - y s,   y c + x s      (x the first, y the second of the two)
 * with c = table[row][i], s = table[row][rot / 2 + i]; elements from rot on
 * stay.  A token's row is positions[token], or its position in its request's
 * cache where positions is NULL.  A token whose row the table does not have
 * has no place: its key and value are dropped, its query is not turned. */
typedef struct mpt_kv_turn {
  const float* table; /* device [rows][stride], 16-byte aligned */
  int64_t stride;     /* a multiple of 4, >= rot */
  int32_t rows;
  int32_t rot; /* a multiple of 16 (adjacent: of 8), up to head_dim */
  int32_t adjacent;
  int32_t heads;            /* of q, 1 to 2^17 */
  const int32_t* positions; /* device [tokens], or NULL */
  const void* q;            /* device, the type of the keys, [tokens][heads][head_dim], or NULL */
  void* q_out;              /* q turned; q itself (with its strides), or no overlap with it; none with
                             * the new keys and values (INVALID_ARG) or the cache */
  int64_t q_stride[2];      /* elements between tokens and heads, multiples of 8 */
  int64_t q_out_stride[2];
} mpt_kv_turn;

/* mpt_kv_write with the keys, and the queries where turn->q is given, turned on
 * the way: products and sums in 32 bits, one rounding to the type.  Queries of
 * every token of a request are turned, also of tokens that the cache drops;
 * q_out of tokens of no request is not written.
 * Errors: INVALID_ARG, TOO_LARGE, CUDA. */
mpt_status mpt_kv_write_rotated(const mpt_kv_cache* cache, const mpt_kv_turn* turn, const void* k_new,
                                const int64_t* k_stride, const void* v_new, const int64_t* v_stride, int64_t tokens,
                                void* stream);

/* ---------------------------------------------------------------------------
 * A cache in 4 bits.  Per token and KV head, each group of 32 elements (the
 * last one may be short) holds x as codes 0..15 with a step s and an offset z:
 *     s = max((max x - min x) / 15, max |x| / 120, 2^-18), rounded up to four
 *         significant bits,
 *     z = rint(min x / s),   c = min(max(rint(x / s) - z, 0), 15),
 * and c stands for (c + z) s, which f16 holds exactly; x is clamped to
 * +-3360 first, NaN becomes 0.  Every step is a 32-bit operation, rounded to
 * nearest even.  4.5 bits an element: 288 n bytes for 8 tokens' keys and values
 * of a head, n = ceil(head_dim / 32).
 * A page is [kv_heads][page_size / 8 tiles][288 n bytes]; a tile of 8 tokens:
 *     keys    [8 tokens][8 n pieces][2 bytes]
 *     marks   [8 tokens][n groups][step, offset]
 *     values  [4 pairs of tokens][8 n pieces][2 tokens][2 bytes]
 *     marks   [4 pairs][n groups][step, offset][2 tokens]
 * a piece being 4 elements in 16 bits, the first the lowest, rotated left by 6;
 * the step's byte the upper bits of 16 s as a positive f16 (5 of exponent, 3 of
 * mantissa), the offset's z + 128.  Missing elements of the last group are
 * written as its first one is.  What reads a step's byte takes those above 222
 * (16 s = 7168) for 222, so no bytes stand for an infinity or a NaN; where an
 * offset is below -120, which no write makes, attention rounds (c + z) s to f16.
 * ------------------------------------------------------------------------- */
typedef struct mpt_kv4_cache {
  void* pages;       /* device, 16-byte aligned */
  int64_t stride[2]; /* bytes between pages and KV heads, multiples of 16 */
  int32_t n_pages;
  int32_t page_size;  /* power of two, 8 to 256 */
  int32_t kv_heads;   /* 1 to 1024 */
  int32_t head_dim;   /* multiple of 8, 8 to 256 */
  int32_t batch;      /* as in mpt_kv_cache, with what follows */
  const int32_t* page_table;
  int64_t table_stride;
  int32_t table_width;
  const int32_t* q_offsets;
  const int32_t* kv_lens;
} mpt_kv4_cache;

/* Bytes of one KV head of a page.  Errors: INVALID_ARG. */
mpt_status mpt_kv4_page_bytes(int32_t page_size, int32_t head_dim, int64_t* bytes);

/* Write the new tokens' keys and values (`type`: BF16 or F16) as codes, the
 * keys and queries turned first where `turn` is given (NULL: not; the turned
 * keys are not rounded to `type` in between).  Otherwise as mpt_kv_write and
 * mpt_kv_write_rotated.  Errors: INVALID_ARG, TOO_LARGE, CUDA. */
mpt_status mpt_kv4_write(const mpt_kv4_cache* cache, const mpt_kv_turn* turn, int32_t type, const void* k_new,
                         const int64_t* k_stride, const void* v_new, const int64_t* v_stride, int64_t tokens,
                         void* stream);

/* Read the new tokens' keys and values (what their codes stand for, rounded to
 * `type`: BF16, F16 or F32) back out of their pages, for a request that is
 * handed to another cache or a check.  0 where the cache has no place for a
 * token; rows of no request are not written.
 *   k_out, v_out: device [tokens][kv_heads][head_dim], strides as in mpt_kv_write;
 *   they must not overlap one another (INVALID_ARG) or the pages; parts of one
 *   tensor may interleave.
 * Errors: INVALID_ARG, TOO_LARGE, CUDA. */
mpt_status mpt_kv4_read(const mpt_kv4_cache* cache, int32_t type, void* k_out, const int64_t* k_stride, void* v_out,
                        const int64_t* v_stride, int64_t tokens, void* stream);

/* Bytes of workspace mpt_kv4_attend needs on the current device, whatever the
 * sizes.  Errors: INVALID_ARG, CUDA. */
mpt_status mpt_kv4_attend_workspace_bytes(size_t* bytes);

/* mpt_kv_attend over a cache in 4 bits; q and out are `type` (BF16 or F16).
 * Keys and values enter the products as the f16 values that their codes stand
 * for, queries as f16, probabilities as f16 at 2^11 times their size at least.
 * A row of bf16 queries is first divided by the power of two 2^e that its largest
 * element is in [2^e, 2^(e+1)) of: elements of 2^(e-17) and more stay as they
 * are, smaller ones are off by up to 2^(e-25) (an error of the score of up to
 * scale 2^(e-25) sum |k|).  Errors: as mpt_kv_attend. */
mpt_status mpt_kv4_attend(const mpt_kv4_cache* cache, int32_t type, const void* q, const int64_t* q_stride,
                          int64_t tokens, int32_t heads, int32_t max_q_len, int32_t causal, float scale, void* out,
                          const int64_t* out_stride, float* lse, void* workspace, size_t workspace_bytes,
                          void* stream);

/* ---------------------------------------------------------------------------
 * Bookkeeping of pages, on the device.  A page is free iff its reference count
 * is <= 0; table row r holds lens[r] tokens on its first
 * ceil(lens[r] / page_size) entries (the rest are -1).  Only a row's last page
 * can be partly filled, and it belongs to that row alone; full pages may be
 * shared by rows.  The calls keep this.
 *   Fresh pages are the free ones of lowest id, in list order.
 *   status: device int32[2], written by the calls that take it: [0] 0, or the
 *     reasons why nothing was changed, MPT_KV_BAD_ROW (a row out of range or
 *     listed twice, a fork onto a row that holds tokens, keep or a length out
 *     of range) + MPT_KV_NO_PAGES (too few free pages) + MPT_KV_ROW_FULL (a
 *     row would need more than `width` pages); [1] the free pages left.
 * Limits: rows <= 2^20, list length n <= min(rows, 16384), n_pages < 2^30,
 * width * page_size < 2^31.
 * Errors of each: INVALID_ARG, TOO_LARGE, CUDA.
 * ------------------------------------------------------------------------- */
#define MPT_KV_BAD_ROW 1
#define MPT_KV_NO_PAGES 2
#define MPT_KV_ROW_FULL 4

typedef struct mpt_kv_book {
  int32_t* table; /* [rows][table_stride] */
  int64_t table_stride;
  int32_t width; /* entries of a row */
  int32_t rows;
  int32_t* lens; /* [rows] */
  int32_t* refs; /* [n_pages] */
  int32_t n_pages;
  int32_t page_size; /* power of two, 8 to 256 */
} mpt_kv_book;

/* Fork: row dst[j] (empty) gets the first keep[j] tokens of row src[j].  Its
 * full pages are shared (one more reference each); a part page is copied to a
 * fresh page, which the caller's copy_src[j] -> copy_dst[j] names (-1, -1
 * where there is none) for mpt_kv_copy_pages.  src may repeat, dst may not.
 *   src, dst, keep, copy_src, copy_dst: device int32[n]. */
mpt_status mpt_kv_fork(const mpt_kv_book* book, const int32_t* src, const int32_t* dst, const int32_t* keep,
                       int32_t n, int32_t* copy_src, int32_t* copy_dst, int32_t* status, void* stream);

/* Extend: row rows[j] grows by more[j] >= 0 tokens, onto fresh pages where its
 * last page is full.  No row twice.  device int32[n] each. */
mpt_status mpt_kv_extend(const mpt_kv_book* book, const int32_t* rows, const int32_t* more, int32_t n,
                         int32_t* status, void* stream);

/* Free: the pages of row rows[j] lose one reference each, the row is emptied
 * (length 0, entries -1).  No row twice. */
mpt_status mpt_kv_free(const mpt_kv_book* book, const int32_t* rows, int32_t n, int32_t* status, void* stream);

/* Compact: with n live pages (references > 0), the i-th live page of id >= n
 * moves to the i-th free page of id < n; reference counts and table entries
 * follow.  copy_src / copy_dst (device int32[n_pages / 2]) get the moves for
 * mpt_kv_copy_pages, then -1. */
mpt_status mpt_kv_compact(const mpt_kv_book* book, int32_t* copy_src, int32_t* copy_dst, int32_t* status,
                          void* stream);

/* Copy whole pages within a pool, src[j] -> dst[j] (device int32[n]) in every
 * plane (a layer's pages; `planes` of them, plane_stride bytes apart; pages
 * page_stride bytes apart, page_bytes of which are copied).  Pairs with an id
 * outside [0, n_pages) are skipped.  No page may be the destination of one
 * pair and a page of another.  All sizes, strides and the pool's address are
 * multiples of 16 bytes.  Errors: INVALID_ARG, TOO_LARGE, CUDA. */
mpt_status mpt_kv_copy_pages(void* pool, int32_t planes, int64_t plane_stride, int32_t n_pages, int64_t page_stride,
                             int64_t page_bytes, const int32_t* src, const int32_t* dst, int32_t n, void* stream);

/* Waits for `stream`, then reports what kernels of this header met on the
 * current device, on any stream, that no call has reported: MPT_ERR_TIMEOUT
 * when a bounded wait on a shared-memory barrier gave up (the results of the
 * calls since the last MPT_OK are not to be used), MPT_ERR_INTERNAL when an
 * index failed its check in the bounds-checked build (mpt_build_info; the
 * access was left out), MPT_OK otherwise.  Errors also: CUDA. */
mpt_status mpt_kv_check(void* stream);

#ifdef __cplusplus
}
#endif

#endif /* MPT_KV_H */
