/*
 * libqllm: a key/value cache in 4-bit codes, what fills it and the attention that reads it.  The q/k/v layer's output goes in
 * (qllm_kv_append), attention's output is the next layer's input.  All conventions as in qllm.h: device pointers unless a name
 * ends in _host or a parameter says "host", the caller's stream, no allocation, no synchronisation, host-checkable arguments
 * checked before anything is launched.  The contents of device arrays need not be trusted here: a page number, a line of the
 * table, a length or a row number outside its range is treated as "not there" (below) and never reached through.
 */
#ifndef QLLM_KV_H
#define QLLM_KV_H

#include <stdint.h>

#include "qllm.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * One layer's cache: pages of page_tokens tokens (32, 64, 128 or 256) for `heads` key/value heads of `dim` channels (64 or 128).
 * The key and the value of a token and head are each quantized by Eq. (2) of qllm.h at 4 bits (qmax 15) over their dim channels:
 * alpha, beta and dim codes, standing for alpha * (code - beta).  Two things differ from there: alpha is (max - min) times the
 * float nearest to 1/15, one rounding and no division, and a vector whose alpha would be below 2^-126 counts as constant
 * (alpha = 1).  A page is qllm_kv_page_bytes(...) = heads * page_tokens * (dim + 16) bytes; head h's part of it, at
 * h * page_tokens * (dim + 16), is
 *   codes of the keys    [page_tokens][dim / 2]  code 2j in bits 0..3, code 2j+1 in bits 4..7 of byte j
 *   codes of the values  [page_tokens][dim / 2]
 *   alpha of the keys    [page_tokens] float        beta of the keys    [page_tokens] int32
 *   alpha of the values  [page_tokens] float        beta of the values  [page_tokens] int32
 * qllm_kv_append writes alphas from 2^-126 on.  Attention takes what others wrote too: an alpha of 0 (a page of zero bytes, tokens that
 * a length counts before they are appended) is a key or value of 0, a value's alpha below 2^-126 may count as 0, and one that is
 * negative or not finite may spoil the rows that see the token.  What lies in places of no token may be anything.
 */
typedef struct {
    int64_t heads, dim, page_tokens, n_pages;
    uint8_t *pages; /* [n_pages][qllm_kv_page_bytes(heads, dim, page_tokens)], 16-byte aligned */
} qllm_kv_cache;

/* Negative return = qllm_status (SHAPE). */
int64_t qllm_kv_page_bytes(int64_t heads, int64_t dim, int64_t page_tokens);

/*
 * The sequences of a step.  Sequence i owns the rows row_start[i] .. row_start[i+1]-1 of the step's tensors: its n_i newest
 * tokens, at the positions length - n_i .. length - 1 of line slot[i] of the table.  Rows of no sequence (behind the last one,
 * or of a line outside the table in qllm_kv_append and qllm_kv_read) are left as they were; sequences may have no rows.
 * Position p of a line lies in page table[line][p / page_tokens]; a page number outside [0, n_pages), or a p beyond the line's
 * end, is "not there": nothing is written, and attention does not see the token.
 * Limits: rows < 2^24, n_seqs <= 2^20, table_ld * page_tokens < 2^31, n_pages < 2^31; the cache may be of any size.
 */
typedef struct {
    int64_t rows;             /* rows of the step's tensors */
    int64_t n_seqs;
    const int32_t *row_start; /* [n_seqs + 1], ascending; NULL: sequence i has row i alone */
    const int32_t *slot;      /* [n_seqs] lines of the table; NULL: line i.  No line twice in qllm_kv_append */
    int64_t n_slots, table_ld;
    const int32_t *table;     /* [n_slots][table_ld] page numbers */
    const int32_t *length;    /* [n_slots] tokens, those of this step included */
} qllm_kv_batch;

typedef enum {
    QLLM_ROPE_NONE = 0,
    QLLM_ROPE_HALVES = 1, /* channels d and d + dim/2 turn together by position * inv_freq[d] */
    QLLM_ROPE_PAIRS = 2   /* channels 2d and 2d + 1 */
} qllm_rope;

/* ------------------------------------------------------------------------------------------
 * Rotary positions on the step's queries and keys, Eq. (2) on its keys and values, codes into the sequences' pages.
 *   q        [rows, ldq], q_heads * dim columns; q_out [rows, ldq_out] receives the rotated queries (may be q itself with the
 *            same stride; must not overlap it, k or v otherwise).  Both NULL: keys and values only.
 *   k, v     [rows, ldk], [rows, ldv], heads * dim columns; x_dtype (fp32 / bf16) for all four.
 *   inv_freq [dim / 2] double, angle per position (ignored, may be NULL, with QLLM_ROPE_NONE: q_out is then a copy).
 * Fixed arithmetic: a = p * inv_freq[d] in double, c = cos a and s = sin a rounded to float; x1' = x1 c - x2 s and
 * x2' = x2 c + x1 s with products and sum in double, rounded once to float; queries are then rounded to x_dtype, keys go to
 * Eq. (2) as they are.  A key or value that is not finite, or whose max - min is not (from 2^128 on), gets
 * unspecified codes, itself alone.
 * Any 2-byte (bf16) or 4-byte (fp32) aligned rows work; 16-byte aligned rows with 16-byte strides take 16-byte accesses.
 * Errors: NULL / SHAPE / DTYPE (also an unknown rope) / ALIGN / HIP.  rows == 0 or n_seqs == 0: no-op.
 */
int32_t qllm_kv_append(const void *q, int64_t ldq, int64_t q_heads, void *q_out, int64_t ldq_out, const void *k, int64_t ldk,
                       const void *v, int64_t ldv, int32_t x_dtype, int32_t rope, const double *inv_freq,
                       const qllm_kv_cache *cache, const qllm_kv_batch *batch, void *hip_stream);

/* What the cache holds for the step's rows: alpha * (code - beta), rounded to float (from |beta| = 2^23 on to double first) and
 * from there to dtype (fp32 / bf16), in k_out [rows, ldk] and v_out [rows, ldv] (either may be NULL).  Rows whose token is not there
 * are left as they were.  Errors as above. */
int32_t qllm_kv_read(const qllm_kv_cache *cache, const qllm_kv_batch *batch, void *k_out, int64_t ldk, void *v_out, int64_t ldv,
                     int32_t dtype, void *hip_stream);

/* ------------------------------------------------------------------------------------------
 * Causal attention of the step's queries over the cache, q_heads a multiple of heads (query head h reads head
 * h / (q_heads / heads)).  A query at position p sees the tokens t <= p of its line that are there, with window > 0 only
 * t > p - window:
 *     out = sum_t e^(scale q.k_t) v_t / sum_t e^(scale q.k_t),   0 where nothing is seen.
 *   scale    any sign; |scale| below 2.35e38 (scores are held in base 2, times log2 e; larger ones: SHAPE).
 *   q        [rows, ldq] q_dtype, out [rows, ldo] out_dtype (fp32 / bf16), q_heads * dim columns.  out may be q itself (one
 *            type, one stride); must not overlap it otherwise.  q_heads <= 2^15, and with G = q_heads / heads: tiles = rows * G / 16 +
 *            n_seqs < 2^23 and tiles * (table_ld * page_tokens / 32 + 8) < 2^31.
 *   workspace  16-byte aligned, qllm_kv_attention_workspace_bytes(cache, batch, q_heads) bytes (read on the host: of the
 *            two structs only the sizes, and whether row_start is NULL; a smaller step may need more); contents undefined
 *            afterwards, two calls in flight at once need one each.
 * Equal calls give equal bits.
 * Codes enter the matrix cores as exact bf16 integers; scores, maxima and sums are fp32.  The weights (times a value's alpha)
 * meet the values in bf16 parts: with fp32 queries, which come in three parts too, 24 bits; with bf16 queries 2^-16 of each is
 * left out at most, in sequences of many rows with bf16 out 2^-8 (one part, rounded, which is also what is summed below the line).
 * A query that is not finite spoils the output of its own row and head alone.
 * The fp32 numbers have to hold: (32 + |beta|) sum |q|, and |scale| alpha times that, of every key that a row sees; values whose
 * alphas are all below 2^-88, or some above 2^80, may overflow a sum or lose bits.
 * In sequences of many rows with bf16 queries a key whose |scale| alpha is below 2^-90 counts as one of 2^-90 (which is nothing
 * for queries below 2^30), and a token whose value's alpha is less than 2^-100 of another's that the query sees may count for
 * less than its share below the line.
 * Errors: NULL / SHAPE / DTYPE / ALIGN / WORKSPACE / HIP.  rows == 0 or n_seqs == 0: no-op.
 */
int64_t qllm_kv_attention_workspace_bytes(const qllm_kv_cache *cache, const qllm_kv_batch *batch, int64_t q_heads);
int32_t qllm_kv_attention(const void *q, int32_t q_dtype, int64_t ldq, int64_t q_heads, const qllm_kv_cache *cache,
                          const qllm_kv_batch *batch, float scale, int64_t window, void *out, int32_t out_dtype, int64_t ldo,
                          void *workspace, int64_t workspace_bytes, void *hip_stream);

/* ------------------------------------------------------------------------------------------
 * Page dst_host[i] becomes a copy of page src_host[i], in each of n_layers layers that lie layer_stride bytes apart.
 * src_host, dst_host: HOST arrays, read before the call returns (under stream capture the graph keeps this very list).  No page
 * may be named as a destination twice, or be written to and read; a pair of a page with itself does nothing.
 * pages 16-byte aligned, page_bytes and layer_stride multiples of 16, layer_stride >= n_pages * page_bytes if n_layers > 1.
 * Errors: NULL / SHAPE / ALIGN / PAGES (a number out of range, a clash) / WORKSPACE (no host memory for the check) / HIP.
 */
int32_t qllm_kv_copy_pages(uint8_t *pages, int64_t n_layers, int64_t layer_stride, int64_t n_pages, int64_t page_bytes,
                           const int32_t *src_host, const int32_t *dst_host, int64_t n, void *hip_stream);

/* ------------------------------------------------------------------------------------------
 * Which page belongs to whom.  HOST pointers; one book serves all layers.  A line holds `length` tokens in its first
 * ceil(length / page_tokens) pages; its other entries are -1.  refs counts the lines that hold a page, 0: the page is free.
 * A page that is only partly filled belongs to one line, so appending never writes into a shared page.
 * Each call checks everything first and changes nothing if it fails: SHAPE (a line out of range, a negative count, a line too
 * short for its tokens, a child that is not empty or is a parent too), PAGES (too few free pages, a book that contradicts
 * itself where the call reads it), WORKSPACE (no host memory).  Requests are served in order; new pages are the lowest free ones.
 */
typedef struct {
    int64_t page_tokens, n_slots, table_ld, n_pages;
    int32_t *table;  /* [n_slots][table_ld] */
    int32_t *length; /* [n_slots] */
    int32_t *refs;   /* [n_pages] */
} qllm_kv_book;

/* Makes room for counts[i] more tokens in line slots[i] (a line named twice grows twice). */
int32_t qllm_kv_reserve_host(const qllm_kv_book *book, const int32_t *slots, const int32_t *counts, int64_t n);
/* Line children[i], empty so far, continues line parents[i]: it shares the parent's full pages and gets a page of its own for a
 * partly filled last one, which has to be copied: page src[j] to page dst[j] for j < the returned number (src, dst: n entries). */
int64_t qllm_kv_fork_host(const qllm_kv_book *book, const int32_t *parents, const int32_t *children, int64_t n, int32_t *src,
                          int32_t *dst);
/* Empties the lines: their pages lose a reference each.  An empty line stays empty. */
int32_t qllm_kv_free_host(const qllm_kv_book *book, const int32_t *slots, int64_t n);
/* With U pages in use: those numbered U and above move, in ascending order, to the free ones below U, in ascending order; table
 * and refs follow.  Page src[j] has to be copied to page dst[j] for j < the returned number (src, dst: n_pages entries). */
int64_t qllm_kv_compact_host(const qllm_kv_book *book, int32_t *src, int32_t *dst);

#ifdef __cplusplus
}
#endif
#endif /* QLLM_KV_H */
