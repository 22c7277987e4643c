/*
 * libqllm: what stands between the layers of a serving step.  The residual stream takes a layer's output, is normalised and
 * quantized for the next layer in one pass (qllm_add_norm_quant); low-rank adapters of many requests are added to what a shared
 * projection made of those codes (qllm_adapter_apply).  All conventions as in qllm.h: device pointers unless a name ends in _host
 * or a parameter says "host", the caller's stream, no allocation, no synchronisation, host-checkable arguments checked before
 * anything is launched.
 */
#ifndef QLLM_BLOCK_H
#define QLLM_BLOCK_H

#include <stdint.h>

#include "qllm.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * A reassembly map (qllm_map of qllm.h) as qllm_add_norm_quant reads it: for every output channel one place on chip, either that of
 * the input channel it copies or that of a channel computed beforehand (any row that is not one entry of scale exactly 1).
 * Made by qllm_gather_map_host; the contents of `index` are trusted.
 */
typedef struct {
    int64_t C_in, C_out;
    int64_t n_computed;   /* as qllm_gather_map_host says; 8 ceil(C_in / 8) + n_computed <= QLLM_GATHER_PLACES */
    const int32_t *index; /* device copy of that function's index, 16-byte aligned */
} qllm_gather;

/* Places (floats) that a workgroup has on chip for a row and its computed channels. */
#define QLLM_GATHER_PLACES 40448

/* HOST pointers.  Call once with index == NULL to get *index_len (int32 words) and *n_computed, then with index pointing at that
 * many words.  Input channel c has place (c mod 8) S + c / 8 with S = ceil(C_in / 8), the j-th computed channel 8 S + j.  Layout:
 *   places    for the output channels up to the next multiple of QLLM_K_PAD, two 16-bit numbers a word, the lower first (past C_out: 0)
 *   computed  [n_computed][8]: {place | place << 16, place | place << 16, scale, scale, scale, scale, m, 0} of the first four entries
 *             (one that is not there: the first one's place, scale 0); m: 0 for up to two entries, 1 for up to four, else where in
 *             `more` the others are
 *   more      pairs of words: {n, 0}, then n entries {place, scale}; pairs 0 and 1 are no row's
 * Errors: NULL, SHAPE (also more places than QLLM_GATHER_PLACES), MAP. */
int32_t qllm_gather_map_host(const int32_t *row_ptr, const int32_t *src, const float *scale, int64_t C_in, int64_t C_out,
                             int32_t *index, int64_t *index_len, int64_t *n_computed);

/* ------------------------------------------------------------------------------------------
 * The residual's addition, the norm, the reassembly and Eq. (2) in one pass over the rows:
 *     s = residual + x, in fp32, rounded once to r_dtype;      y = norm(s) as in qllm_norm_reassemble_quant;
 *     x^ = the map's combination of y (gather NULL: y itself);  codes, alpha, beta, rowsum of x^ as there, bit for bit what that
 * call makes of s.
 *   x         [N, ldx] x_dtype, or NULL: nothing is added, s = residual.
 *   residual  [N, ldr] r_dtype.
 *   sum_out   [N, lds] r_dtype receives s; may be residual itself (with lds == ldr), or x itself (one type, lds == ldx); NULL: s
 *             is not kept (nor is it with x NULL).
 *   y_out     [N, ldy] o_dtype or NULL: y before the reassembly, as adapters read it.
 *   out       the codes (rows of qllm_packed_row_bytes(C_out, bits), fully overwritten), or NULL: only s and y_out are made.
 *   values_out  [N, ldv] o_dtype or NULL: what the codes stand for, alpha * (code - beta) rounded to float, then to o_dtype; C_out
 *             columns; needs out.
 * No output may overlap another or an input, but for sum_out as said.  Rows may begin anywhere their type allows (2 or 4 bytes).
 * A row whose values are not finite gives unspecified codes, y and values, itself alone.
 * N < 2^31, C and C_out <= QLLM_MAX_CHANNELS.
 * Errors: NULL / SHAPE / BITS / DTYPE / ALIGN / HIP.  N == 0: no-op.
 */
int32_t qllm_add_norm_quant(const void *x, int32_t x_dtype, int64_t ldx, const void *residual, int32_t r_dtype, int64_t ldr, int64_t N,
                            int64_t C, void *sum_out, int64_t lds, int32_t norm, const float *gamma, const float *beta, float eps,
                            const qllm_gather *gather, int32_t bits, const qllm_qact *out, void *y_out, int64_t ldy, void *values_out,
                            int64_t ldv, int32_t o_dtype, void *hip_stream);

/* ------------------------------------------------------------------------------------------
 * Low-rank adapters.  A pool of n_adapters places, each with two factors of up to `rank` ranks for a projection of C inputs and O
 * outputs.  A fused projection (q | k | v, gate | up) has n_parts parts of its outputs, part_O[p] each, in this order, and a first
 * factor for each:
 *   A  [n_adapters][n_parts * rank][C], rank r of part p is row p * rank + r;   B  [n_adapters][O][rank];   w_dtype (fp32 / bf16) both
 *   scale  [n_adapters] float, or NULL: 1
 *   ranks  [n_adapters] int32, each adapter's own number of ranks (clamped to 0 .. rank), or NULL: all `rank`.  What A and B hold
 *          past an adapter's own ranks may be anything.
 */
#define QLLM_ADAPTER_PARTS 4
typedef struct {
    int64_t n_adapters, C, O, rank; /* rank: a multiple of 8, at most 256; n_adapters <= 8192; C, O < 2^24 */
    int32_t n_parts;                /* 1 .. QLLM_ADAPTER_PARTS; part_O sums up to O */
    int64_t part_O[QLLM_ADAPTER_PARTS];
    int32_t w_dtype;
    const void *A, *B;              /* 16-byte aligned */
    const float *scale;
    const int32_t *ranks;
} qllm_adapters;

/*
 * Which rows are whose: one plan serves all layers and projections of a step whose pools have n_adapters places.
 *   row_start [n_seqs + 1] ascending: sequence i owns the rows row_start[i] .. row_start[i + 1] - 1; NULL: row i alone.
 *   adapter   [n_seqs] its place in the pool; outside [0, n_adapters): the sequence has no adapter.
 * The plan lists the rows of the sequences adapter by adapter; rows of no sequence are not in it.
 *   plan      qllm_adapter_plan_bytes(rows, n_adapters) bytes, 16-byte aligned.
 * Device arrays that contradict this (rows out of range, sequences that overlap) are never reached through; rows may then be
 * missing or be served twice.
 * Limits: rows < 2^24, n_seqs <= 2^20.  Errors: NULL / SHAPE / ALIGN / WORKSPACE / HIP.
 */
int64_t qllm_adapter_plan_bytes(int64_t rows, int64_t n_adapters);
int32_t qllm_adapter_plan(int64_t rows, int64_t n_seqs, const int32_t *row_start, const int32_t *adapter, int64_t n_adapters, void *plan,
                          int64_t plan_bytes, void *hip_stream);

/* ------------------------------------------------------------------------------------------
 * For every row n of a sequence with adapter a, over the columns o of part p:
 *     out[n, o] = y[n, o] + scale_a sum_{r < ranks_a} B_a[o, r] sum_c A_a[p rank + r, c] x[n, c]
 * and out = y for the rows of a sequence without one.  Rows of no sequence are left as they were.
 *   x    [rows, ldx] x_dtype, C columns: what the projection's input was before it was quantized (qllm_add_norm_quant's y_out).
 *   y    [rows, ldy] y_dtype, O columns; out [rows, ldo] y_dtype, may be y itself (one stride), must not overlap it, x, A or B otherwise.
 *   plan      of qllm_adapter_plan for these rows and this n_adapters; of other numbers: nothing is done.
 *   workspace 16-byte aligned, qllm_adapter_workspace_bytes(adapters, rows) bytes (of the struct only sizes are read; never less
 *             for more rows); contents undefined afterwards, two calls in flight at once need one each.
 * Equal calls give equal bits.
 * The first product takes bf16 x and A through the bf16 matrix cores, other types as fp32; sums are fp32.  Its result times scale_a meets B
 * with all its 24 bits (bf16 B: in three bf16 parts, from 2^-110 on; nothing below 2^-133); the sum with y is fp32, rounded once.
 * A row of x that is not finite spoils its own row of out; an adapter that is not finite the rows that name it.
 * Limits: rows < 2^24, (rows / 64 + n_adapters + 1) * (O / 256 + n_parts) <= 2^24.
 * Errors: NULL / SHAPE / DTYPE / ALIGN / WORKSPACE / HIP.  rows == 0: no-op.
 */
int64_t qllm_adapter_workspace_bytes(const qllm_adapters *adapters, int64_t rows);
int32_t qllm_adapter_apply(const void *x, int32_t x_dtype, int64_t ldx, int64_t rows, const qllm_adapters *adapters, const void *plan,
                           int64_t plan_bytes, const void *y, int64_t ldy, void *out, int64_t ldo, int32_t y_dtype, void *workspace,
                           int64_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* QLLM_BLOCK_H */
