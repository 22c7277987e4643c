// Internal to libqllm: what the translation units of the 4-bit key/value cache share.
#ifndef QLLM_KV_COMMON_H
#define QLLM_KV_COMMON_H

#include <hip/hip_runtime.h>

#include <stdint.h>

#include "kv_index.h"
#include "qllm_kv.h"

extern "C" void qllm_note_hip_error(const char *step, const char *name);

namespace qllm_kv_detail {

// The sequences of a step and one layer's pages, as a kernel gets them (sizes checked on the host: all below 2^31).
struct Step {
    int32_t rows, n_seqs, n_slots, table_ld, n_pages, heads, page_shift; // tokens of a page: 1 << page_shift
    const int32_t *row_start, *slot, *table, *length;
    uint8_t *pages;
    int64_t page_bytes;
};

// A sequence's rows and tokens, whatever the device arrays say: rows within the step's, no line outside the table.
struct Seq {
    int32_t row, n;   // its rows
    int32_t line;     // of the table, -1: none
    int32_t len;      // tokens, those beyond the line's last page included
};

__device__ __forceinline__ int32_t row_of(const Step &s, int32_t i)
{
    if (!s.row_start) return i;
    const int32_t r = s.row_start[i];
    return r < 0 ? 0 : (r > s.rows ? s.rows : r);
}

__device__ __forceinline__ Seq seq_of(const Step &s, int32_t i)
{
    Seq q;
    q.row = row_of(s, i);
    const int32_t n = row_of(s, i + 1) - q.row;
    q.n = n > 0 ? n : 0;
    const int32_t line = s.slot ? s.slot[i] : i;
    q.line = line >= 0 && line < s.n_slots ? line : -1;
    const int32_t len = q.line >= 0 ? s.length[q.line] : 0;
    q.len = len > 0 ? len : 0;
    return q;
}

// The page of position p of a line, -1 where it is not there (any p).
__device__ __forceinline__ int32_t page_of(const Step &s, int32_t line, int32_t p)
{
    const int32_t k = entry_of(p, s.page_shift, s.table_ld);
    if (line < 0 || k < 0) return -1;
    const int32_t page = s.table[(int64_t)line * s.table_ld + k];
    return page >= 0 && page < s.n_pages ? page : -1;
}

// The largest i < n_seqs with first(i) <= x for an ascending first, by one wave: 64 candidates per trip to memory, then 64 between
// two of them.  Any answer in [0, n_seqs) where first does not ascend.
template <class F>
__device__ __forceinline__ int32_t last_not_above(int32_t n_seqs, int64_t x, F first)
{
    const int32_t lane = threadIdx.x & 63;
    int32_t found = 0, width = n_seqs;
    for (;;) {
        const int32_t step = (int32_t)((uint32_t)(width + 63) / 64u);
        const bool in = lane * step < width && first(found + lane * step) <= x;
        const int32_t count = __popcll(__ballot(in));
        const int32_t skipped = count > 1 ? (count - 1) * step : 0;
        found += skipped;
        if (step <= 1) return found;
        width = step < width - skipped ? step : width - skipped;
    }
}

// Checks shared by the entry points; fills a Step.
inline int32_t prepare_step(const qllm_kv_cache *cache, const qllm_kv_batch *batch, bool contents, Step *out)
{
    if (!cache || !batch) return QLLM_ERR_NULL;
    const int64_t pb = qllm_kv_page_bytes(cache->heads, cache->dim, cache->page_tokens);
    if (pb < 0) return QLLM_ERR_SHAPE;
    if (cache->n_pages <= 0 || cache->n_pages > INT32_MAX) return QLLM_ERR_SHAPE;
    if (batch->rows < 0 || batch->rows >= (1 << 24) || batch->n_seqs < 0 || batch->n_seqs > (1 << 20)) return QLLM_ERR_SHAPE;
    if (batch->n_slots <= 0 || batch->n_slots > INT32_MAX || batch->table_ld <= 0) return QLLM_ERR_SHAPE;
    if (batch->table_ld > INT32_MAX / cache->page_tokens) return QLLM_ERR_SHAPE; // positions are int32
    if (!batch->row_start && batch->rows < batch->n_seqs) return QLLM_ERR_SHAPE;
    if (!batch->slot && batch->n_slots < batch->n_seqs) return QLLM_ERR_SHAPE;
    if (!contents) return QLLM_OK;
    if (!cache->pages || !batch->table || !batch->length) return QLLM_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(cache->pages) & 15u) return QLLM_ERR_ALIGN;
    if ((reinterpret_cast<uintptr_t>(batch->row_start) | reinterpret_cast<uintptr_t>(batch->slot) | reinterpret_cast<uintptr_t>(batch->table) |
         reinterpret_cast<uintptr_t>(batch->length)) & 3u) return QLLM_ERR_ALIGN;
    out->rows = (int32_t)batch->rows, out->n_seqs = (int32_t)batch->n_seqs, out->n_slots = (int32_t)batch->n_slots;
    out->table_ld = (int32_t)batch->table_ld, out->n_pages = (int32_t)cache->n_pages, out->heads = (int32_t)cache->heads;
    out->page_shift = __builtin_ctzll((unsigned long long)cache->page_tokens);
    out->row_start = batch->row_start, out->slot = batch->slot, out->table = batch->table, out->length = batch->length;
    out->pages = cache->pages, out->page_bytes = pb;
    return QLLM_OK;
}

inline int32_t launched(const char *what)
{
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return QLLM_OK;
    qllm_note_hip_error(what, hipGetErrorName(e));
    return QLLM_ERR_HIP;
}

} // namespace qllm_kv_detail

#endif
