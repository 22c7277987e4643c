// Internal to libqllm: index arithmetic of the cache's kernels at the edges of int32.  Positions may come close to 2^31 (a line has less
// than 2^31 of them) and lie below 0 (rows before the first token).  Nothing here overflows; plain C++ too, for a test on the host.
#ifndef QLLM_KV_INDEX_H
#define QLLM_KV_INDEX_H

#include <stdint.h>

#if defined(__HIPCC__)
#define QLLM_KV_INDEX __host__ __device__ __forceinline__
#else
#define QLLM_KV_INDEX inline
#endif

namespace qllm_kv_detail {

// The entry of a line of the table that position p belongs to, -1 where the line has none: negative p, or beyond its end.
QLLM_KV_INDEX int32_t entry_of(int32_t p, int32_t page_shift, int32_t table_ld)
{
    const int32_t k = p >> page_shift;
    return k >= 0 && k < table_ld ? k : -1;
}

// The first position of a block of 32 tokens that begins at or before position `last`, -1 for the others.  (Compared by blocks: lists
// that reach beyond the longest line ask for blocks that begin at 2^31 and later.)
QLLM_KV_INDEX int32_t block_begin(int32_t block, int32_t last) { return block >= 0 && block <= last >> 5 ? block * 32 : -1; }

// The first position that a query at position pos sees: 0, or with window > 0 the first of the newest `window`.  (Compared before
// subtracted: pos may be as low as -2^24, the window as large as 2^31 - 1.)
QLLM_KV_INDEX int32_t first_seen(int32_t pos, int32_t window) { return window > 0 && pos >= window ? pos - window + 1 : 0; }

} // namespace qllm_kv_detail

#endif
