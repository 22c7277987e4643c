// Which page of the key/value cache belongs to whom: host side, no GPU.  Every call runs through its requests twice, first on
// numbers of its own (lengths, references, how many fresh pages), then for good, so that a call that fails has changed nothing.
#include <stdint.h>

#include <memory>
#include <new>

#include "qllm_kv.h"

namespace {

int32_t check_book(const qllm_kv_book *b)
{
    if (!b || !b->table || !b->length || !b->refs) return QLLM_ERR_NULL;
    if (b->n_slots <= 0 || b->n_slots > INT32_MAX || b->table_ld <= 0 || b->n_pages <= 0 || b->n_pages > INT32_MAX) return QLLM_ERR_SHAPE;
    const int64_t p = b->page_tokens;
    if ((p != 32 && p != 64 && p != 128 && p != 256) || b->table_ld > INT32_MAX / p) return QLLM_ERR_SHAPE;
    return QLLM_OK;
}

int64_t pages_for(const qllm_kv_book *b, int64_t tokens) { return (tokens + b->page_tokens - 1) / b->page_tokens; }

// A line's length and pages as the book should have them.
bool line_is_sound(const qllm_kv_book *b, int64_t line)
{
    const int64_t len = b->length[line];
    if (len < 0 || pages_for(b, len) > b->table_ld) return false;
    const int32_t *row = b->table + line * b->table_ld;
    for (int64_t k = 0; k < pages_for(b, len); ++k)
        if (row[k] < 0 || row[k] >= b->n_pages || b->refs[row[k]] <= 0) return false;
    return true;
}

struct Fresh { // the lowest free page, then the next
    const qllm_kv_book *b;
    int64_t at = 0;
    int32_t take()
    {
        while (b->refs[at] != 0) ++at;
        b->refs[at] = 1;
        return (int32_t)at++;
    }
};

int64_t free_pages(const qllm_kv_book *b)
{
    int64_t n = 0;
    for (int64_t p = 0; p < b->n_pages; ++p) n += b->refs[p] == 0;
    return n;
}

bool line_ok(const qllm_kv_book *b, int32_t line) { return line >= 0 && line < b->n_slots; }

} // namespace

extern "C" int64_t qllm_kv_page_bytes(int64_t heads, int64_t dim, int64_t page_tokens)
{
    if (heads <= 0 || heads > (1 << 16) || (dim != 64 && dim != 128)) return QLLM_ERR_SHAPE;
    if (page_tokens != 32 && page_tokens != 64 && page_tokens != 128 && page_tokens != 256) return QLLM_ERR_SHAPE;
    return heads * page_tokens * (dim + 16);
}

extern "C" int32_t qllm_kv_reserve_host(const qllm_kv_book *b, const int32_t *slots, const int32_t *counts, int64_t n)
{
    const int32_t rc = check_book(b);
    if (rc != QLLM_OK) return rc;
    if (n < 0) return QLLM_ERR_SHAPE;
    if (n > 0 && (!slots || !counts)) return QLLM_ERR_NULL;
    std::unique_ptr<int64_t[]> len(new (std::nothrow) int64_t[(size_t)b->n_slots]);
    if (!len) return QLLM_ERR_WORKSPACE;
    for (int64_t i = 0; i < n; ++i) {
        if (!line_ok(b, slots[i]) || counts[i] < 0) return QLLM_ERR_SHAPE;
        len[slots[i]] = b->length[slots[i]];
        if (!line_is_sound(b, slots[i])) return QLLM_ERR_PAGES;
        const int64_t part = len[slots[i]] % b->page_tokens;
        if (part && b->refs[b->table[slots[i] * b->table_ld + len[slots[i]] / b->page_tokens]] != 1) return QLLM_ERR_PAGES;
    }
    int64_t fresh = 0;
    for (int64_t i = 0; i < n; ++i) {
        const int64_t now = len[slots[i]] + counts[i];
        if (pages_for(b, now) > b->table_ld) return QLLM_ERR_SHAPE;
        fresh += pages_for(b, now) - pages_for(b, len[slots[i]]);
        len[slots[i]] = now;
    }
    if (fresh > free_pages(b)) return QLLM_ERR_PAGES;
    Fresh f{b};
    for (int64_t i = 0; i < n; ++i) {
        const int64_t was = b->length[slots[i]], now = was + counts[i];
        for (int64_t k = pages_for(b, was); k < pages_for(b, now); ++k) b->table[slots[i] * b->table_ld + k] = f.take();
        b->length[slots[i]] = (int32_t)now;
    }
    return QLLM_OK;
}

extern "C" int64_t qllm_kv_fork_host(const qllm_kv_book *b, const int32_t *parents, const int32_t *children, int64_t n, int32_t *src, int32_t *dst)
{
    const int32_t rc = check_book(b);
    if (rc != QLLM_OK) return rc;
    if (n < 0) return QLLM_ERR_SHAPE;
    if (n > 0 && (!parents || !children || !src || !dst)) return QLLM_ERR_NULL;
    constexpr uint8_t CHILD = 1, SOUND = 2; // of a line: a child of this call; a parent that has been checked
    std::unique_ptr<uint8_t[]> known(new (std::nothrow) uint8_t[(size_t)b->n_slots]());
    if (!known) return QLLM_ERR_WORKSPACE;
    int64_t fresh = 0;
    for (int64_t i = 0; i < n; ++i) {
        if (!line_ok(b, parents[i]) || !line_ok(b, children[i])) return QLLM_ERR_SHAPE;
        if (b->length[children[i]] != 0 || known[children[i]]) return QLLM_ERR_SHAPE;
        known[children[i]] = CHILD;
    }
    for (int64_t i = 0; i < n; ++i) {
        if (known[parents[i]] == CHILD) return QLLM_ERR_SHAPE;
        if (known[parents[i]] != SOUND && !line_is_sound(b, parents[i])) return QLLM_ERR_PAGES;
        known[parents[i]] = SOUND;
        // n_slots lines share a page at most, far below int32
        fresh += b->length[parents[i]] % b->page_tokens != 0;
    }
    if (fresh > free_pages(b)) return QLLM_ERR_PAGES;
    Fresh f{b};
    int64_t copies = 0;
    for (int64_t i = 0; i < n; ++i) {
        const int64_t len = b->length[parents[i]], whole = len / b->page_tokens;
        const int32_t *from = b->table + parents[i] * b->table_ld;
        int32_t *to = b->table + children[i] * b->table_ld;
        for (int64_t k = 0; k < whole; ++k) {
            to[k] = from[k];
            b->refs[from[k]] += 1;
        }
        if (len % b->page_tokens) {
            to[whole] = f.take();
            src[copies] = from[whole], dst[copies] = to[whole];
            ++copies;
        }
        b->length[children[i]] = (int32_t)len;
    }
    return copies;
}

extern "C" int32_t qllm_kv_free_host(const qllm_kv_book *b, const int32_t *slots, int64_t n)
{
    const int32_t rc = check_book(b);
    if (rc != QLLM_OK) return rc;
    if (n < 0) return QLLM_ERR_SHAPE;
    if (n > 0 && !slots) return QLLM_ERR_NULL;
    std::unique_ptr<int32_t[]> less(new (std::nothrow) int32_t[(size_t)b->n_pages]());
    std::unique_ptr<uint8_t[]> seen(new (std::nothrow) uint8_t[(size_t)b->n_slots]());
    if (!less || !seen) return QLLM_ERR_WORKSPACE;
    for (int64_t i = 0; i < n; ++i) {
        if (!line_ok(b, slots[i])) return QLLM_ERR_SHAPE;
        if (!line_is_sound(b, slots[i])) return QLLM_ERR_PAGES;
        if (seen[slots[i]]) continue;
        seen[slots[i]] = 1;
        for (int64_t k = 0; k < pages_for(b, b->length[slots[i]]); ++k) {
            const int32_t p = b->table[slots[i] * b->table_ld + k];
            if (++less[p] > b->refs[p]) return QLLM_ERR_PAGES; // held by more lines than it counts
        }
    }
    for (int64_t i = 0; i < n; ++i) {
        int32_t *row = b->table + slots[i] * b->table_ld;
        for (int64_t k = 0; k < pages_for(b, b->length[slots[i]]); ++k) {
            b->refs[row[k]] -= 1;
            row[k] = -1;
        }
        b->length[slots[i]] = 0;
    }
    return QLLM_OK;
}

extern "C" int64_t qllm_kv_compact_host(const qllm_kv_book *b, int32_t *src, int32_t *dst)
{
    const int32_t rc = check_book(b);
    if (rc != QLLM_OK) return rc;
    if (!src || !dst) return QLLM_ERR_NULL;
    for (int64_t i = 0; i < b->n_slots; ++i)
        if (!line_is_sound(b, i)) return QLLM_ERR_PAGES;
    std::unique_ptr<int32_t[]> to(new (std::nothrow) int32_t[(size_t)b->n_pages]);
    if (!to) return QLLM_ERR_WORKSPACE;
    int64_t used = 0, moves = 0, hole = 0;
    for (int64_t p = 0; p < b->n_pages; ++p) used += b->refs[p] != 0, to[p] = (int32_t)p;
    for (int64_t p = used; p < b->n_pages; ++p) {
        if (b->refs[p] == 0) continue;
        while (b->refs[hole] != 0) ++hole; // as many holes below `used` as pages in use at or above it
        src[moves] = (int32_t)p, dst[moves] = (int32_t)hole, ++moves;
        to[p] = (int32_t)hole++;
    }
    for (int64_t m = 0; m < moves; ++m) {
        b->refs[dst[m]] = b->refs[src[m]];
        b->refs[src[m]] = 0;
    }
    for (int64_t i = 0; i < b->n_slots; ++i)
        for (int64_t k = 0; k < pages_for(b, b->length[i]); ++k) {
            int32_t &page = b->table[i * b->table_ld + k];
            page = to[page];
        }
    return moves;
}
