// A reassembly map as qllm_add_norm_quant reads it (see qllm_gather in qllm_block.h).
#include <stdint.h>
#include <string.h>

#include "qllm_block.h"

extern "C" int32_t qllm_gather_map_host(const int32_t *row_ptr, const int32_t *src, const float *scale, int64_t C_in, int64_t C_out,
                                        int32_t *index, int64_t *index_len, int64_t *n_computed)
{
    if (!row_ptr || !src || !scale || !index_len || !n_computed) return QLLM_ERR_NULL;
    if (C_in <= 0 || C_in > QLLM_MAX_CHANNELS || C_out <= 0 || C_out > QLLM_MAX_CHANNELS) return QLLM_ERR_SHAPE;
    if (row_ptr[0] != 0) return QLLM_ERR_MAP;
    const int64_t S = (C_in + 7) / 8, padded = (C_out + QLLM_K_PAD - 1) / QLLM_K_PAD * QLLM_K_PAD;
    int64_t computed = 0, more = 2; // the first two pairs of `more` are no row's
    for (int64_t ch = 0; ch < C_out; ++ch) {
        if (row_ptr[ch + 1] <= row_ptr[ch]) return QLLM_ERR_MAP;
        for (int64_t e = row_ptr[ch]; e < row_ptr[ch + 1]; ++e)
            if (src[e] < 0 || src[e] >= C_in) return QLLM_ERR_MAP;
        if (row_ptr[ch + 1] - row_ptr[ch] == 1 && scale[row_ptr[ch]] == 1.0f) continue;
        ++computed;
        if (row_ptr[ch + 1] - row_ptr[ch] > 4) more += row_ptr[ch + 1] - row_ptr[ch] - 3;
    }
    if (8 * S + computed > QLLM_GATHER_PLACES) return QLLM_ERR_SHAPE;
    const int64_t at_computed = padded / 2, at_more = at_computed + 8 * computed, len = at_more + 2 * more;
    *index_len = len;
    *n_computed = computed;
    if (!index) return QLLM_OK;
    memset(index, 0, (size_t)len * sizeof(int32_t));
    auto place_of = [S](int64_t c) { return (c & 7) * S + (c >> 3); };
    auto bits_of = [](float f) {
        int32_t v;
        memcpy(&v, &f, sizeof v);
        return v;
    };
    int64_t j = 0, at = 2;
    for (int64_t ch = 0; ch < C_out; ++ch) {
        int64_t place;
        const int64_t e0 = row_ptr[ch], n = row_ptr[ch + 1] - e0;
        if (n == 1 && scale[e0] == 1.0f) {
            place = place_of(src[e0]);
        } else {
            place = 8 * S + j;
            int32_t *c = index + at_computed + 8 * j++;
            for (int64_t k = 0; k < 4; ++k) { // an entry that is not there: the first one's place, scale 0
                const uint32_t p = (uint32_t)place_of(src[k < n ? e0 + k : e0]);
                c[k / 2] = (int32_t)((uint32_t)c[k / 2] | p << (16 * (k & 1)));
                c[2 + k] = k < n ? bits_of(scale[e0 + k]) : 0;
            }
            if (n > 4) {
                c[6] = (int32_t)at;
                index[at_more + 2 * at++] = (int32_t)(n - 4);
                for (int64_t e = e0 + 4; e < e0 + n; ++e, ++at) {
                    index[at_more + 2 * at] = (int32_t)place_of(src[e]);
                    index[at_more + 2 * at + 1] = bits_of(scale[e]);
                }
            } else if (n > 2) {
                c[6] = 1;
            }
        }
        const uint32_t word = (uint32_t)index[ch / 2];
        index[ch / 2] = (int32_t)(ch & 1 ? word | (uint32_t)place << 16 : word | (uint32_t)place);
    }
    return QLLM_OK;
}
