// Internal to libqllm: eight values to their codes (Eq. 2), packed, and the packed codes of a group to its row.
#ifndef QLLM_PACK_CODES_H
#define QLLM_PACK_CODES_H

#include "fused_common.h"

namespace qllm_detail {

// Eq. (2) for a row whose quotients are too large for the fused-multiply-add trick.
__device__ __noinline__ uint32_t slow_code(float x, float inv, int32_t beta, int32_t qmax)
{
    const double q = rne_product_slow(x, inv) + (double)beta;
    return (uint32_t)fmin(fmax(q, 0.0), (double)qmax);
}

// Quantizes 8 values (Eq. 2) and packs their codes, first value lowest.
//
// Fast form: b = bits(fma(x, inv, MAGIC)) is MAGIC_BITS + rne(x*inv); clamping b to [lo, lo + qmax]
// with lo = MAGIC_BITS - beta (one median-of-three) leaves lo + code.  The values are packed with
// shift-and-add in wrapping 32-bit arithmetic and the common offset lo * (1 + 2^BITS + 2^(2 BITS) + ...)
// is taken off once.  `live`: bit k clear forces code k to 0 (channels past the end of the row).
template <int BITS>
__device__ __forceinline__ void quant_pack(const float *val, uint32_t live, int32_t fast, float inv, int32_t beta,
                                           uint32_t &w0, uint32_t &w1)
{
    constexpr int QMAX = (1 << BITS) - 1;
    uint32_t c[GROUP], bias = 0;
    if (fast) {
        // floats in [2^23, 2^24) are integers and order like their bit patterns: clamp them as floats
        const float lo = __int_as_float(MAGIC_BITS - beta), hi = __int_as_float(MAGIC_BITS - beta + QMAX);
        bias = (uint32_t)(MAGIC_BITS - beta);
#pragma unroll
        for (int k = 0; k < GROUP; ++k)
            c[k] = __float_as_uint(__builtin_amdgcn_fmed3f(__builtin_fmaf(val[k], inv, MAGIC), lo, hi));
    } else {
#pragma unroll
        for (int k = 0; k < GROUP; ++k) c[k] = slow_code(val[k], inv, beta, QMAX); // rare; kept out of line
    }
    if (live != 0xffu) {
#pragma unroll
        for (int k = 0; k < GROUP; ++k) c[k] = (live >> k & 1u) ? c[k] : bias;
    }
    if constexpr (BITS == 4) {
        uint32_t p = 0;
#pragma unroll
        for (int k = GROUP - 1; k >= 0; --k) p = (p << 4) + c[k];
        w0 = p - bias * 0x11111111u;
        w1 = 0;
    } else if constexpr (BITS == 8) {
        uint32_t p0 = 0, p1 = 0;
#pragma unroll
        for (int k = 3; k >= 0; --k) {
            p0 = (p0 << 8) + c[k];
            p1 = (p1 << 8) + c[k + 4];
        }
        w0 = p0 - bias * 0x01010101u;
        w1 = p1 - bias * 0x01010101u;
    } else {
        uint32_t h0 = 0, h1 = 0; // four 6-bit codes each
#pragma unroll
        for (int k = 3; k >= 0; --k) {
            h0 = (h0 << 6) + c[k];
            h1 = (h1 << 6) + c[k + 4];
        }
        h0 = (h0 - bias * 0x41041u) & 0xffffffu;
        h1 = (h1 - bias * 0x41041u) & 0xffffffu;
        w0 = h0 | (h1 << 24);
        w1 = h1 >> 8;
    }
}

// Sum of the 8 codes of a packed group.
template <int BITS>
__device__ __forceinline__ int32_t code_sum(uint32_t w0, uint32_t w1)
{
    if constexpr (BITS == 4) {
        return (int32_t)__builtin_amdgcn_udot8(w0, 0x11111111u, 0u, false);
    } else if constexpr (BITS == 8) {
        return (int32_t)__builtin_amdgcn_udot4(w0, 0x01010101u, __builtin_amdgcn_udot4(w1, 0x01010101u, 0u, false), false);
    } else {
        const uint32_t h0 = w0 & 0xffffffu, h1 = (w0 >> 24) | (w1 << 8);
        const uint32_t f = (h0 & 0x3f03fu) + ((h0 >> 6) & 0x3f03fu) + (h1 & 0x3f03fu) + ((h1 >> 6) & 0x3f03fu);
        return (int32_t)((f & 0xfffu) + (f >> 12));
    }
}

// Packed codes of output group g into the row.
template <int BITS>
__device__ __forceinline__ void store_group(uint8_t *out_row, int g, uint32_t w0, uint32_t w1)
{
    if constexpr (BITS == 4) {
        reinterpret_cast<uint32_t *>(out_row)[g] = w0;
    } else if constexpr (BITS == 8) {
        reinterpret_cast<uint2 *>(out_row)[g] = make_uint2(w0, w1);
    } else { // 6 bytes, 2-byte aligned
        uint16_t *o16 = reinterpret_cast<uint16_t *>(out_row + (int64_t)g * 6);
        o16[0] = (uint16_t)w0;
        o16[1] = (uint16_t)(w0 >> 16);
        o16[2] = (uint16_t)w1;
    }
}

} // namespace qllm_detail

#endif
