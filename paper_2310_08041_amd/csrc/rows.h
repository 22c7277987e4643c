// Internal to libqllm: eight neighbouring elements of a row in memory, float32 or bfloat16, that may begin at any multiple of an
// element's size (global memory takes wide accesses at such addresses), and the rounding to bfloat16.
#ifndef QLLM_ROWS_H
#define QLLM_ROWS_H

#include <hip/hip_runtime.h>

#include <stdint.h>

namespace qllm_detail {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_at2 __attribute__((aligned(2)));
typedef u32x4 u32x4_at4 __attribute__((aligned(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef u32x2 u32x2_at2 __attribute__((aligned(2)));
typedef __bf16 bf16_pair __attribute__((ext_vector_type(2)));
typedef float f32_pair __attribute__((ext_vector_type(2)));

// two floats rounded to bfloat16, to nearest even, the first in the low half
__device__ __forceinline__ uint32_t to_bf16(float lo, float hi)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32_pair{lo, hi}, bf16_pair));
}

// Eight elements as they sit in memory; `n` of them are there (from 8 on: all), the others are not reached for and count as 0.
template <typename T>
struct Eight;
template <>
struct Eight<uint16_t> {
    u32x4 q;
    __device__ __forceinline__ void load(const uint16_t *p, int n)
    {
        if (n >= 8) {
            q = *reinterpret_cast<const u32x4_at2 *>(p);
        } else {
            q = u32x4{0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < 7; ++j)
                if (j < n) q[j / 2] |= (uint32_t)p[j] << (16 * (j & 1));
        }
    }
    __device__ __forceinline__ void widen(float *v) const
    {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            v[2 * k] = __uint_as_float(q[k] << 16);
            v[2 * k + 1] = __uint_as_float(q[k] & 0xffff0000u);
        }
    }
    __device__ __forceinline__ void round(const float *v)
    {
#pragma unroll
        for (int k = 0; k < 4; ++k) q[k] = to_bf16(v[2 * k], v[2 * k + 1]);
    }
    template <bool STREAM = false>
    __device__ __forceinline__ void store(uint16_t *p, int n) const
    {
        if (n >= 8) {
            if constexpr (STREAM) __builtin_nontemporal_store(q, reinterpret_cast<u32x4_at2 *>(p));
            else *reinterpret_cast<u32x4_at2 *>(p) = q;
        } else {
#pragma unroll
            for (int j = 0; j < 7; ++j)
                if (j < n) p[j] = (uint16_t)(q[j / 2] >> (16 * (j & 1)));
        }
    }
};
template <>
struct Eight<float> {
    u32x4 a, b;
    __device__ __forceinline__ void load(const float *p, int n)
    {
        if (n >= 8) {
            a = reinterpret_cast<const u32x4_at4 *>(p)[0];
            b = reinterpret_cast<const u32x4_at4 *>(p)[1];
        } else {
            a = b = u32x4{0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (j < n) a[j] = __float_as_uint(p[j]);
                if (j + 4 < n) b[j] = __float_as_uint(p[j + 4]);
            }
        }
    }
    __device__ __forceinline__ void widen(float *v) const
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = __uint_as_float(a[j]), v[j + 4] = __uint_as_float(b[j]);
    }
    __device__ __forceinline__ void round(const float *v)
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) a[j] = __float_as_uint(v[j]), b[j] = __float_as_uint(v[j + 4]);
    }
    template <bool STREAM = false>
    __device__ __forceinline__ void store(float *p, int n) const
    {
        if (n >= 8) {
            if constexpr (STREAM) {
                __builtin_nontemporal_store(a, reinterpret_cast<u32x4_at4 *>(p));
                __builtin_nontemporal_store(b, reinterpret_cast<u32x4_at4 *>(p) + 1);
            } else {
                reinterpret_cast<u32x4_at4 *>(p)[0] = a;
                reinterpret_cast<u32x4_at4 *>(p)[1] = b;
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (j < n) p[j] = __uint_as_float(a[j]);
                if (j + 4 < n) p[j + 4] = __uint_as_float(b[j]);
            }
        }
    }
};

} // namespace qllm_detail

#endif
