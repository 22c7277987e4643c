// Internal to libqllm: sums, minima and maxima over a wavefront, and the norms' reciprocal square root.
#ifndef QLLM_WAVE_REDUCE_H
#define QLLM_WAVE_REDUCE_H

#include <hip/hip_runtime.h>

#include <stdint.h>

namespace qllm_detail {

// (float)(1 / sqrt(t)) for t > 0: the hardware's reciprocal-square-root estimate refined by two Newton
// steps in fp64 (relative error of a few 1e-16), then rounded to fp32.  It equals the fp32 rounding of
// the exact value unless that lies within ~1e-16 (relative) of a rounding boundary of fp32.
__device__ __forceinline__ float rsqrt_to_f32(double t)
{
    double r = __builtin_amdgcn_rsq(t);
    const double h = 0.5 * t;
#pragma unroll
    for (int n = 0; n < 2; ++n) {
        const double e = __builtin_fma(-(h * r), r, 0.5);
        r = __builtin_fma(r, e, r);
    }
    return (float)r;
}

// ---- wavefront reductions on the data-parallel-primitive (DPP) path: no LDS round trips.
// Four butterfly steps inside each row of 16 lanes, then the four row results are combined from
// lanes 0, 16, 32, 48.  The order of the additions is fixed, so the result is reproducible.
// Each step is ONE instruction that takes its first operand from another lane.  They are written
// out because the optimiser, given the lane movement as a builtin, spends four instructions a step
// (a zeroed destination, the move, a NaN-quieting pass, the operation).  Every lane of the wavefront
// must be active; the s_nop covers the two wait states a DPP operand needs after it was written.
#define QLLM_DPP_STEP(fn, type, cons, op, ctrl)                                                          \
    __device__ __forceinline__ type fn(type v)                                                           \
    {                                                                                                    \
        type r;                                                                                          \
        asm("s_nop 1\n\t" op " %0, %1, %1 " ctrl " row_mask:0xf bank_mask:0xf" : "=" cons(r) : cons(v)); \
        return r;                                                                                        \
    }
#define QLLM_DPP_FAMILY(name, type, op)                                  \
    QLLM_DPP_STEP(name##_xor1, type, "v", op, "quad_perm:[1,0,3,2]")     \
    QLLM_DPP_STEP(name##_xor2, type, "v", op, "quad_perm:[2,3,0,1]")     \
    QLLM_DPP_STEP(name##_half_mirror, type, "v", op, "row_half_mirror")  \
    QLLM_DPP_STEP(name##_mirror, type, "v", op, "row_mirror")            \
    __device__ __forceinline__ type name##_row16(type v) /* all 16 lanes of a row end with the row's result */ \
    {                                                                    \
        return name##_mirror(name##_half_mirror(name##_xor2(name##_xor1(v)))); \
    }
QLLM_DPP_FAMILY(dpp_min, float, "v_min_f32_dpp")
QLLM_DPP_FAMILY(dpp_max, float, "v_max_f32_dpp")
QLLM_DPP_FAMILY(dpp_add, int32_t, "v_add_u32_dpp")

// v + (v of the partner lane) in fp64: the two halves move separately, the addition is ordinary
#define QLLM_DPP_ADD_F64(fn, ctrl)                                                                           \
    __device__ __forceinline__ double fn(double v)                                                           \
    {                                                                                                        \
        const uint64_t u = __double_as_longlong(v);                                                          \
        uint32_t lo, hi;                                                                                     \
        asm("s_nop 1\n\tv_mov_b32_dpp %0, %2 " ctrl " row_mask:0xf bank_mask:0xf\n\t"                        \
            "v_mov_b32_dpp %1, %3 " ctrl " row_mask:0xf bank_mask:0xf"                                       \
            : "=&v"(lo), "=&v"(hi)                                                                           \
            : "v"((uint32_t)u), "v"((uint32_t)(u >> 32)));                                                   \
        return v + __longlong_as_double((long long)((uint64_t)lo | ((uint64_t)hi << 32)));                   \
    }
QLLM_DPP_ADD_F64(dpp_addd_xor1, "quad_perm:[1,0,3,2]")
QLLM_DPP_ADD_F64(dpp_addd_xor2, "quad_perm:[2,3,0,1]")
QLLM_DPP_ADD_F64(dpp_addd_half_mirror, "row_half_mirror")
QLLM_DPP_ADD_F64(dpp_addd_mirror, "row_mirror")
__device__ __forceinline__ double dpp_addd_row16(double v)
{
    return dpp_addd_mirror(dpp_addd_half_mirror(dpp_addd_xor2(dpp_addd_xor1(v))));
}

__device__ __forceinline__ float lane_f32(float v, int l)
{
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), l));
}
__device__ __forceinline__ double lane_f64(double v, int l)
{
    const uint64_t u = __double_as_longlong(v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)u, l);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(u >> 32), l);
    return __longlong_as_double((long long)((uint64_t)lo | ((uint64_t)hi << 32)));
}

__device__ __forceinline__ double wave_sum(double v)
{
    v = dpp_addd_row16(v);
    return (lane_f64(v, 0) + lane_f64(v, 16)) + (lane_f64(v, 32) + lane_f64(v, 48));
}
__device__ __forceinline__ void wave_minmax(float &mn, float &mx)
{
    mn = dpp_min_row16(mn);
    mx = dpp_max_row16(mx);
    mn = fminf(fminf(lane_f32(mn, 0), lane_f32(mn, 16)), fminf(lane_f32(mn, 32), lane_f32(mn, 48)));
    mx = fmaxf(fmaxf(lane_f32(mx, 0), lane_f32(mx, 16)), fmaxf(lane_f32(mx, 32), lane_f32(mx, 48)));
}
__device__ __forceinline__ int32_t wave_sum_i32(int32_t v)
{
    v = dpp_add_row16(v);
    return __builtin_amdgcn_readlane(v, 0) + __builtin_amdgcn_readlane(v, 16) + __builtin_amdgcn_readlane(v, 32) +
           __builtin_amdgcn_readlane(v, 48);
}

// Sum of the 16 per-wave slots (zero where there is no wave): lane w of every row of 16 lanes fetches
// slot w and a butterfly adds them, so every lane ends with the same total without a dependent chain
// of LDS reads.  The slots are not reused before another barrier has passed.
__device__ __forceinline__ double total16(const double *slots, int lane)
{
    return dpp_addd_row16(slots[lane & 15]);
}

} // namespace qllm_detail

#endif
