// The residual's addition, the norm, the reassembly (Eq. 3, Eq. 4) and Eq. (2) in one pass over the rows.
//
// s = round(residual + x); y = norm(s), statistics in fp64; x^ = the map's combination of y; codes of x^ at 4, 6 or 8 bits.
// What it has to move is x, the residual, s and the codes (7 bytes a channel for bf16 and 8 bits): bound by memory.
//
// A workgroup has a row.  Its lanes hold 8 channels of it each, once to four times, from the loads to the codes: without a map
// nothing of the row goes through LDS.  With one y is staged there, channel c at place (c mod 8) S + c / 8 so that lanes which hold
// neighbouring chunks touch neighbouring words, whatever a map shifts them by; channels that are not copies are computed from it
// first and get places of their own behind it, and then every output channel is one read from the place that the map's index names.
//
// Compiled with -ffp-contract=off: every fp32 product and sum is rounded on its own, as qllm_norm_reassemble_quant rounds them.
#include <hip/hip_runtime.h>

#include <stdint.h>

#include "fused_common.h"
#include "qllm_block.h"
#include "rows.h"
#include "wave_reduce.h"

using namespace qllm_detail;

namespace {

struct AddNormArgs {
    const void *x, *residual;
    void *sum, *y, *values;
    int64_t ldx, ldr, lds, ldy, ldv;
    const float *gamma, *beta;
    int32_t N, C, norm, o_bf16;
    double eps, inv_C;
    const uint32_t *places; // of 8 output channels: 4 words
    const int32_t *first;
    const int2 *entries;
    int32_t n_computed, S, K, groups; // groups of 8 codes in a row, padding included
    uint8_t *codes;
    int64_t row_bytes;
    float *alpha;
    int32_t *zero, *rowsum;
    int32_t bits;
};

// the 8 codes of a group, one byte each, to the row's packed bytes
__device__ __forceinline__ void store_codes(uint8_t *row, int g, int bits, const uint32_t *c)
{
    if (bits == 8) {
        reinterpret_cast<uint2 *>(row)[g] = make_uint2(c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24, c[4] | c[5] << 8 | c[6] << 16 | c[7] << 24);
    } else if (bits == 4) {
        reinterpret_cast<uint32_t *>(row)[g] = c[0] | c[1] << 4 | c[2] << 8 | c[3] << 12 | c[4] << 16 | c[5] << 20 | c[6] << 24 | c[7] << 28;
    } else {
        const uint32_t lo = c[0] | c[1] << 6 | c[2] << 12 | c[3] << 18, hi = c[4] | c[5] << 6 | c[6] << 12 | c[7] << 18;
        uint16_t *to = reinterpret_cast<uint16_t *>(row + (int64_t)g * 6);
        to[0] = (uint16_t)lo;
        to[1] = (uint16_t)(lo >> 16 | hi << 8);
        to[2] = (uint16_t)(hi >> 8);
    }
}

__device__ __forceinline__ void store_out(void *to, int64_t at, bool bf16, const float *v, int n)
{
    if (bf16) {
        Eight<uint16_t> e;
        e.round(v);
        e.store(static_cast<uint16_t *>(to) + at, n);
    } else {
        Eight<float> e;
        e.round(v);
        e.store(static_cast<float *>(to) + at, n);
    }
}

template <int WAVES>
__device__ __forceinline__ double over_waves(double v, double *slots)
{
    v = wave_sum(v);
    if constexpr (WAVES == 1) return v;
    if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = v;
    __syncthreads();
    v = slots[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) v += slots[w];
    return v;
}

template <typename XT, typename RT, int THREADS, int ITERS, bool MAPPED>
__global__ __launch_bounds__(THREADS) void add_norm_kernel(const AddNormArgs a)
{
    constexpr int WAVES = THREADS / 64;
    extern __shared__ __align__(16) float places[]; // MAPPED: y by places, then the computed channels
    __shared__ double red_d[2][WAVES];
    __shared__ float red_f[2][WAVES];
    __shared__ int32_t red_i[WAVES];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int64_t row = blockIdx.x;

    // ---- s = round(residual + x)
    float v[ITERS][GROUP];
    {
        Eight<XT> xe[ITERS];
        Eight<RT> re[ITERS];
        const XT *x = static_cast<const XT *>(a.x) + row * a.ldx;
        const RT *r = static_cast<const RT *>(a.residual) + row * a.ldr;
#pragma unroll
        for (int it = 0; it < ITERS; ++it) {
            const int c0 = (tid + it * THREADS) * GROUP;
            re[it].load(r + c0, a.C - c0);
            if (a.x) xe[it].load(x + c0, a.C - c0);
        }
#pragma unroll
        for (int it = 0; it < ITERS; ++it) {
            const int c0 = (tid + it * THREADS) * GROUP;
            re[it].widen(v[it]);
            if (a.x) {
                float u[GROUP];
                xe[it].widen(u);
#pragma unroll
                for (int j = 0; j < GROUP; ++j) v[it][j] += u[j];
                re[it].round(v[it]);
                if (a.sum) re[it].store(static_cast<RT *>(a.sum) + row * a.lds + c0, a.C - c0);
                re[it].widen(v[it]);
            }
        }
    }

    // ---- y = norm(s); elements past the row are 0 and stay out of the sums
    float mu = 0.0f, rstd = 1.0f;
    if (a.norm == QLLM_NORM_RMS) {
        double q = 0.0;
#pragma unroll
        for (int it = 0; it < ITERS; ++it)
#pragma unroll
            for (int j = 0; j < GROUP; ++j) q = __builtin_fma((double)v[it][j], (double)v[it][j], q);
        rstd = rsqrt_to_f32(over_waves<WAVES>(q, red_d[0]) * a.inv_C + a.eps);
    } else if (a.norm == QLLM_NORM_LAYER) {
        double s = 0.0, q = 0.0;
#pragma unroll
        for (int it = 0; it < ITERS; ++it)
#pragma unroll
            for (int j = 0; j < GROUP; ++j) s += (double)v[it][j];
        const double mean = over_waves<WAVES>(s, red_d[0]) * a.inv_C;
#pragma unroll
        for (int it = 0; it < ITERS; ++it)
#pragma unroll
            for (int j = 0; j < GROUP; ++j) {
                const double d = (double)v[it][j] - mean;
                if ((tid + it * THREADS) * GROUP + j < a.C) q = __builtin_fma(d, d, q);
            }
        rstd = rsqrt_to_f32(over_waves<WAVES>(q, red_d[1]) * a.inv_C + a.eps);
        mu = (float)mean;
    }
#pragma unroll
    for (int it = 0; it < ITERS; ++it) {
        const int c0 = (tid + it * THREADS) * GROUP;
        if (a.norm != QLLM_NORM_NONE) {
            Eight<float> e;
            float g[GROUP];
            e.load(a.gamma + c0, a.C - c0);
            e.widen(g);
#pragma unroll
            for (int j = 0; j < GROUP; ++j) {
                if (a.norm == QLLM_NORM_LAYER) v[it][j] -= mu;
                v[it][j] = v[it][j] * rstd * g[j];
            }
            if (a.norm == QLLM_NORM_LAYER && a.beta) {
                e.load(a.beta + c0, a.C - c0);
                e.widen(g);
#pragma unroll
                for (int j = 0; j < GROUP; ++j) v[it][j] += g[j];
            }
        }
        if (a.y) store_out(a.y, row * a.ldy + c0, a.o_bf16, v[it], a.C - c0);
        if constexpr (MAPPED) {
            if (c0 < a.C)
#pragma unroll
                for (int j = 0; j < GROUP; ++j) places[j * a.S + tid + it * THREADS] = v[it][j];
        }
    }
    if (!a.codes) return;

    // ---- x^: computed channels first, then one read for every channel
    if constexpr (MAPPED) {
        __syncthreads();
        for (int j = tid; j < a.n_computed; j += THREADS) {
            const int32_t e0 = a.first[j], e1 = a.first[j + 1];
            int2 e = a.entries[e0];
            float sum = __int_as_float(e.y) * places[e.x];
            for (int k = e0 + 1; k < e1; ++k) {
                e = a.entries[k];
                sum = sum + __int_as_float(e.y) * places[e.x];
            }
            places[GROUP * a.S + j] = sum;
        }
        __syncthreads();
#pragma unroll
        for (int it = 0; it < ITERS; ++it) {
            const int g = tid + it * THREADS;
            if (g < a.groups) {
                const uint4 p = reinterpret_cast<const uint4 *>(a.places)[g];
                const uint32_t w[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
                for (int j = 0; j < GROUP; ++j) v[it][j] = places[j & 1 ? w[j / 2] >> 16 : w[j / 2] & 0xffffu];
            }
        }
    }

    // ---- Eq. (2)
    float mn = __builtin_inff(), mx = -__builtin_inff();
#pragma unroll
    for (int it = 0; it < ITERS; ++it)
#pragma unroll
        for (int j = 0; j < GROUP; ++j)
            if ((tid + it * THREADS) * GROUP + j < a.K) {
                mn = fminf(mn, v[it][j]);
                mx = fmaxf(mx, v[it][j]);
            }
    wave_minmax(mn, mx);
    if constexpr (WAVES > 1) {
        if (lane == 0) red_f[0][wave] = mn, red_f[1][wave] = mx;
        __syncthreads();
        mn = red_f[0][0], mx = red_f[1][0];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) mn = fminf(mn, red_f[0][w]), mx = fmaxf(mx, red_f[1][w]);
    }
    const int32_t qmax = (1 << a.bits) - 1;
    const float range = mx - mn, alpha = range > 0.0f ? range / (float)qmax : 1.0f, inv = 1.0f / alpha;
    const bool fast = fabsf(mn * inv) < FAST_LIMIT && fabsf(mx * inv) < FAST_LIMIT;
    int32_t beta;
    if (fast) beta = -rne_product_fast(mn, inv);
    else beta = (int32_t)fmin(fmax(-rne_product_slow(mn, inv), -2147483647.0), 2147483647.0);
    // floats in [2^23, 2^24) are integers and order like their bit patterns: a code is clamped as such a float
    const float lowest = __int_as_float(MAGIC_BITS - beta), highest = __int_as_float(MAGIC_BITS - beta + qmax);
    uint8_t *to = a.codes + row * a.row_bytes;
    int32_t sum = 0;
#pragma unroll
    for (int it = 0; it < ITERS; ++it) {
        const int g = tid + it * THREADS;
        if (g >= a.groups) continue;
        uint32_t c[GROUP];
        float stands[GROUP];
#pragma unroll
        for (int j = 0; j < GROUP; ++j) {
            if (fast) {
                c[j] = __float_as_uint(__builtin_amdgcn_fmed3f(__builtin_fmaf(v[it][j], inv, MAGIC), lowest, highest)) - (uint32_t)(MAGIC_BITS - beta);
                stands[j] = alpha * (float)((int32_t)c[j] - beta);
            } else {
                const double q = fmin(fmax(rne_product_slow(v[it][j], inv) + (double)beta, 0.0), (double)qmax);
                c[j] = (uint32_t)q;
                stands[j] = (float)((double)alpha * (q - (double)beta));
            }
            if (g * GROUP + j >= a.K) c[j] = 0;
            sum += (int32_t)c[j];
        }
        store_codes(to, g, a.bits, c);
        if (a.values) store_out(a.values, row * a.ldv + (int64_t)g * GROUP, a.o_bf16, stands, a.K - g * GROUP);
    }
    sum = wave_sum_i32(sum);
    if constexpr (WAVES > 1) {
        if (lane == 0) red_i[wave] = sum;
        __syncthreads();
    }
    if (tid == 0) {
        if constexpr (WAVES > 1)
            for (int w = 1; w < WAVES; ++w) sum += red_i[w];
        a.alpha[row] = alpha;
        a.zero[row] = beta;
        a.rowsum[row] = sum;
    }
}

template <typename XT, typename RT, int THREADS, int ITERS, bool MAPPED>
int32_t launch(const AddNormArgs &a, hipStream_t stream)
{
    auto *kernel = add_norm_kernel<XT, RT, THREADS, ITERS, MAPPED>;
    const size_t lds = MAPPED ? (size_t)(GROUP * a.S + a.n_computed) * sizeof(float) : 0;
    if (lds > 48 * 1024) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) {
            (void)hipGetLastError();
            qllm_note_hip_error("add_norm: raising the LDS limit", hipGetErrorName(e));
            return QLLM_ERR_HIP;
        }
    }
    (void)hipGetLastError(); // drop any stale error of the calling thread: only this launch is judged
    hipLaunchKernelGGL(kernel, dim3((unsigned)a.N), dim3(THREADS), lds, stream, a);
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return QLLM_OK;
    qllm_note_hip_error("add_norm: launch", hipGetErrorName(e));
    return QLLM_ERR_HIP;
}

template <typename XT, typename RT, bool MAPPED>
int32_t by_width(const AddNormArgs &a, hipStream_t stream)
{
    const int units = a.S > a.groups ? a.S : a.groups; // chunks of 8 channels, in or out
    if (units <= 64) return launch<XT, RT, 64, 1, MAPPED>(a, stream);
    if (units <= 256) return launch<XT, RT, 256, 1, MAPPED>(a, stream);
    if (units <= 512) return launch<XT, RT, 512, 1, MAPPED>(a, stream);
    if (units <= 1024) return launch<XT, RT, 1024, 1, MAPPED>(a, stream);
    if (units <= 2048) return launch<XT, RT, 1024, 2, MAPPED>(a, stream);
    return launch<XT, RT, 1024, 4, MAPPED>(a, stream);
}

template <typename XT, typename RT>
int32_t by_map(const AddNormArgs &a, hipStream_t stream)
{
    return a.places ? by_width<XT, RT, true>(a, stream) : by_width<XT, RT, false>(a, stream);
}

bool misses(const void *p, int64_t to) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(to - 1)) != 0; }
int64_t size_of(int32_t dtype) { return dtype == QLLM_BF16 ? 2 : 4; }

} // namespace

extern "C" int32_t qllm_add_norm_quant(const void *x, int32_t x_dtype, int64_t ldx, const void *residual, int32_t r_dtype, int64_t ldr,
                                       int64_t N, int64_t C, void *sum_out, int64_t lds, int32_t norm, const float *gamma,
                                       const float *beta, float eps, const qllm_gather *gather, int32_t bits, const qllm_qact *out,
                                       void *y_out, int64_t ldy, void *values_out, int64_t ldv, int32_t o_dtype, void *hip_stream)
{
    if (!residual) return QLLM_ERR_NULL;
    for (int32_t d : {x ? x_dtype : QLLM_F32, r_dtype, y_out || values_out ? o_dtype : QLLM_F32})
        if (d != QLLM_F32 && d != QLLM_BF16) return QLLM_ERR_DTYPE;
    if (norm != QLLM_NORM_NONE && norm != QLLM_NORM_LAYER && norm != QLLM_NORM_RMS) return QLLM_ERR_DTYPE;
    if (norm != QLLM_NORM_NONE && !gamma) return QLLM_ERR_NULL;
    if (N < 0 || N > INT32_MAX || C <= 0 || C > QLLM_MAX_CHANNELS || ldr < C || (x && ldx < C) || (x && sum_out && lds < C) || (y_out && ldy < C))
        return QLLM_ERR_SHAPE;
    if (x && sum_out && ((sum_out == residual && lds != ldr) || (sum_out == x && (lds != ldx || x_dtype != r_dtype)))) return QLLM_ERR_SHAPE;
    if (values_out && !out) return QLLM_ERR_NULL;
    int64_t K = C;
    if (out) {
        if (!out->codes || !out->scale || !out->zero || !out->rowsum) return QLLM_ERR_NULL;
        if (bits != 4 && bits != 6 && bits != 8) return QLLM_ERR_BITS;
        if (gather) {
            if (!gather->index) return QLLM_ERR_NULL;
            K = gather->C_out;
            if (gather->C_in != C || K <= 0 || K > QLLM_MAX_CHANNELS || gather->n_computed < 0 || gather->n_computed > K ||
                GROUP * ((C + GROUP - 1) / GROUP) + gather->n_computed > QLLM_GATHER_PLACES)
                return QLLM_ERR_SHAPE;
            if (misses(gather->index, 16)) return QLLM_ERR_ALIGN;
        }
        if (values_out && ldv < K) return QLLM_ERR_SHAPE;
        if (misses(out->codes, 16) || misses(out->scale, 4) || misses(out->zero, 4) || misses(out->rowsum, 4)) return QLLM_ERR_ALIGN;
    }
    if ((x && misses(x, size_of(x_dtype))) || misses(residual, size_of(r_dtype)) || (x && misses(sum_out, size_of(r_dtype))) ||
        misses(gamma, 4) || misses(beta, 4) || ((y_out || values_out) && (misses(y_out, size_of(o_dtype)) || misses(values_out, size_of(o_dtype)))))
        return QLLM_ERR_ALIGN;
    if (N == 0) return QLLM_OK;

    AddNormArgs a{};
    a.x = x, a.residual = residual, a.sum = x ? sum_out : nullptr, a.y = y_out, a.values = values_out;
    a.ldx = ldx, a.ldr = ldr, a.lds = lds, a.ldy = ldy, a.ldv = ldv;
    a.gamma = gamma, a.beta = beta, a.eps = (double)eps, a.inv_C = 1.0 / (double)C;
    a.N = (int32_t)N, a.C = (int32_t)C, a.norm = norm, a.o_bf16 = o_dtype == QLLM_BF16;
    a.S = (int32_t)((C + GROUP - 1) / GROUP), a.K = (int32_t)K;
    if (out) {
        const int64_t padded = (K + QLLM_K_PAD - 1) / QLLM_K_PAD * QLLM_K_PAD;
        a.groups = (int32_t)(padded / GROUP);
        a.codes = out->codes, a.row_bytes = qllm_packed_row_bytes(K, bits), a.alpha = out->scale, a.zero = out->zero, a.rowsum = out->rowsum;
        a.bits = bits;
        if (gather) {
            a.places = reinterpret_cast<const uint32_t *>(gather->index);
            a.first = gather->index + padded / 2;
            a.entries = reinterpret_cast<const int2 *>(a.first + (gather->n_computed + 2) / 2 * 2);
            a.n_computed = (int32_t)gather->n_computed;
        }
    }
    hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
    if (!x || x_dtype == r_dtype) return r_dtype == QLLM_BF16 ? by_map<uint16_t, uint16_t>(a, stream) : by_map<float, float>(a, stream);
    return r_dtype == QLLM_BF16 ? by_map<float, uint16_t>(a, stream) : by_map<uint16_t, float>(a, stream);
}
