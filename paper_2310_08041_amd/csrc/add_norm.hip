// The residual's addition, the norm, the reassembly (Eq. 3, Eq. 4) and Eq. (2) in one pass over the rows.
//
// s = round(residual + x); y = norm(s), statistics in fp64; x^ = the map's combination of y; codes of x^ at 4, 6 or 8 bits.
// What it has to move is x, the residual, s and the codes (7 bytes a channel for bf16 and 8 bits): bound by memory, 4.8 TB/s of the 5.1 that
// a large copy reaches (4096 x 5120 bf16 to 8 bits 30.7 us; through a map 35, which is latency: staging, computed channels, places from L2).
//
// A workgroup has a row.  Its lanes hold 8 channels of it each, once to four times, from the loads to the codes: without a map
// nothing of the row goes through LDS.  With one y is staged there, channel c at place (c mod 8) S + c / 8 so that lanes which hold
// neighbouring chunks touch neighbouring words, whatever a map shifts them by; channels that are not copies are computed from it
// first and get places of their own behind it, and then every output channel is one read from the place that the map's index names.
//
// A row a workgroup and as many workgroups as there are rows: 50 to 64 registers leave eight waves a SIMD, whose rows are at different
// stages (workgroups that stay and keep gamma and the map take 100 registers and more and 42 to 66 us where these take 31 and 40).
//
// Compiled with -ffp-contract=off: every fp32 product and sum is rounded on its own, as qllm_norm_reassemble_quant rounds them.
#include <hip/hip_runtime.h>

#include <stdint.h>

#include "fused_common.h"
#include "lds_limit.h"
#include "pack_codes.h"
#include "qllm_block.h"
#include "rows.h"
#include "wave_reduce.h"

using namespace qllm_detail;

namespace {

constexpr int MOST_LANES = 1024;
constexpr int64_t MANY_CHUNKS = 3 << 16;
constexpr int64_t MOST_LAUNCHED = 1ll << 31; // lanes of a launch, which counts them in 32 bits; more rows take another

// see qllm_gather_map_host
struct alignas(16) Computed {
    uint32_t place01, place23;
    float scale[4];
    int32_t more, none;
};

struct AddNormArgs {
    const void *x, *residual;
    void *sum, *y, *values;
    int64_t ldx, ldr, lds, ldy, ldv;
    int64_t first; // row of the launch
    const float *gamma, *beta;
    int32_t N, C, norm, o_bf16;
    double eps, inv_C;
    const uint32_t *places; // of 8 output channels: 4 words
    const Computed *computed;
    const int2 *more;
    int32_t n_computed, S, K, groups; // groups of 8 codes in a row, padding included
    uint8_t *codes;
    int64_t row_bytes;
    float *alpha;
    int32_t *zero, *rowsum;
    int32_t bits;
};

// the codes of the live ones of 8 values into the row's group g (of the others: 0); returns their sum
template <int BITS>
__device__ __forceinline__ int32_t put_codes(uint8_t *row, int g, const float *v, uint32_t live, float inv, int32_t beta)
{
    uint32_t w0, w1;
    quant_pack<BITS>(v, live, 1, inv, beta, w0, w1);
    store_group<BITS>(row, g, w0, w1);
    return code_sum<BITS>(w0, w1);
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

__device__ __forceinline__ void put_out(void *to, int64_t at, bool bf16, float v)
{
    if (bf16) static_cast<uint16_t *>(to)[at] = (uint16_t)to_bf16(v, 0.0f);
    else static_cast<float *>(to)[at] = v;
}

// Over the workgroup's waves (16 at most): lane l of every wave takes the slot of wave l mod 16, and a butterfly adds them.
__device__ __forceinline__ double over_waves(double v, double *slots, int waves)
{
    v = wave_sum(v);
    if (waves == 1) return v;
    const int lane = threadIdx.x & 63;
    if (lane == 0) slots[threadIdx.x >> 6] = v;
    __syncthreads();
    return dpp_addd_row16((lane & 15) < waves ? slots[lane & 15] : 0.0);
}

// WHOLE: every chunk of 8 input channels is in the row as a whole or not at all.
template <typename XT, typename RT, int ITERS, bool MAPPED, bool WHOLE>
__global__ __launch_bounds__(MOST_LANES) void add_norm_kernel(const AddNormArgs a)
{
    extern __shared__ __align__(16) float places[]; // MAPPED: y by places, then the computed channels
    __shared__ double red_d[2][16];
    __shared__ float red_f[2][16];
    __shared__ uint32_t arrived; // waves << 24, and the sum of their codes
    const int THREADS = blockDim.x, WAVES = THREADS >> 6;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int64_t row = a.first + blockIdx.x;
    // elements of chunk `it` of the lane that are there, of a row of n and of the row that came
    auto left_of = [&](int it, int n) { return n - (tid + it * THREADS) * GROUP; };
    auto there = [&](int it) {
        const int left = left_of(it, a.C);
        return WHOLE ? (left > 0 ? GROUP : 0) : left;
    };

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
            re[it].load(r + c0, there(it));
            if (a.x) xe[it].load(x + c0, there(it));
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
                if (a.sum) re[it].template store<(ITERS > 1)>(static_cast<RT *>(a.sum) + row * a.lds + c0, there(it)); // not read soon: past the caches
                re[it].widen(v[it]);
            }
        }
    }

    // what depends on the map and on gamma alone is asked for while the statistics are on their way
    Eight<float> gamma[ITERS];
    uint4 place[MAPPED ? ITERS : 1];
    Computed computed = {}; // the first that falls to the lane
    if (a.norm != QLLM_NORM_NONE) {
#pragma unroll
        for (int it = 0; it < ITERS; ++it) {
            const int c0 = (tid + it * THREADS) * GROUP;
            gamma[it].load(a.gamma + c0, there(it));
        }
    }
    if constexpr (MAPPED) {
#pragma unroll
        for (int it = 0; it < ITERS; ++it) place[it] = reinterpret_cast<const uint4 *>(a.places)[min(tid + it * THREADS, a.groups - 1)];
        if (tid < a.n_computed) computed = a.computed[tid];
    }

    // ---- y = norm(s); elements past the row are 0 and stay out of the sums
    float mu = 0.0f, rstd = 1.0f;
    if (a.norm == QLLM_NORM_RMS) {
        double q[2] = {0.0, 0.0}; // two chains
#pragma unroll
        for (int it = 0; it < ITERS; ++it)
#pragma unroll
            for (int j = 0; j < GROUP; ++j) q[j & 1] = __builtin_fma((double)v[it][j], (double)v[it][j], q[j & 1]);
        rstd = rsqrt_to_f32(over_waves(q[0] + q[1], red_d[0], WAVES) * a.inv_C + a.eps);
    } else if (a.norm == QLLM_NORM_LAYER) {
        double s = 0.0, q = 0.0;
#pragma unroll
        for (int it = 0; it < ITERS; ++it)
#pragma unroll
            for (int j = 0; j < GROUP; ++j) s += (double)v[it][j];
        const double mean = over_waves(s, red_d[0], WAVES) * a.inv_C;
#pragma unroll
        for (int it = 0; it < ITERS; ++it)
#pragma unroll
            for (int j = 0; j < GROUP; ++j) asm volatile("" : "+v"(v[it][j])); // converted again rather than kept in 64 bits over the sum
#pragma unroll
        for (int it = 0; it < ITERS; ++it)
#pragma unroll
            for (int j = 0; j < GROUP; ++j) {
                const double d = (double)v[it][j] - mean;
                if (j < there(it)) q = __builtin_fma(d, d, q);
            }
        rstd = rsqrt_to_f32(over_waves(q, red_d[1], WAVES) * a.inv_C + a.eps);
        mu = (float)mean;
    }
#pragma unroll
    for (int it = 0; it < ITERS; ++it) {
        const int c0 = (tid + it * THREADS) * GROUP;
        if (a.norm != QLLM_NORM_NONE) {
            float g[GROUP];
            gamma[it].widen(g);
#pragma unroll
            for (int j = 0; j < GROUP; ++j) {
                if (a.norm == QLLM_NORM_LAYER) v[it][j] -= mu;
                v[it][j] = v[it][j] * rstd * g[j];
            }
            if (a.norm == QLLM_NORM_LAYER && a.beta) {
                Eight<float> e;
                e.load(a.beta + c0, there(it));
                e.widen(g);
#pragma unroll
                for (int j = 0; j < GROUP; ++j) v[it][j] += g[j];
            }
        }
        if (a.y) store_out(a.y, row * a.ldy + c0, a.o_bf16, v[it], there(it));
        if constexpr (MAPPED) {
            if (c0 < a.C)
#pragma unroll
                for (int j = 0; j < GROUP; ++j) places[j * a.S + tid + it * THREADS] = v[it][j];
        }
    }
    if (!a.codes) return;

    // ---- x^: computed channels by lanes of their own, and one read for every channel.  What is read in the place of a computed channel
    // here is a NaN, which the minimum and the maximum pass over, or its value already: that lane brings it into them.
    float mn = __builtin_inff(), mx = -__builtin_inff();
    auto gather = [&]() {
#pragma unroll
        for (int it = 0; it < ITERS; ++it) {
            const uint32_t w[4] = {place[it].x, place[it].y, place[it].z, place[it].w};
#pragma unroll
            for (int j = 0; j < GROUP; ++j)
                v[it][j] = __hip_atomic_load(&places[j & 1 ? w[j / 2] >> 16 : w[j / 2] & 0xffffu], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
        }
    };
    if constexpr (MAPPED) {
        for (int j = tid; j < a.n_computed; j += THREADS) places[GROUP * a.S + j] = __builtin_nanf("");
        __syncthreads();
        for (int j = tid; j < a.n_computed; j += THREADS) {
            if (j != tid) computed = a.computed[j];
            float sum = computed.scale[0] * places[computed.place01 & 0xffffu];
            sum = sum + computed.scale[1] * places[computed.place01 >> 16];
            if (computed.more) { // entries beyond the second
                sum = sum + computed.scale[2] * places[computed.place23 & 0xffffu];
                sum = sum + computed.scale[3] * places[computed.place23 >> 16];
                if (computed.more > 1) { // beyond the fourth
                    const int2 *more = a.more + computed.more;
                    const int count = more[0].x;
                    for (int k = 1; k <= count; ++k) sum = sum + __int_as_float(more[k].y) * places[more[k].x];
                }
            }
            __hip_atomic_store(&places[GROUP * a.S + j], sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
            mn = fminf(mn, sum), mx = fmaxf(mx, sum);
        }
        gather();
    }

    // ---- Eq. (2)
#pragma unroll
    for (int it = 0; it < ITERS; ++it) {
        const int n = left_of(it, a.K);
        if (n >= GROUP) {
#pragma unroll
            for (int j = 0; j < GROUP; j += 2) { // three operands an instruction
                mn = fminf(fminf(mn, v[it][j]), v[it][j + 1]);
                mx = fmaxf(fmaxf(mx, v[it][j]), v[it][j + 1]);
            }
        } else if (n > 0) {
#pragma unroll
            for (int j = 0; j < GROUP - 1; ++j)
                if (j < n) mn = fminf(mn, v[it][j]), mx = fmaxf(mx, v[it][j]);
        }
    }
    wave_minmax(mn, mx);
    if (WAVES > 1) {
        if (lane == 0) red_f[0][wave] = mn, red_f[1][wave] = mx;
        if (tid == 0) arrived = 0;
        __syncthreads();
        const int w = min(lane & 15, WAVES - 1);
        mn = dpp_min_row16(red_f[0][w]), mx = dpp_max_row16(red_f[1][w]);
    }
    if constexpr (MAPPED) {
        // The computed channels' values are there now.  A wave alone has had no barrier: its LDS operations are done in their order, which
        // the fence keeps the compiler to without an instruction.
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        gather();
    }
    const int32_t qmax = (1 << a.bits) - 1;
    const float range = mx - mn, alpha = range > 0.0f ? range / (float)qmax : 1.0f, inv = 1.0f / alpha;
    const bool fast = fabsf(mn * inv) < FAST_LIMIT && fabsf(mx * inv) < FAST_LIMIT;
    int32_t beta;
    if (fast) beta = -rne_product_fast(mn, inv);
    else beta = (int32_t)fmin(fmax(-rne_product_slow(mn, inv), -2147483647.0), 2147483647.0);
    uint8_t *to = a.codes + row * a.row_bytes;
    int32_t sum = 0;
#pragma unroll
    for (int it = 0; it < ITERS; ++it) {
        const int g = tid + it * THREADS, n = left_of(it, a.K);
        if (g >= a.groups) continue;
        const uint32_t live = n >= GROUP ? 0xffu : n > 0 ? (1u << n) - 1u : 0u;
        float inv_of = inv;
        int32_t beta_of = beta;
        if (!fast) { // rare: the codes one by one, to be packed as values that are codes already
#pragma unroll
            for (int j = 0; j < GROUP; ++j) {
                const uint32_t code = slow_code(v[it][j], inv, beta, qmax);
                if (a.values && j < n) put_out(a.values, row * a.ldv + (int64_t)g * GROUP + j, a.o_bf16, (float)((double)alpha * ((double)code - (double)beta)));
                v[it][j] = (float)code;
            }
            inv_of = 1.0f, beta_of = 0;
        } else if (a.values) {
            // a code is clamped as a float in [2^23, 2^24); what is left of it without 1.5 * 2^23 is code - beta
            const float lowest = __int_as_float(MAGIC_BITS - beta), highest = __int_as_float(MAGIC_BITS - beta + qmax);
            float stands[GROUP];
#pragma unroll
            for (int j = 0; j < GROUP; ++j) stands[j] = alpha * (__builtin_amdgcn_fmed3f(__builtin_fmaf(v[it][j], inv, MAGIC), lowest, highest) - MAGIC);
            store_out(a.values, row * a.ldv + (int64_t)g * GROUP, a.o_bf16, stands, n);
        }
        if (a.bits == 8) sum += put_codes<8>(to, g, v[it], live, inv_of, beta_of);
        else if (a.bits == 4) sum += put_codes<4>(to, g, v[it], live, inv_of, beta_of);
        else sum += put_codes<6>(to, g, v[it], live, inv_of, beta_of);
    }
    sum = wave_sum_i32(sum);
    if (lane == 0) {
        // the wave that comes last has the row's sum: no barrier for it (below 2^23: 32768 codes of 8 bits)
        const uint32_t before = WAVES > 1 ? atomicAdd(&arrived, (1u << 24) + (uint32_t)sum) : 0u;
        if (before >> 24 == (uint32_t)(WAVES - 1)) a.rowsum[row] = (int32_t)((before + (uint32_t)sum) & 0xffffffu);
    }
    if (tid == 0) a.alpha[row] = alpha, a.zero[row] = beta;
}

template <typename XT, typename RT, int ITERS, bool MAPPED>
int32_t launch(AddNormArgs a, int units, hipStream_t stream)
{
    auto *kernel = a.C % GROUP == 0 ? add_norm_kernel<XT, RT, ITERS, MAPPED, true> : add_norm_kernel<XT, RT, ITERS, MAPPED, false>;
    const size_t lds = MAPPED ? (size_t)(GROUP * a.S + a.n_computed) * sizeof(float) : 0;
    if (lds > 48 * 1024) {
        const int32_t e = raise_lds_limit(reinterpret_cast<const void *>(kernel), QLLM_GATHER_PLACES * (int)sizeof(float), "add_norm: raising the LDS limit");
        if (e != QLLM_OK) return e;
    }
    const int lanes = (units + ITERS * 64 - 1) / (ITERS * 64) * 64;
    (void)hipGetLastError(); // drop any stale error of the calling thread: only this launch is judged
    for (const int64_t most = MOST_LAUNCHED / lanes; a.first < a.N; a.first += most) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)(a.N - a.first < most ? a.N - a.first : most)), dim3(lanes), lds, stream, a);
        const hipError_t e = hipGetLastError();
        if (e == hipSuccess) continue;
        qllm_note_hip_error("add_norm: launch", hipGetErrorName(e));
        return QLLM_ERR_HIP;
    }
    return QLLM_OK;
}

template <typename XT, typename RT, bool MAPPED>
int32_t by_width(const AddNormArgs &a, hipStream_t stream)
{
    const int units = a.S > a.groups ? a.S : a.groups; // chunks of 8 channels, in or out
    // One chunk a lane is the shorter way through a row of few others, two keep more of it in flight and share what a wave does per row:
    // us, one : two, bf16 to 8 bits, rows of 2048 channels 512 4.8 : 5.1, 768 5.6 : 5.2; of 4096 256 4.7 : 4.9, 512 6.2 : 5.7, 1024 10.2 : 8.6;
    // of 8192 16 5.2 : 4.9 (sixteen waves are too many), 2048 36 : 31.  Four (5120 channels 32.0 : 30.6 with two) only where a row needs it.
    if (units <= 512 && (units <= 64 || a.N * (int64_t)units < MANY_CHUNKS)) return launch<XT, RT, 1, MAPPED>(a, units, stream);
    if (units <= 2 * MOST_LANES) return launch<XT, RT, 2, MAPPED>(a, units, stream);
    return launch<XT, RT, 4, MAPPED>(a, units, stream);
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
            a.computed = reinterpret_cast<const Computed *>(gather->index + padded / 2);
            a.more = reinterpret_cast<const int2 *>(gather->index + padded / 2 + 8 * gather->n_computed);
            a.n_computed = (int32_t)gather->n_computed;
        }
    }
    hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
    if (!x || x_dtype == r_dtype) return r_dtype == QLLM_BF16 ? by_map<uint16_t, uint16_t>(a, stream) : by_map<float, float>(a, stream);
    return r_dtype == QLLM_BF16 ? by_map<float, uint16_t>(a, stream) : by_map<uint16_t, float>(a, stream);
}
