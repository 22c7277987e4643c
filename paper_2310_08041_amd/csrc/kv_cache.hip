// Filling the 4-bit key/value cache (rotary positions, Eq. (2) per token and head), reading it back, copying pages.
#include <hip/hip_runtime.h>

#include <stdint.h>

#include <new>

#include "fused_common.h"
#include "kv_common.h"

namespace {

using namespace qllm_kv_detail;
using qllm_detail::FAST_LIMIT;

constexpr int THREADS = 256;
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}

// Eight neighbouring values of a row as they lie in memory (bf16: one 16-byte word, fp32: two); vec: they are 16-byte aligned.
template <bool F32>
struct Raw {
    uint4 w[F32 ? 2 : 1];
};
template <bool F32>
__device__ __forceinline__ Raw<F32> load8(const void *base, int64_t at, bool vec)
{
    Raw<F32> r;
    if (vec) {
        const uint4 *p = reinterpret_cast<const uint4 *>(static_cast<const uint8_t *>(base) + at * (F32 ? 4 : 2));
#pragma unroll
        for (int i = 0; i < (F32 ? 2 : 1); ++i) r.w[i] = p[i];
    } else if (F32) {
        const uint32_t *p = static_cast<const uint32_t *>(base) + at;
#pragma unroll
        for (int i = 0; i < (F32 ? 2 : 1); ++i) r.w[i] = make_uint4(p[4 * i], p[4 * i + 1], p[4 * i + 2], p[4 * i + 3]);
    } else {
        const uint16_t *p = static_cast<const uint16_t *>(base) + at;
        r.w[0] = make_uint4(p[0] | (uint32_t)p[1] << 16, p[2] | (uint32_t)p[3] << 16, p[4] | (uint32_t)p[5] << 16, p[6] | (uint32_t)p[7] << 16);
    }
    return r;
}
template <bool F32>
__device__ __forceinline__ void widen8(const Raw<F32> &r, float (&x)[8])
{
    const uint32_t *w = reinterpret_cast<const uint32_t *>(r.w);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = F32 ? __uint_as_float(w[F32 ? e : 0]) : __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
}

template <bool F32>
__device__ __forceinline__ void store8(void *base, int64_t at, bool vec, const float (&x)[8])
{
    if (F32) {
        float *p = static_cast<float *>(base) + at;
        if (vec) {
            *reinterpret_cast<float4 *>(p) = make_float4(x[0], x[1], x[2], x[3]);
            *reinterpret_cast<float4 *>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) p[e] = x[e];
        }
    } else {
        uint16_t *p = static_cast<uint16_t *>(base) + at;
        const uint4 w = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
        if (vec) {
            *reinterpret_cast<uint4 *>(p) = w;
        } else {
            const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int e = 0; e < 8; ++e) p[e] = (uint16_t)(v[e / 2] >> (16 * (e & 1)));
        }
    }
}

struct AppendArgs {
    Step s;
    const void *q, *k, *v;
    void *q_out;
    int64_t ldq, ldq_out, ldk, ldv;
    int32_t q_heads, rope, vec;
    int32_t slices, slice; // of a row's heads: how many, heads in each
    const double *inv_freq;
};

// The token of a row: its sequence is the last one that begins at or before the row.  false: the row is of none, or of a line
// outside the table, or lies before the first token.
__device__ __forceinline__ bool token_of(const Step &s, int32_t row, int32_t *line, int32_t *pos)
{
    const int32_t i = s.row_start ? last_not_above(s.n_seqs, row, [&](int32_t k) { return (int64_t)row_of(s, k); }) : row;
    if (i >= s.n_seqs) return false;
    const Seq q = seq_of(s, i);
    const int32_t j = row - q.row;
    *line = q.line;
    *pos = q.len - q.n + j;
    return j >= 0 && j < q.n && q.line >= 0 && *pos >= 0;
}

// The value of the lane LANES / 2 further in a head's LANES lanes, and a minimum or maximum over them, without a trip through LDS
// where the hardware can (16 lanes: rotations within a row of 16; 8: mirrored halves, then quads).
template <int LANES>
__device__ __forceinline__ float across(float x)
{
    const int32_t v = __float_as_int(x);
    return __int_as_float(LANES == 16 ? __builtin_amdgcn_mov_dpp(v, 0x128, 0xf, 0xf, true) : __builtin_amdgcn_ds_swizzle(v, 0x101f));
}
template <int LANES, class F>
__device__ __forceinline__ float over_lanes(float x, F pick)
{
#define QLLM_PICK(CTRL) x = pick(x, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), CTRL, 0xf, 0xf, true)))
    if (LANES == 16) {
        QLLM_PICK(0x128);
        QLLM_PICK(0x124);
        QLLM_PICK(0x122);
        QLLM_PICK(0x121);
    } else {
        QLLM_PICK(0x141);
        QLLM_PICK(0xb1);
        QLLM_PICK(0x4e);
    }
#undef QLLM_PICK
    return x;
}

// A wave has one row, or a slice of its heads where there are few rows; D / 8 lanes per head, 8 channels per lane.  It works the
// row's angles out for itself (64 lanes, D / 2 of them) and keeps them in LDS; nothing waits for another wave.  Heads are asked for
// two turns ahead.  2048 rows of 32 + 32 + 32 heads: 28 us with a workgroup per row, which is mostly waiting for the next link of
// row -> sequence -> position -> angles.
template <int D, bool F32>
__global__ __launch_bounds__(THREADS) void append_kernel(const AppendArgs a)
{
    constexpr int LANES = D / 8, PER = 64 / LANES, HALF = LANES / 2; // lanes of a head, heads at a time
    // (cos, - sin) and (cos, sin): for a pair's first channel and its second.  Neighbouring lanes read neighbouring entries.
    __shared__ double2 turns[THREADS / 64][2][D / 2];
    const Step &s = a.s;
    const int32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), tid = threadIdx.x & 63, lane = tid % LANES;
    double2(&turn)[2][D / 2] = turns[wave];
    // Neighbouring rows go to one XCD (workgroup b to XCD b % 8), whose L2 puts a page's lines together: a line holds two tokens'
    // codes of a head, 32 tokens' parameters.
    const int32_t block = blockIdx.x % 8 * (gridDim.x / 8) + blockIdx.x / 8;
    const int32_t task = block * (THREADS / 64) + wave, row = __builtin_amdgcn_readfirstlane((int32_t)((uint32_t)task / (uint32_t)a.slices));
    if (row >= s.rows) return;
    const int32_t q_heads = a.q ? a.q_heads : 0, all = q_heads + 2 * s.heads;
    const int32_t begin = (task - row * a.slices) * a.slice, units = begin + a.slice < all ? begin + a.slice : all; // its heads: begin .. units - 1
    const bool vec = a.vec;
    const int32_t s_heads = s.heads;
    // head u of the row: 0 query, 1 key, 2 value
    const auto kind_of = [&](int32_t u) { return u < q_heads ? 0 : (u < q_heads + s.heads ? 1 : 2); };
    const auto head_of = [&](int32_t u, int32_t kind) { return u - (kind > 0 ? q_heads : 0) - (kind > 1 ? s.heads : 0); };
    // (by masks and not by a conditional expression of the arguments: that becomes a choice of a place among the kernel's arguments,
    // and every fetch a trip to memory for its own address first)
    constexpr int SIZE = F32 ? 4 : 2;
    const uint64_t at_v = reinterpret_cast<uint64_t>(a.v) + row * a.ldv * SIZE;
    const uint64_t k_off = reinterpret_cast<uint64_t>(a.k) + row * a.ldk * SIZE - at_v, q_off = reinterpret_cast<uint64_t>(a.q) + row * a.ldq * SIZE - at_v;
    const auto fetch = [=](int32_t u) {
        Raw<F32> r = {};
        if (u < units) {
            const uint64_t is_q = -(uint64_t)(u < q_heads), is_k = -(uint64_t)(u >= q_heads && u < q_heads + s_heads);
            const int32_t head = u - (u >= q_heads ? q_heads : 0) - (u >= q_heads + s_heads ? s_heads : 0);
            r = load8<F32>(reinterpret_cast<const void *>(at_v + (is_q & q_off) + (is_k & k_off)), head * D + 8 * lane, vec);
        }
        return r;
    };
    Raw<F32> raw[2] = {fetch(begin + tid / LANES), fetch(begin + PER + tid / LANES)};
    int32_t line, pos;
    if (!token_of(s, row, &line, &pos)) return; // the same for the whole wave
    const int32_t page = page_of(s, line, pos);
    if (a.rope != QLLM_ROPE_NONE && begin < q_heads + s_heads) { // not for values alone
        if (tid < D / 2) {
            double sn, cs;
            sincos((double)pos * a.inv_freq[tid], &sn, &cs);
            const int32_t at = a.rope == QLLM_ROPE_HALVES ? tid % 8 * HALF + tid / 8 : tid % 4 * LANES + tid / 4;
            turn[0][at] = make_double2((float)cs, -(float)sn);
            turn[1][at] = make_double2((float)cs, (float)sn);
        }
        __builtin_amdgcn_wave_barrier();
    }
    const int32_t P = 1 << s.page_shift, in_page = pos & (P - 1);
    const auto heads = [&](int32_t base, Raw<F32> &next) { // lanes beyond the last head go through it too: they take part in the exchanges
        const int32_t u = base + tid / LANES, kind = kind_of(u), head = head_of(u, kind);
        const bool real = u < units;
        float x[8];
        widen8<F32>(next, x);
        next = fetch(u + 2 * PER);
        // x1 c - x2 s and x2 c + x1 s: the products are exact in double, the sum is rounded there once (a fused multiply-add
        // of an exact product is that sum), then to float
        if (a.rope != QLLM_ROPE_NONE && __any(kind != 2)) { // values do not turn
            float y[8];
            if (a.rope == QLLM_ROPE_HALVES) { // the partner's channels sit half the head's lanes away
                const double2 *t = turn[lane >= HALF] + lane % HALF;
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = (float)__builtin_fma((double)x[e], t[HALF * e].x, (double)across<LANES>(x[e]) * t[HALF * e].y);
            } else {
                const double2 *t = turn[1] + lane;
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const double x1 = x[e], x2 = x[e + 1], c = t[LANES * (e / 2)].x, sn = t[LANES * (e / 2)].y;
                    y[e] = (float)__builtin_fma(x1, c, -(x2 * sn)), y[e + 1] = (float)__builtin_fma(x2, c, x1 * sn);
                }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = kind != 2 ? y[e] : x[e];
        }
        if (kind == 0) {
            if (real) store8<F32>(a.q_out, (int64_t)row * a.ldq_out + head * D + 8 * lane, vec, x);
        }
        if (base + PER <= q_heads) return; // queries all
        // Eq. (2) over the head's channels
        float lo = x[0], hi = x[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) lo = fminf(lo, x[e]), hi = fmaxf(hi, x[e]);
        lo = over_lanes<LANES>(lo, [](float p, float q) { return fminf(p, q); });
        hi = over_lanes<LANES>(hi, [](float p, float q) { return fmaxf(p, q); });
        if (!real || kind == 0 || page < 0) return;
        float alpha = (hi - lo) * (1.0f / 15.0f);
        if (!(alpha >= 0x1p-126f)) alpha = 1.0f;
        const float inv = 1.0f / alpha;
        // A float near MAGIC = 1.5 2^23 is MAGIC plus an integer, in its value as in its bits: one fused multiply-add rounds the
        // exact product to the nearest integer, and code 0 is the number MAGIC - beta.
        int32_t beta;
        uint32_t codes = 0;
        if (fabsf(lo * inv) < FAST_LIMIT && fabsf(hi * inv) < FAST_LIMIT) {
            beta = -qllm_detail::rne_product_fast(lo, inv);
            const float zero = qllm_detail::MAGIC - (float)beta, most = zero + 15.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                codes += __float_as_uint(__builtin_amdgcn_fmed3f(__builtin_fmaf(x[e], inv, qllm_detail::MAGIC), zero, most)) << (4 * e);
            codes -= __float_as_uint(zero) * 0x11111111u;
        } else {
            const double z = -qllm_detail::rne_product_slow(lo, inv);
            beta = (int32_t)fmin(fmax(z, -2147483647.0), 2147483647.0);
#pragma unroll
            for (int e = 0; e < 8; ++e) codes |= (uint32_t)qllm_detail::quant_code<15>(x[e], inv, beta, 0) << (4 * e);
        }
        uint8_t *part = s.pages + page * s.page_bytes + (int64_t)head * P * (D + 16);
        const int32_t value = kind - 1;
        *reinterpret_cast<uint32_t *>(part + ((int64_t)value * P + in_page) * (D / 2) + 4 * lane) = codes;
        uint8_t *params = part + (int64_t)P * D + 8 * (int64_t)value * P;
        if (lane == 0) *reinterpret_cast<float *>(params + 4 * in_page) = alpha;
        if (lane == 1) *reinterpret_cast<int32_t *>(params + 4 * P + 4 * in_page) = beta;
    };
    for (int32_t base = begin; base < units; base += 2 * PER) {
        heads(base, raw[0]);
        if (base + PER < units) heads(base + PER, raw[1]);
    }
}

struct ReadArgs {
    Step s;
    void *k_out, *v_out;
    int64_t ldk, ldv;
    int32_t vec;
};

template <int D, bool F32>
__global__ __launch_bounds__(THREADS) void read_kernel(const ReadArgs a)
{
    constexpr int LANES = D / 8, PER = THREADS / LANES;
    const Step &s = a.s;
    const int32_t row = blockIdx.x, tid = threadIdx.x;
    int32_t line, pos;
    if (!token_of(s, row, &line, &pos)) return;
    const int32_t page = page_of(s, line, pos);
    if (page < 0) return;
    const int32_t P = 1 << s.page_shift, in_page = pos & (P - 1), lane = tid % LANES;
    // (addresses by masks: see append_kernel)
    const uint64_t at_k = reinterpret_cast<uint64_t>(a.k_out) + row * a.ldk * (F32 ? 4 : 2);
    const uint64_t v_off = reinterpret_cast<uint64_t>(a.v_out) + row * a.ldv * (F32 ? 4 : 2) - at_k;
    const bool has_k = a.k_out != nullptr, has_v = a.v_out != nullptr, vec = a.vec;
    for (int32_t u = tid / LANES; u < 2 * s.heads; u += PER) {
        const int32_t value = u >= s.heads, head = value ? u - s.heads : u;
        if ((value && !has_v) || (!value && !has_k)) continue;
        const uint8_t *part = s.pages + page * s.page_bytes + (int64_t)head * P * (D + 16);
        const uint32_t codes = *reinterpret_cast<const uint32_t *>(part + ((int64_t)value * P + in_page) * (D / 2) + 4 * lane);
        const uint8_t *params = part + (int64_t)P * D + 8 * (int64_t)value * P;
        const float alpha = *reinterpret_cast<const float *>(params + 4 * in_page);
        const int32_t beta = *reinterpret_cast<const int32_t *>(params + 4 * P + 4 * in_page);
        float x[8];
        if (beta > -(1 << 23) && beta < 1 << 23) { // code - beta is exact in float
            const float zero = (float)beta;
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = alpha * ((float)(codes >> (4 * e) & 15u) - zero);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = (float)((double)alpha * ((double)(codes >> (4 * e) & 15u) - (double)beta));
        }
        store8<F32>(reinterpret_cast<void *>(at_k + (-(uint64_t)value & v_off)), head * D + 8 * lane, vec, x);
    }
}

// The pairs travel as kernel arguments: no list in device memory, nothing to upload.
constexpr int PAIRS = 256;
struct Pairs {
    int32_t src[PAIRS], dst[PAIRS];
};

// 16 bytes a lane and step, four steps of a workgroup in flight; grid: pieces of a page, pairs, layers.
__global__ __launch_bounds__(THREADS) void copy_pages_kernel(uint8_t *pages, int64_t layer_stride, int64_t page_bytes, const Pairs pairs)
{
    uint8_t *layer = pages + (int64_t)blockIdx.z * layer_stride;
    const uint4 *src = reinterpret_cast<const uint4 *>(layer + (int64_t)pairs.src[blockIdx.y] * page_bytes);
    uint4 *dst = reinterpret_cast<uint4 *>(layer + (int64_t)pairs.dst[blockIdx.y] * page_bytes);
    const int64_t words = page_bytes / 16, at = (int64_t)blockIdx.x * THREADS * 4 + threadIdx.x;
    if (at + 3 * THREADS < words) {
        const uint4 x0 = src[at], x1 = src[at + THREADS], x2 = src[at + 2 * THREADS], x3 = src[at + 3 * THREADS];
        dst[at] = x0, dst[at + THREADS] = x1, dst[at + 2 * THREADS] = x2, dst[at + 3 * THREADS] = x3;
    } else {
        for (int64_t i = at; i < words; i += THREADS) dst[i] = src[i];
    }
}

// Rows of 16-byte accesses; else QLLM_ERR_ALIGN where a row misses its own type's alignment.
int32_t row_access(int32_t dtype, const void *const *ptrs, const int64_t *lds, int n, int32_t *vec)
{
    const int64_t size = dtype == QLLM_F32 ? 4 : 2;
    uintptr_t bits = 0;
    for (int i = 0; i < n; ++i)
        if (ptrs[i]) {
            if (reinterpret_cast<uintptr_t>(ptrs[i]) & (uintptr_t)(size - 1)) return QLLM_ERR_ALIGN;
            bits |= reinterpret_cast<uintptr_t>(ptrs[i]) | (uintptr_t)(lds[i] * size);
        }
    *vec = (bits & 15u) == 0;
    return QLLM_OK;
}

} // namespace

extern "C" int32_t qllm_kv_append(const void *q, int64_t ldq, int64_t q_heads, void *q_out, int64_t ldq_out, const void *k, int64_t ldk,
                                  const void *v, int64_t ldv, int32_t x_dtype, int32_t rope, const double *inv_freq,
                                  const qllm_kv_cache *cache, const qllm_kv_batch *batch, void *hip_stream)
{
    AppendArgs a;
    const int32_t rc = prepare_step(cache, batch, true, &a.s);
    if (rc != QLLM_OK) return rc;
    const bool some = batch->rows > 0; // an empty tensor has no address
    if (some && (!k || !v)) return QLLM_ERR_NULL;
    if ((x_dtype != QLLM_F32 && x_dtype != QLLM_BF16) || rope < QLLM_ROPE_NONE || rope > QLLM_ROPE_PAIRS) return QLLM_ERR_DTYPE;
    if ((some && !q != !q_out) || (rope != QLLM_ROPE_NONE && !inv_freq)) return QLLM_ERR_NULL;
    const int64_t width = cache->heads * cache->dim;
    if (ldk < width || ldv < width) return QLLM_ERR_SHAPE;
    if (q && (q_heads <= 0 || q_heads > (1 << 16) || ldq < q_heads * cache->dim || ldq_out < q_heads * cache->dim)) return QLLM_ERR_SHAPE;
    if (reinterpret_cast<uintptr_t>(inv_freq) & 7u) return QLLM_ERR_ALIGN;
    const void *ptrs[4] = {q, q_out, k, v};
    const int64_t lds[4] = {ldq, ldq_out, ldk, ldv};
    const int32_t ra = row_access(x_dtype, ptrs, lds, 4, &a.vec);
    if (ra != QLLM_OK) return ra;
    if (batch->rows == 0 || batch->n_seqs == 0) return QLLM_OK;
    a.q = q, a.k = k, a.v = v, a.q_out = q_out;
    a.ldq = ldq, a.ldq_out = ldq_out, a.ldk = ldk, a.ldv = ldv;
    a.q_heads = (int32_t)q_heads, a.rope = rope, a.inv_freq = inv_freq;
    // Few rows: as many slices of their heads as give the card 4096 waves, 16 on each of 256 CUs
    const int64_t rows = batch->row_start ? batch->rows : batch->n_seqs, heads = (q ? q_heads : 0) + 2 * cache->heads, per = 512 / cache->dim;
    int64_t slices = 4096 / rows;
    slices = slices < 1 ? 1 : slices;
    a.slice = (int32_t)(((heads + slices - 1) / slices + per - 1) / per * per);
    a.slices = (int32_t)((heads + a.slice - 1) / a.slice);
    const dim3 grid((unsigned)((rows * a.slices + THREADS / 64 * 8 - 1) / (THREADS / 64 * 8) * 8));
    hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
    (void)hipGetLastError();
    if (cache->dim == 128) {
        if (x_dtype == QLLM_F32) hipLaunchKernelGGL((append_kernel<128, true>), grid, dim3(THREADS), 0, stream, a);
        else hipLaunchKernelGGL((append_kernel<128, false>), grid, dim3(THREADS), 0, stream, a);
    } else {
        if (x_dtype == QLLM_F32) hipLaunchKernelGGL((append_kernel<64, true>), grid, dim3(THREADS), 0, stream, a);
        else hipLaunchKernelGGL((append_kernel<64, false>), grid, dim3(THREADS), 0, stream, a);
    }
    return launched("cache append: launch");
}

extern "C" int32_t qllm_kv_read(const qllm_kv_cache *cache, const qllm_kv_batch *batch, void *k_out, int64_t ldk, void *v_out, int64_t ldv,
                                int32_t dtype, void *hip_stream)
{
    ReadArgs a;
    const int32_t rc = prepare_step(cache, batch, true, &a.s);
    if (rc != QLLM_OK) return rc;
    if (dtype != QLLM_F32 && dtype != QLLM_BF16) return QLLM_ERR_DTYPE;
    const int64_t width = cache->heads * cache->dim;
    if ((k_out && ldk < width) || (v_out && ldv < width)) return QLLM_ERR_SHAPE;
    const void *ptrs[2] = {k_out, v_out};
    const int64_t lds[2] = {ldk, ldv};
    const int32_t ra = row_access(dtype, ptrs, lds, 2, &a.vec);
    if (ra != QLLM_OK) return ra;
    if (batch->rows == 0 || batch->n_seqs == 0 || (!k_out && !v_out)) return QLLM_OK;
    a.k_out = k_out, a.v_out = v_out, a.ldk = ldk, a.ldv = ldv;
    const dim3 grid((unsigned)(batch->row_start ? batch->rows : batch->n_seqs));
    hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
    (void)hipGetLastError();
    if (cache->dim == 128) {
        if (dtype == QLLM_F32) hipLaunchKernelGGL((read_kernel<128, true>), grid, dim3(THREADS), 0, stream, a);
        else hipLaunchKernelGGL((read_kernel<128, false>), grid, dim3(THREADS), 0, stream, a);
    } else {
        if (dtype == QLLM_F32) hipLaunchKernelGGL((read_kernel<64, true>), grid, dim3(THREADS), 0, stream, a);
        else hipLaunchKernelGGL((read_kernel<64, false>), grid, dim3(THREADS), 0, stream, a);
    }
    return launched("cache read: launch");
}

extern "C" int32_t qllm_kv_copy_pages(uint8_t *pages, int64_t n_layers, int64_t layer_stride, int64_t n_pages, int64_t page_bytes,
                                      const int32_t *src_host, const int32_t *dst_host, int64_t n, void *hip_stream)
{
    if (!pages || (n > 0 && (!src_host || !dst_host))) return QLLM_ERR_NULL;
    if (n < 0 || n_layers < 0 || n_layers > 65535 || n_pages <= 0 || n_pages > INT32_MAX || page_bytes <= 0 || page_bytes > (1ll << 40)) return QLLM_ERR_SHAPE;
    if (n_layers > 1 && layer_stride / page_bytes < n_pages) return QLLM_ERR_SHAPE;
    if ((reinterpret_cast<uintptr_t>(pages) & 15u) || (page_bytes & 15) || (n_layers > 1 && (layer_stride & 15))) return QLLM_ERR_ALIGN;
    if (n == 0 || n_layers == 0) return QLLM_OK;
    if (n > n_pages) return QLLM_ERR_PAGES; // some page is copied to twice
    for (int64_t i = 0; i < n; ++i)
        if (src_host[i] < 0 || src_host[i] >= n_pages || dst_host[i] < 0 || dst_host[i] >= n_pages) return QLLM_ERR_PAGES;
    uint8_t *marks = new (std::nothrow) uint8_t[(size_t)n_pages]();
    if (!marks) return QLLM_ERR_WORKSPACE;
    bool clash = false;
    for (int64_t i = 0; i < n; ++i) {
        clash |= marks[dst_host[i]] != 0;
        marks[dst_host[i]] = src_host[i] == dst_host[i] ? 1 : 2; // 2: written to
    }
    for (int64_t i = 0; i < n; ++i) clash |= src_host[i] != dst_host[i] && marks[src_host[i]] == 2;
    delete[] marks;
    if (clash) return QLLM_ERR_PAGES;
    const int64_t pieces = (page_bytes / 16 + THREADS * 4 - 1) / (THREADS * 4);
    hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
    (void)hipGetLastError();
    int64_t at = 0;
    while (at < n) {
        Pairs p = {};
        int m = 0;
        for (; at < n && m < PAIRS; ++at)
            if (src_host[at] != dst_host[at]) p.src[m] = src_host[at], p.dst[m] = dst_host[at], ++m;
        if (!m) break;
        hipLaunchKernelGGL(copy_pages_kernel, dim3((unsigned)pieces, (unsigned)m, (unsigned)n_layers), dim3(THREADS), 0, stream, pages, layer_stride,
                           page_bytes, p);
        const int32_t rc = launched("cache pages: copy");
        if (rc != QLLM_OK) return rc;
    }
    return QLLM_OK;
}
