// Causal attention over the 4-bit key/value cache.
//
// For a kv head the queries of its group of query heads are rows of one matrix: row r of a sequence's n rows x G heads is token
// r / G, head r % G.  Codes are integers, so with k = alpha (c - beta) the score of a token is
//     scale alpha (q . (16 + c) - (16 + beta) sum q),
// the first product on the matrix cores: 16 + c is an exact bf16 whose bits are 0x4180 | c << 3, two vector instructions for a
// pair of codes.  In the same way sum_t p_t v_t = sum_t (p_t alpha_t)(16 + c_t) - sum_t (p_t alpha_t)(16 + beta_t), with p_t alpha_t
// rounded to bf16 first and the rounded number used in both sums.  The scores are formed transposed (tokens x rows): their
// accumulator then is, register for register, the operand that meets the values, and nothing crosses lanes in between.
#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include "kv_common.h"

namespace {

using namespace qllm_kv_detail;

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int ROWS = 16, STEP = 32, WAVES = 4; // rows of a tile, tokens of a step, waves of a workgroup
constexpr float LOG2E = 1.44269504088896341f;
constexpr float SLACK = 8.0f; // the running maximum follows only when the scores pass it by this much: weights stay below 2^8

struct AttendArgs {
    Step s;
    const void *q;
    void *out;
    int64_t ldq, ldo;
    int32_t q_heads, group, window; // window 0: none
    float scale2;                   // scale * log2 e
};

__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}

// 16 + code of nibble i (0..3) of both halves of w, as a pair of bf16
template <int I>
__device__ __forceinline__ uint32_t pair16(uint32_t w)
{
    const uint32_t t = I == 0 ? w << 3 : w >> (4 * I - 3);
    return (t & 0x00780078u) | 0x41804180u;
}

// 8 codes of a dword as a matrix-core operand: elements are codes 0, 4, 1, 5, 2, 6, 3, 7
__device__ __forceinline__ bf16x8 operand16(uint32_t w)
{
    return __builtin_bit_cast(bf16x8, u32x4{pair16<0>(w), pair16<1>(w), pair16<2>(w), pair16<3>(w)});
}

// A row tile of a workgroup: rows first .. first + 15 of a sequence's n * group rows, and what they may see.
struct Tile {
    Seq seq;
    int32_t first, rows;
};

// Sequence i's tiles begin at number row_start[i] * group / ROWS + i: at least as many numbers as it has tiles, in order.
__device__ __forceinline__ Tile tile_of(const AttendArgs &a, int64_t number)
{
    Tile t;
    int32_t i;
    int64_t begin;
    if (a.s.row_start) {
        auto first = [&](int32_t k) { return (int64_t)row_of(a.s, k) * a.group / ROWS + k; };
        i = last_not_above(a.s.n_seqs, number, first);
        begin = first(i);
    } else {
        const int64_t per = (a.group + ROWS - 1) / ROWS;
        i = (int32_t)(number / per);
        begin = i * per;
    }
    t.seq = seq_of(a.s, i);
    const int64_t at = (number - begin) * ROWS;
    t.rows = t.seq.n * a.group;
    t.first = at < 0 || at > t.rows ? t.rows : (int32_t)at;
    return t;
}

template <bool F32>
__device__ __forceinline__ float load1(const void *p, int64_t at)
{
    return F32 ? static_cast<const float *>(p)[at] : __uint_as_float((uint32_t)static_cast<const uint16_t *>(p)[at] << 16);
}

// fp32 as a sum of PARTS bf16 (three hold all 24 bits)
template <int PARTS>
__device__ __forceinline__ void split(float x, float (&part)[PARTS])
{
#pragma unroll
    for (int i = 0; i < PARTS; ++i) {
        part[i] = __uint_as_float(pack_bf16(x, 0.0f) << 16);
        x -= part[i];
    }
}

template <int D, bool F32Q, bool F32O>
__global__ __launch_bounds__(WAVES * 64) void attend_kernel(const AttendArgs a)
{
    constexpr int PARTS = F32Q ? 3 : 1;
    constexpr int KS = D / 32, DT = D / 16; // steps of 32 channels; tiles of 16 channels (one channel of each lane row)
    __shared__ float mrg_m[WAVES][ROWS], mrg_l[WAVES][ROWS], mrg_o[WAVES][ROWS][D + 4];

    const Step &s = a.s;
    const int32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
    const int32_t head = blockIdx.y, P = 1 << s.page_shift;
    const Tile t = tile_of(a, blockIdx.x);
    if (t.first >= t.rows) return;

    // this lane's row (a column of the transposed products) and the tokens it sees: lo .. hi
    const int32_t row = t.first + r, token = row / a.group;
    const bool real = row < t.rows;
    const int32_t cap = s.table_ld << s.page_shift, limit = t.seq.line < 0 ? 0 : (t.seq.len < cap ? t.seq.len : cap);
    const auto pos_of = [&](int32_t tok) { return t.seq.len - t.seq.n + tok; };
    const auto hi_of = [&](int32_t p) { return p < limit ? p : limit - 1; };
    const auto lo_of = [&](int32_t p) { return a.window > 0 && p - a.window + 1 > 0 ? p - a.window + 1 : 0; };
    const int32_t pos = pos_of(token), hi = real ? hi_of(pos) : -1, lo = lo_of(pos);
    const int32_t last_row = t.first + ROWS < t.rows ? t.first + ROWS - 1 : t.rows - 1;
    const int32_t p_first = pos_of(t.first / a.group), p_last = pos_of(last_row / a.group);
    const int32_t all_lo = lo_of(p_first), all_hi = hi_of(p_last);       // seen by some row
    const int32_t each_lo = lo_of(p_last), each_hi = hi_of(p_first);     // seen by every row

    // queries: element e of step k of lane group g is channel (D / 4) g + 8 k + {0, 4, 1, 5, 2, 6, 3, 7}[e]
    bf16x8 qo[PARTS][KS];
    float qsum = 0.0f;
    {
        const int64_t at = (int64_t)(t.seq.row + token) * a.ldq + (int64_t)(head * a.group + row - token * a.group) * D + D / 4 * g;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            float x[8], part[8][PARTS];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[e] = real ? load1<F32Q>(a.q, at + 8 * k + (e >> 1) + 4 * (e & 1)) : 0.0f;
                qsum += x[e];
                split<PARTS>(x[e], part[e]);
            }
#pragma unroll
            for (int i = 0; i < PARTS; ++i)
                qo[i][k] = __builtin_bit_cast(bf16x8, u32x4{pack_bf16(part[0][i], part[1][i]), pack_bf16(part[2][i], part[3][i]),
                                                            pack_bf16(part[4][i], part[5][i]), pack_bf16(part[6][i], part[7][i])});
        }
        qsum += __shfl_xor(qsum, 16);
        qsum += __shfl_xor(qsum, 32);
    }

    f32x4 acc[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.0f, off = 0.0f; // running maximum; this lane's parts of the sums of p and of p alpha (16 + beta)

    for (int32_t st = all_lo / STEP + wave; st * STEP <= all_hi; st += WAVES) {
        const int32_t t0 = st * STEP;
        const int32_t page = page_of(s, t.seq.line, t0);
        if (page < 0) continue;
        const uint8_t *part = s.pages + page * s.page_bytes + (int64_t)head * P * (D + 16);
        const int32_t in_page = t0 & (P - 1);
        const uint8_t *kc = part + (int64_t)in_page * (D / 2), *vc = kc + (int64_t)P * (D / 2);
        const float *par = reinterpret_cast<const float *>(part + (int64_t)P * D) + in_page;

        float sc[8], va[8], vb[8]; // scores, alpha and 16 + beta of the values, of tokens 16 h + 4 g + i
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t w[KS];
            const uint8_t *src = kc + (16 * h + r) * (D / 2) + D / 8 * g;
            if (D == 128) {
                const uint4 x = *reinterpret_cast<const uint4 *>(src);
                w[0] = x.x, w[1] = x.y, w[KS - 2] = x.z, w[KS - 1] = x.w;
            } else {
                const uint2 x = *reinterpret_cast<const uint2 *>(src);
                w[0] = x.x, w[1] = x.y;
            }
            f32x4 d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = PARTS - 1; i >= 0; --i)
#pragma unroll
                for (int k = 0; k < KS; ++k) d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(operand16(w[k]), qo[i][k], d, 0, 0, 0);
            const int32_t at = 16 * h + 4 * g;
            const float4 ka = *reinterpret_cast<const float4 *>(par + at);
            const int4 kb = *reinterpret_cast<const int4 *>(par + P + at);
            const float4 wa = *reinterpret_cast<const float4 *>(par + 2 * P + at);
            const int4 wb = *reinterpret_cast<const int4 *>(par + 3 * P + at);
            const float kav[4] = {ka.x, ka.y, ka.z, ka.w}, vav[4] = {wa.x, wa.y, wa.z, wa.w};
            const int32_t kbv[4] = {kb.x, kb.y, kb.z, kb.w}, vbv[4] = {wb.x, wb.y, wb.z, wb.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                sc[4 * h + i] = kav[i] * a.scale2 * __builtin_fmaf(-((float)kbv[i] + 16.0f), qsum, d[i]);
                va[4 * h + i] = vav[i];
                vb[4 * h + i] = (float)vbv[i] + 16.0f;
            }
        }
        if (t0 < each_lo || t0 + STEP - 1 > each_hi) { // some row does not see some token; what lies there may be anything
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int32_t tok = t0 + 16 * (i >> 2) + 4 * g + (i & 3);
                const bool seen = tok >= lo && tok <= hi;
                sc[i] = seen ? sc[i] : -INFINITY;
                va[i] = seen ? va[i] : 0.0f;
                vb[i] = seen ? vb[i] : 0.0f;
            }
        }
        float top = sc[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) top = fmaxf(top, sc[i]);
        if (__any(top > m + SLACK)) {
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float now = fmaxf(m, top);
            const float f = now == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - now);
            m = now, l *= f, off *= f;
#pragma unroll
            for (int i = 0; i < DT; ++i) acc[i] *= f;
        }
        const float base = m == -INFINITY ? 0.0f : m;
        float pv[8], part_p[8][PARTS];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float p = __builtin_amdgcn_exp2f(sc[i] - base);
            l += p;
            pv[i] = p * va[i];
            split<PARTS>(pv[i], part_p[i]);
#pragma unroll
            for (int j = 0; j < PARTS; ++j) off = __builtin_fmaf(part_p[i][j], vb[i], off);
        }
        // values: tokens of element e as the scores have them, 16 (e / 4) + 4 g + e % 4; channels (D / 16) r .. of this lane
        uint32_t w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint8_t *src = vc + (16 * (e >> 2) + 4 * g + (e & 3)) * (D / 2) + D / 32 * r;
            w[e] = D == 128 ? *reinterpret_cast<const uint32_t *>(src) : *reinterpret_cast<const uint16_t *>(src);
        }
        uint32_t low[4], high[4]; // codes 0..3 and 4..7 of two neighbouring tokens
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            low[e] = __builtin_amdgcn_perm(w[2 * e + 1], w[2 * e], 0x05040100u);
            high[e] = __builtin_amdgcn_perm(w[2 * e + 1], w[2 * e], 0x07060302u);
        }
        const auto tile = [&](int i, bf16x8 v) {
#pragma unroll
            for (int j = PARTS - 1; j >= 0; --j) {
                const bf16x8 p = __builtin_bit_cast(bf16x8, u32x4{pack_bf16(part_p[0][j], part_p[1][j]), pack_bf16(part_p[2][j], part_p[3][j]),
                                                                  pack_bf16(part_p[4][j], part_p[5][j]), pack_bf16(part_p[6][j], part_p[7][j])});
                acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p, acc[i], 0, 0, 0);
            }
        };
        const auto four = [&](const uint32_t (&x)[4], int at) {
            tile(at + 0, __builtin_bit_cast(bf16x8, u32x4{pair16<0>(x[0]), pair16<0>(x[1]), pair16<0>(x[2]), pair16<0>(x[3])}));
            tile(at + 1, __builtin_bit_cast(bf16x8, u32x4{pair16<1>(x[0]), pair16<1>(x[1]), pair16<1>(x[2]), pair16<1>(x[3])}));
            tile(at + 2, __builtin_bit_cast(bf16x8, u32x4{pair16<2>(x[0]), pair16<2>(x[1]), pair16<2>(x[2]), pair16<2>(x[3])}));
            tile(at + 3, __builtin_bit_cast(bf16x8, u32x4{pair16<3>(x[0]), pair16<3>(x[1]), pair16<3>(x[2]), pair16<3>(x[3])}));
        };
        four(low, 0);
        if (D == 128) four(high, DT - 4);
    }

    l += __shfl_xor(l, 16), off += __shfl_xor(off, 16);
    l += __shfl_xor(l, 32), off += __shfl_xor(off, 32);
    // accumulator i of tile c is channel (D / 16) (4 g + i) + c of this lane's row
    if (g == 0) mrg_m[wave][r] = m, mrg_l[wave][r] = l;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < DT; ++c) mrg_o[wave][r][DT * (4 * g + i) + c] = acc[c][i] - off;
    __syncthreads();
    for (int32_t x = threadIdx.x; x < ROWS * D; x += WAVES * 64) {
        const int32_t n = x / D, c = x % D, rw = t.first + n;
        if (rw >= t.rows) break;
        float top = -INFINITY, sum = 0.0f, o = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) top = fmaxf(top, mrg_m[w][n]);
        if (top == -INFINITY) top = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float f = __builtin_amdgcn_exp2f(mrg_m[w][n] - top);
            sum += f * mrg_l[w][n];
            o += f * mrg_o[w][n][c];
        }
        const float y = sum > 0.0f ? o / sum : (sum == 0.0f ? 0.0f : sum);
        const int32_t tok = rw / a.group;
        const int64_t at = (int64_t)(t.seq.row + tok) * a.ldo + (int64_t)(head * a.group + rw - tok * a.group) * D + c;
        if (F32O) static_cast<float *>(a.out)[at] = y;
        else static_cast<uint16_t *>(a.out)[at] = (uint16_t)pack_bf16(y, 0.0f);
    }
}

int32_t check(const qllm_kv_cache *cache, const qllm_kv_batch *batch, int64_t q_heads)
{
    if (q_heads <= 0 || q_heads > (1 << 16) || q_heads % cache->heads || cache->heads > 65535) return QLLM_ERR_SHAPE;
    if (batch->rows * (q_heads / cache->heads) + batch->n_seqs > INT32_MAX) return QLLM_ERR_SHAPE;
    return QLLM_OK;
}

} // namespace

extern "C" int64_t qllm_kv_attention_workspace_bytes(const qllm_kv_cache *cache, const qllm_kv_batch *batch, int64_t q_heads)
{
    Step s;
    int32_t rc = prepare_step(cache, batch, false, &s);
    if (rc == QLLM_OK) rc = check(cache, batch, q_heads);
    return rc != QLLM_OK ? rc : 256;
}

extern "C" int32_t qllm_kv_attention(const void *q, int32_t q_dtype, int64_t ldq, int64_t q_heads, const qllm_kv_cache *cache,
                                     const qllm_kv_batch *batch, float scale, int64_t window, void *out, int32_t out_dtype, int64_t ldo,
                                     void *workspace, int64_t workspace_bytes, void *hip_stream)
{
    AttendArgs a;
    int32_t rc = prepare_step(cache, batch, true, &a.s);
    if (rc != QLLM_OK) return rc;
    if (batch->rows > 0 && (!q || !out)) return QLLM_ERR_NULL; // an empty tensor has no address
    rc = check(cache, batch, q_heads);
    if (rc != QLLM_OK) return rc;
    if ((q_dtype != QLLM_F32 && q_dtype != QLLM_BF16) || (out_dtype != QLLM_F32 && out_dtype != QLLM_BF16)) return QLLM_ERR_DTYPE;
    if (ldq < q_heads * cache->dim || ldo < q_heads * cache->dim || window < 0 || !(fabsf(scale) <= 3e38f)) return QLLM_ERR_SHAPE;
    if ((reinterpret_cast<uintptr_t>(q) & (q_dtype == QLLM_F32 ? 3u : 1u)) || (reinterpret_cast<uintptr_t>(out) & (out_dtype == QLLM_F32 ? 3u : 1u)))
        return QLLM_ERR_ALIGN;
    if (!workspace || workspace_bytes < qllm_kv_attention_workspace_bytes(cache, batch, q_heads)) return QLLM_ERR_WORKSPACE;
    if (reinterpret_cast<uintptr_t>(workspace) & 15u) return QLLM_ERR_ALIGN;
    if (batch->rows == 0 || batch->n_seqs == 0) return QLLM_OK;
    a.q = q, a.out = out, a.ldq = ldq, a.ldo = ldo;
    a.q_heads = (int32_t)q_heads, a.group = (int32_t)(q_heads / cache->heads);
    a.window = window > INT32_MAX ? 0 : (int32_t)window;
    a.scale2 = scale * LOG2E;
    const int64_t tiles = batch->row_start ? batch->rows * a.group / ROWS + batch->n_seqs : batch->n_seqs * ((a.group + ROWS - 1) / ROWS);
    const dim3 grid((unsigned)tiles, (unsigned)cache->heads);
    hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
    (void)hipGetLastError();
#define QLLM_ATTEND(D, FQ, FO) hipLaunchKernelGGL((attend_kernel<D, FQ, FO>), grid, dim3(WAVES * 64), 0, stream, a)
    const int32_t kind = (cache->dim == 128 ? 4 : 0) + (q_dtype == QLLM_F32 ? 2 : 0) + (out_dtype == QLLM_F32 ? 1 : 0);
    switch (kind) {
    case 0: QLLM_ATTEND(64, false, false); break;
    case 1: QLLM_ATTEND(64, false, true); break;
    case 2: QLLM_ATTEND(64, true, false); break;
    case 3: QLLM_ATTEND(64, true, true); break;
    case 4: QLLM_ATTEND(128, false, false); break;
    case 5: QLLM_ATTEND(128, false, true); break;
    case 6: QLLM_ATTEND(128, true, false); break;
    default: QLLM_ATTEND(128, true, true); break;
    }
#undef QLLM_ATTEND
    return launched("cache attention: launch");
}
