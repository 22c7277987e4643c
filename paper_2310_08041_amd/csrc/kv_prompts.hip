// Causal attention over the 4-bit key/value cache: the kernel for prompts and chunks of prompts, which is bound by the matrix cores
// and the softmax beside them (kv_attend.h has the formulas).
//
// A workgroup of four waves owns 128 rows of a sequence and kv head, a wave 32 of them (columns of the transposed products), and
// walks the tokens they see in tiles of 64.  A tile's codes become bf16 operands 16 + c in LDS once for the four waves, while the
// tile before is multiplied: keys token by token, values channel by channel in the order in which the weights come out of the
// scores.  The softmax's vector instructions take as long as the products, so what can be a product is one:
//   - a key's zero point is 16 more channels (bf16 parts of - (16 + beta) meet those of the query's sum);
//   - the values' alpha comes in there too, as log2 alpha_v / (scale alpha_k) against a one: the weights leave the exponential as
//     p alpha_v, ready to be rounded;
//   - one product more per 16 tokens, shared by all channels, has - (16 + beta) of the values in its rows 0..2 (in parts) and
//     1 / alpha_v in the next ones: the zero points' share of the values' sums, and the sum of the weights.
// The zero points' sums are added to the others every few tiles, so that the two stay small and lose nothing to each other.
//
// The weights meet the values in bf16 parts, the same ones above and below the line.  With float32 out two of them, as in the kernel for
// few rows; with bf16 out one, rounded: error against 64 bits 0.0021 where bf16 out by itself costs 0.0017 (which two parts leave it at).
// One part and two, us: 2048 tokens x 32 heads 60 and 72 (float32 out 84 and 94), 2000 tokens behind 14000 x 8 heads of 8 1103 and 1450
// (float32 out 1158 and 1504).
//
// Two workgroups share a CU, so that one lays out while the other multiplies.  A launch of no more workgroups than the card holds
// leaves CUs with one, or with a long and a short one: there a workgroup has two groups of four waves, every other tile of tokens
// each, each with its own LDS, one of them half a turn behind, and joins their results at the end.  D 128, us, one group first:
// 2048 tokens x 32 heads 72 and 58, 1024 x 32 40 and 32, 512 rows behind 3500 tokens x 8 heads of 8 117 and 80, 4 x 100 behind
// 16000 430 and 284; more workgroups, 4096 x 32 171 and 182, 8 x 512 x 32 67 and 80.
// Where even so half of the CUs had nothing to do, a tile's tokens are shared by several workgroups, whose results a second kernel
// joins.  One part first, 8 heads of 8: 128 tokens behind 16000 273 and 90, behind 4000 79 and 37, 8 x 16 behind 2000 47 and 38;
// 128 behind 900 30 and 36.
#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include "kv_attend.h"

namespace {

using namespace qllm_kv_detail;

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int PROWS = 128, TILE = 64, WAVES = 4, THREADS = WAVES * 64; // rows of a workgroup, tokens of a tile, waves of a group
static_assert(TILE == 1 << 6, "tiles are compared by shifts");
constexpr int TOGETHER = 4; // tiles between two additions of the zero points' sums
constexpr int LEAST = 8;    // tiles of tokens of a part

// A tile of tokens as operands.
template <int D>
struct Operands {
    // a token's keys and zero point, a channel's values; rows are an odd number of 16 bytes apart: 16 of them cover all banks
    static constexpr int KS = D + 16 + 8, VS = TILE + 8;
    uint16_t k[TILE][KS]; // 8 channels at a time in the order 0, 4, 1, 5, 2, 6, 3, 7
    // Row r + 32 c: channel D / 32 r + c (a thread lays D / 32 neighbouring channels, 16 threads write 16 neighbouring rows); tokens
    // of 16: the 8 of lane half 0 (0..3, 8..11), then the others.
    uint16_t v[D][VS];
    uint16_t rows[8][VS]; // of the shared product, tokens in the order of v: - (16 + beta) of the values and 1 / alpha, three bf16 parts each
    float ka[TILE];       // scale alpha of the keys
};

// What a thread asks of memory for a tile: a quarter of a token's keys, 8 tokens of D / 32 channels of the values, one token's
// alpha and beta (of its key in quarter 0, of its value in quarter 1) and its value's alpha.
template <int D>
struct Asked {
    uint32_t k[D / 32], v[8];
    float alpha, value_alpha;
    int32_t beta;
};

// Tile `k` of a kv head, from the one with the longest way back on (sequence after sequence, the tiles of a sequence in order, all
// of it backwards); false: there is none.  By one wave.  More sequences than it has lanes: their tiles are numbered from
// row_start * group / PROWS + i on, with gaps, which takes no sum over all of them.
__device__ __forceinline__ bool tile_at(const AttendArgs &a, int32_t k, Tile *t)
{
    const Step &s = a.s;
    const int32_t lane = threadIdx.x & 63;
    int32_t i, number;
    if (s.n_seqs <= 64) { // a sequence a lane
        Seq mine = {0, 0, -1, 0};
        if (lane < s.n_seqs) mine = seq_of(s, lane);
        const int32_t rows = mine.n * a.group;
        const int32_t tiles = rows <= a.few ? 0 : (int32_t)(((uint32_t)rows + PROWS - 1) / PROWS);
        int32_t upto = tiles;
        for (int32_t o = 1; o < s.n_seqs; o <<= 1) {
            const int32_t y = __shfl_up(upto, o);
            if (lane >= o) upto = __builtin_elementwise_add_sat(upto, y);
        }
        number = __builtin_amdgcn_readlane(upto, s.n_seqs - 1) - 1 - k;
        if (number < 0) return false;
        i = __popcll(__ballot(lane < s.n_seqs && upto <= number));
        i = i < s.n_seqs ? i : s.n_seqs - 1;
        number -= __builtin_amdgcn_readlane(upto - tiles, i);
        t->seq = Seq{__builtin_amdgcn_readlane(mine.row, i), __builtin_amdgcn_readlane(mine.n, i), __builtin_amdgcn_readlane(mine.line, i),
                     __builtin_amdgcn_readlane(mine.len, i)};
    } else {
        const auto first = [&](int32_t j) { return (int64_t)row_of(s, j) * a.group / PROWS + j; };
        number = (int32_t)((int64_t)s.rows * a.group / PROWS) + s.n_seqs - 1 - k;
        i = last_not_above(s.n_seqs, number, first);
        number -= (int32_t)first(i);
        const Seq q = seq_of(s, i); // the same in every lane
        t->seq = Seq{__builtin_amdgcn_readfirstlane(q.row), __builtin_amdgcn_readfirstlane(q.n), __builtin_amdgcn_readfirstlane(q.line),
                     __builtin_amdgcn_readfirstlane(q.len)};
    }
    t->rows = t->seq.n * a.group;
    const int64_t at = __builtin_amdgcn_readfirstlane(number) * (int64_t)PROWS;
    t->first = (int32_t)at;
    return at >= 0 && at < t->rows && t->rows > a.few;
}

// The tiles of tokens that some row of a tile sees, and how many workgroups share them.
struct Span {
    int32_t begin, end, parts;
};
__device__ __forceinline__ Span span_of(const AttendArgs &a, const Sight &v)
{
    Span x;
    x.begin = v.all_lo / TILE, x.end = v.all_hi < v.all_lo ? x.begin : v.all_hi / TILE + 1;
    x.parts = (x.end - x.begin) / LEAST;
    x.parts = x.parts < 1 ? 1 : (x.parts > a.parts ? a.parts : x.parts);
    return x;
}

// Quarter k of a row: element e of it of tile c is channel D / 32 (8 k + 4 h + e) + c.
template <int D, bool F32O>
__device__ __forceinline__ void put_quarter(const AttendArgs &a, int32_t head, int32_t q_row, int32_t head_of_row, int32_t k, const f32x4 (&x)[D / 32], float l)
{
    constexpr int DT = D / 32;
    const int32_t h = (threadIdx.x & 63) >> 5;
    const int64_t at = (int64_t)q_row * a.ldo + (head * a.group + head_of_row) * D + DT * (8 * k + 4 * h);
#pragma unroll
    for (int j = 0; j < 4; j += 4 / DT) { // four channels at a time
        float y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = quotient(x[e % DT][j + e / DT], l);
        if (F32O) {
            float *dst = static_cast<float *>(a.out) + at + DT * j;
            if (a.out_vec) *reinterpret_cast<float4 *>(dst) = make_float4(y[0], y[1], y[2], y[3]);
            else
                for (int e = 0; e < 4; ++e) dst[e] = y[e];
        } else {
            uint16_t *dst = static_cast<uint16_t *>(a.out) + at + DT * j;
            const uint2 w = make_uint2(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]));
            if (a.out_vec) *reinterpret_cast<uint2 *>(dst) = w;
            else dst[0] = (uint16_t)w.x, dst[1] = (uint16_t)(w.x >> 16), dst[2] = (uint16_t)w.y, dst[3] = (uint16_t)(w.y >> 16);
        }
    }
}
__device__ __forceinline__ f32x4 quarter_of(const f32x16 &x, int k) { return f32x4{x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]}; }

// Where a wave of a part keeps its results: the quarters of a lane's sums one after the other, 16 bytes a lane; a maximum and a sum.
__device__ __forceinline__ int64_t part_at(const AttendArgs &a, int32_t head, int32_t k, int32_t part, int32_t wave)
{
    return (((int64_t)k * a.s.heads + head) * a.parts + part) * WAVES + wave;
}

template <int D, bool F32O, int GROUPS>
__global__ __launch_bounds__(GROUPS * THREADS, 2) void prompts_kernel(const AttendArgs a)
{
    constexpr int KSTEPS = D / 16, DT = D / 32, WPARTS = F32O ? 2 : 1; // bf16 parts of a weight
    __shared__ __attribute__((aligned(16))) Operands<D> operands[GROUPS][2];

    const Step &s = a.s;
    const int32_t tid = threadIdx.x % THREADS, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 31, h = lane >> 5;
    const int32_t group = __builtin_amdgcn_readfirstlane(threadIdx.x / THREADS);
    Operands<D> *const op = operands[group];

    // Workgroups of one kv head go to the same XCD (head fastest) where heads are a multiple of 8: its L2 holds the tokens they share.
    // The tile with the longest way back first, workgroups without a tile last.
    const int32_t head = blockIdx.x % s.heads, part = (int32_t)(blockIdx.x / s.heads) % a.parts, k_tile = (int32_t)(blockIdx.x / s.heads) / a.parts;
    Tile t;
    if (!tile_at(a, k_tile, &t)) return;
    const int32_t tok0 = (int32_t)((uint32_t)t.first / (uint32_t)a.group), head0 = t.first - tok0 * a.group;
    const Sight v = sight_of(a, t, tok0, head0, PROWS);
    const Span span = span_of(a, v);
    if (part >= span.parts) return;

    // this lane's row, and what the wave's rows see
    const int32_t n = wave * 32 + col, token = tok0 + (int32_t)a.by_group.divide((uint32_t)(head0 + n)), head_of_row = head0 + n - (token - tok0) * a.group;
    const bool real = t.first + n < t.rows;
    const int32_t pos = t.seq.len - t.seq.n + token, hi = real ? hi_at(v.limit, pos) : -1, lo = lo_at(a, pos);
    const int32_t wave_rows = t.rows - t.first - wave * 32 < 32 ? t.rows - t.first - wave * 32 : 32; // may be none
    const int32_t w_first = t.seq.len - t.seq.n + tok0 + (int32_t)a.by_group.divide((uint32_t)(head0 + wave * 32));
    const int32_t w_last = t.seq.len - t.seq.n + tok0 + (int32_t)a.by_group.divide((uint32_t)(head0 + wave * 32 + (wave_rows > 0 ? wave_rows - 1 : 0)));
    const int32_t some_lo = lo_at(a, w_first), some_hi = wave_rows > 0 ? hi_at(v.limit, w_last) : -1;
    const int32_t each_lo = lo_at(a, w_last), each_hi = hi_at(v.limit, w_first);

    // page numbers of up to 64 blocks of 32 tokens, one a lane
    const int32_t tile_begin = span.begin + (int32_t)((int64_t)(span.end - span.begin) * part / span.parts);
    const int32_t tile_end = span.begin + (int32_t)((int64_t)(span.end - span.begin) * (part + 1) / span.parts);
    int32_t listed = tile_begin; // the first tile of the list
    const auto pages_from = [&](int32_t tile) { return page_of(s, t.seq.line, block_begin(tile * (TILE / 32) + lane, v.all_hi)); };
    int32_t pages = pages_from(listed);

    const int32_t P = 1 << s.page_shift;
    const int32_t k_tok = tid >> 2, k_part = tid & 3;                       // keys: token, quarter
    const int32_t v_chunk = wave * 2 + h, v_tok = v_chunk / 2 * 16 + 4 * (v_chunk & 1); // values: 8 tokens, v_tok + 0..3 and + 8..11
    const Codes16 codes;
    const auto part_of = [&](int32_t page) { return s.pages + (page < 0 ? 0 : page) * s.page_bytes + (int64_t)head * P * (D + 16); };
    const auto ask = [&](int32_t tile, Asked<D> &x, int32_t (&page)[2]) {
        if (tile - listed >= 32) listed = tile, pages = pages_from(tile);
#pragma unroll
        for (int b = 0; b < 2; ++b) page[b] = tile < tile_end ? __builtin_amdgcn_readlane(pages, 2 * (tile - listed) + b) : -1;
        const int32_t t0 = (int32_t)((uint32_t)tile * TILE); // (a tile behind the longest line's end begins at 2^31: only its place in a page counts)
        {
            const int32_t tok = t0 + k_tok; // its block is the same for the whole wave
            const uint8_t *part = part_of(k_tok < 32 ? page[0] : page[1]);
            const uint8_t *src = part + (tok & (P - 1)) * (D / 2) + D / 8 * k_part;
            if (D == 128) {
                const uint4 w = *reinterpret_cast<const uint4 *>(src);
                x.k[0] = w.x, x.k[1] = w.y, x.k[D / 32 - 2] = w.z, x.k[D / 32 - 1] = w.w;
            } else {
                const uint2 w = *reinterpret_cast<const uint2 *>(src);
                x.k[0] = w.x, x.k[1] = w.y;
            }
            const uint8_t *par = part + P * D + ((k_part & 1) * 2 * P + (tok & (P - 1))) * 4;
            x.alpha = *reinterpret_cast<const float *>(par);
            x.beta = *reinterpret_cast<const int32_t *>(par + 4 * P);
            x.value_alpha = *reinterpret_cast<const float *>(part + P * D + (2 * P + (tok & (P - 1))) * 4);
        }
        {
            const int32_t tok = t0 + v_tok;
            const uint8_t *src = part_of(wave < 2 ? page[0] : page[1]) + (P + (tok & (P - 1))) * (D / 2) + D / 64 * col;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint8_t *w = src + (8 * (e >> 2) + (e & 3)) * (D / 2);
                x.v[e] = D == 128 ? *reinterpret_cast<const uint16_t *>(w) : *w;
            }
        }
    };
    // An alpha that append does not write, in a page of zeros say: the value is 0 whatever its codes, its token weighs as any other.  It
    // goes through the products as alpha 1, zero point 0 and operands 0.  (No logarithm of 0, no infinite reciprocal of a subnormal.)
    const auto is_nothing = [](float value_alpha) { return fabsf(value_alpha) < 0x1p-126f; };
    const auto lay_params = [&](const Asked<D> &x, int32_t b) { // into buffer b
        Operands<D> &o = op[b];
        if (k_part < 2) { // (tokens that no row sees may hold anything: nothing here that is not finite meets a weight of zero)
            float part[3];
            split<3>(k_part == 1 && is_nothing(x.alpha) ? 0.0f : -16.0f - (float)x.beta, part);
            if (k_part == 0) {
                // a factor this small is a key that is zero to every query: 2^-90 in its place keeps the quotient finite
                float ka = x.alpha * a.scale2;
                ka = fabsf(ka) < 0x1p-90f ? copysignf(0x1p-90f, ka) : ka;
                float more[3];
                split<3>(__builtin_amdgcn_logf(is_nothing(x.value_alpha) ? 1.0f : x.value_alpha) / ka, more);
                o.ka[k_tok] = ka;
                *reinterpret_cast<u32x4 *>(&o.k[k_tok][D]) =
                    u32x4{pack_bf16(part[0], part[0]), pack_bf16(part[0], part[1]), pack_bf16(part[1], part[1]), pack_bf16(part[2], part[2])};
                *reinterpret_cast<u32x4 *>(&o.k[k_tok][D + 8]) = u32x4{pack_bf16(part[2], more[0]), pack_bf16(more[1], more[2]), 0, 0};
            } else {
                const int32_t u = k_tok & 15, place = (k_tok & ~15) + (u >> 2 & 1) * 8 + (u >> 3) * 4 + (u & 3);
                float r[3];
                split<3>(is_nothing(x.alpha) ? 1.0f : (x.alpha > 0.0f && x.alpha < INFINITY ? __builtin_amdgcn_rcpf(x.alpha) : 0.0f), r);
#pragma unroll
                for (int i = 0; i < 3; ++i) {
                    o.rows[i][place] = (uint16_t)(__float_as_uint(part[i]) >> 16);
                    o.rows[3 + i][place] = (uint16_t)(__float_as_uint(r[i]) >> 16);
                }
            }
        }
    };
    const auto lay_codes = [&](const Asked<D> &x, int32_t b) {
        Operands<D> &o = op[b];
#pragma unroll
        for (int i = 0; i < D / 32; ++i) *reinterpret_cast<bf16x8 *>(&o.k[k_tok][D / 4 * k_part + 8 * i]) = codes.operand(x.k[i]);
        uint32_t pair[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) pair[e] = x.v[2 * e] | x.v[2 * e + 1] << 16;
        const auto place = [&](int c) { return reinterpret_cast<u32x4 *>(&o.v[32 * c + col][8 * v_chunk]); };
        *place(0) = u32x4{codes.pair<0>(pair[0]), codes.pair<0>(pair[1]), codes.pair<0>(pair[2]), codes.pair<0>(pair[3])};
        *place(1) = u32x4{codes.pair<1>(pair[0]), codes.pair<1>(pair[1]), codes.pair<1>(pair[2]), codes.pair<1>(pair[3])};
        if (D == 128) {
            *place(2) = u32x4{codes.pair<2>(pair[0]), codes.pair<2>(pair[1]), codes.pair<2>(pair[2]), codes.pair<2>(pair[3])};
            *place(D / 32 - 1) = u32x4{codes.pair<3>(pair[0]), codes.pair<3>(pair[1]), codes.pair<3>(pair[2]), codes.pair<3>(pair[3])};
        }
        // the wave lays values of the 16 tokens whose parameters it has, token u of them in lanes 4 u ..
        const uint64_t nothing = __ballot(is_nothing(x.value_alpha));
        if (nothing) {
            u32x4 keep;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int32_t u = 4 * h + 8 * (e >> 1) + 2 * (e & 1);
                keep[e] = (nothing >> (4 * u) & 1 ? 0u : 0xffffu) | (nothing >> (4 * u + 4) & 1 ? 0u : 0xffff0000u);
            }
#pragma unroll 1
            for (int c = 0; c < D / 32; ++c) *place(c) &= keep;
        }
    };

    Asked<D> asked;
    int32_t page[2], next[2], later[2];
    ask(tile_begin + group, asked, page); // on its way while the queries come

    // queries: element e of step k of lane half h is channel 16 k + 8 h + {0, 4, 1, 5, 2, 6, 3, 7}[e]; behind them the parts of their sum
    bf16x8 q[KSTEPS], qz;
    {
        const int64_t from = (int64_t)(t.seq.row + token) * a.ldq + (head * a.group + head_of_row) * D + 8 * h;
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < KSTEPS; ++i) {
            uint32_t d[4] = {0, 0, 0, 0};
            const uint16_t *src = static_cast<const uint16_t *>(a.q) + from + 16 * i;
            if (real && a.q_vec) {
                const uint4 w = *reinterpret_cast<const uint4 *>(src);
                d[0] = w.x, d[1] = w.y, d[2] = w.z, d[3] = w.w;
            } else if (real) {
#pragma unroll
                for (int e = 0; e < 4; ++e) d[e] = src[2 * e] | (uint32_t)src[2 * e + 1] << 16;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) sum += __uint_as_float(d[e] << 16) + __uint_as_float(d[e] & 0xffff0000u);
            q[i] = __builtin_bit_cast(bf16x8, u32x4{__builtin_amdgcn_perm(d[2], d[0], 0x05040100u), __builtin_amdgcn_perm(d[2], d[0], 0x07060302u),
                                                    __builtin_amdgcn_perm(d[3], d[1], 0x05040100u), __builtin_amdgcn_perm(d[3], d[1], 0x07060302u)});
        }
        sum += __shfl_xor(sum, 32);
        float part[3];
        split<3>(sum, part); // z, z, z, z', z', z', z'', z'' | z'' meet q, q', q'', q, q', q'', q, q' | q'', three parts more a one
        qz = h == 0 ? __builtin_bit_cast(bf16x8, u32x4{pack_bf16(part[0], part[1]), pack_bf16(part[2], part[0]), pack_bf16(part[1], part[2]), pack_bf16(part[0], part[1])})
                    : __builtin_bit_cast(bf16x8, u32x4{pack_bf16(part[2], 1.0f), pack_bf16(1.0f, 1.0f), 0, 0});
    }

    // Row (i & 3) + 8 (i >> 2) + 4 h of the shared product is element i of a lane: both halves find the values' zero points in
    // elements 0..2 and the sum of the weights in 3..5.
    const int32_t shared_row = (col & 3) + (col >> 3 == 1 ? 4 : 0);
    f32x16 acc[DT], off;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        off[e] = 0.0f;
#pragma unroll
        for (int i = 0; i < DT; ++i) acc[i][e] = 0.0f;
    }
    float m = -INFINITY;

    const auto work = [&](int32_t tile, int32_t b, bool add, const int32_t (&page)[2]) {
        const Operands<D> &o = op[b];
        const int32_t t0 = tile * TILE;
        f32x16 sc[2];
        const uint16_t *row = &o.k[col][8 * h];
        bf16x8 kk[KSTEPS + 1];
#pragma unroll
        for (int i = 0; i <= KSTEPS; ++i) kk[i] = *reinterpret_cast<const bf16x8 *>(row + 16 * i);
#pragma unroll
        for (int x = 0; x < 2; ++x) {
#pragma unroll
            for (int e = 0; e < 16; ++e) sc[x][e] = 0.0f;
#pragma unroll
            for (int i = 0; i <= KSTEPS; ++i) {
                sc[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kk[i], i < KSTEPS ? q[i] : qz, sc[x], 0, 0, 0);
                if (x == 0) kk[i] = *reinterpret_cast<const bf16x8 *>(row + 32 * o.KS + 16 * i);
            }
        }
        // the reads of the first 32 tokens, then a product and a read of the others in turn, then products alone
        __builtin_amdgcn_sched_group_barrier(0x100, KSTEPS + 1, 0);
#pragma unroll
        for (int i = 0; i <= KSTEPS; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, KSTEPS + 1, 0);
        // log2 of p alpha_v, less m; the maximum follows where that passes SLACK, or where a row has none yet
        const float base = m == -INFINITY ? 0.0f : m;
        float top = -INFINITY;
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float4 ka = *reinterpret_cast<const float4 *>(&o.ka[32 * x + 8 * j + 4 * h]);
                const float f[4] = {ka.x, ka.y, ka.z, ka.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) sc[x][4 * j + i] = __builtin_fmaf(f[i], sc[x][4 * j + i], -base);
            }
        if (t0 < each_lo || t0 + TILE - 1 > each_hi || page[0] < 0 || page[1] < 0) { // some row does not see some token; what lies there may be anything
            int32_t mine = t0 + 4 * h;
            asm volatile("" : "+v"(mine)); // keeps the comparisons in here
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int32_t tok = mine + 32 * x + 8 * (e >> 2) + (e & 3);
                    const bool seen = tok >= lo && tok <= hi && page[x] >= 0;
                    sc[x][e] = seen ? sc[x][e] : -INFINITY;
                }
        }
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int e = 0; e < 16; ++e) top = fmaxf(top, sc[x][e]);
        const bool fresh = m == -INFINITY;
        if (__any(top > SLACK || (fresh && top > -INFINITY))) {
            top = fmaxf(top, __shfl_xor(top, 32));
            const float up = top == -INFINITY ? 0.0f : (fresh ? top : fmaxf(top, 0.0f)), f = fresh ? 1.0f : __builtin_amdgcn_exp2f(-up);
            m = fresh && top == -INFINITY ? m : base + up;
            off *= f;
#pragma unroll
            for (int i = 0; i < DT; ++i) acc[i] *= f;
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int e = 0; e < 16; ++e) sc[x][e] -= up;
        }
        // A product's operand is read while the products of the 16 tokens before are on their way (without: 1 to 2 % more time).
        const auto operand_of = [&](int y, int i) {
            return i == 0 ? *reinterpret_cast<const bf16x8 *>(&o.rows[shared_row][16 * y + 8 * h]) : *reinterpret_cast<const bf16x8 *>(&o.v[32 * (i - 1) + col][16 * y + 8 * h]);
        };
        bf16x8 vv[DT + 1];
#pragma unroll
        for (int i = 0; i <= DT; ++i) vv[i] = operand_of(0, i);
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            float w[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = __builtin_amdgcn_exp2f(sc[y >> 1][8 * (y & 1) + e]);
            bf16x8 p[WPARTS];
            split8<WPARTS>(w, p);
#pragma unroll
            for (int i = 0; i <= DT; ++i) {
#pragma unroll
                for (int j = WPARTS - 1; j >= 0; --j) {
                    if (i == 0) off = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vv[0], p[j], off, 0, 0, 0);
                    else acc[i - 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vv[i], p[j], acc[i - 1], 0, 0, 0);
                }
                if (y < 3) vv[i] = operand_of(y + 1, i);
            }
        }
        __builtin_amdgcn_sched_group_barrier(0x100, DT + 1, 0);
#pragma unroll
        for (int i = 0; i < 3 * (DT + 1); ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, WPARTS, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, WPARTS * (DT + 1), 0);
        if (add) {
            const float zero = off[0] + off[1] + off[2];
#pragma unroll
            for (int i = 0; i < DT; ++i) acc[i] += zero;
            off[0] = off[1] = off[2] = 0.0f;
        }
    };

    lay_params(asked, 0);
    lay_codes(asked, 0);
    ask(tile_begin + group + GROUPS, asked, next); // past the last: page 0, dropped
    __syncthreads();
    for (int32_t i = 0; tile_begin + GROUPS * i < tile_end; ++i) {
        const int32_t b = i & 1, tile = tile_begin + GROUPS * i + group;
        const auto lay = [&] {
            lay_params(asked, 1 - b);
            lay_codes(asked, 1 - b);
            ask(tile + 2 * GROUPS, asked, later);
        };
        if (GROUPS > 1 && group == 1) lay();
        __builtin_amdgcn_s_setprio(1); // laying a tile out gives way to the work of the CU's other waves (1184 -> 1139 us for 2000 tokens behind 14000)
        if (tile <= some_hi >> 6 && tile >= some_lo >> 6) work(tile, b, i % TOGETHER == TOGETHER - 1, page);
        __builtin_amdgcn_s_setprio(0);
        if (GROUPS == 1 || group == 0) lay();
        page[0] = next[0], page[1] = next[1], next[0] = later[0], next[1] = later[1];
        __syncthreads();
    }

    const float zero = off[0] + off[1] + off[2];
    float l = off[3] + off[4] + off[5];
#pragma unroll
    for (int i = 0; i < DT; ++i) acc[i] += zero;
    if (GROUPS > 1) { // the second group's results to the first
        constexpr int Q = DT * 4;
        f32x4 *room = reinterpret_cast<f32x4 *>(&operands[0][0]) + wave * (Q + 1) * 64 + lane;
        static_assert(sizeof(operands) >= WAVES * (Q + 1) * 64 * sizeof(f32x4), "a group's results fit where the operands were");
        if (group == 1) {
#pragma unroll
            for (int i = 0; i < Q; ++i) room[i * 64] = quarter_of(acc[i / 4], i % 4);
            room[Q * 64] = f32x4{m, l, 0.0f, 0.0f};
        }
        __syncthreads();
        if (group == 1) return;
        const f32x4 ml = room[Q * 64];
        const float top = fmaxf(m, ml[0]), base = top == -INFINITY ? 0.0f : top, f = __builtin_amdgcn_exp2f(m - base), g = __builtin_amdgcn_exp2f(ml[0] - base);
        l = f * l + g * ml[1], m = top;
#pragma unroll
        for (int i = 0; i < Q; ++i) {
            const f32x4 o = room[i * 64];
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i / 4][i % 4 * 4 + e] = f * acc[i / 4][i % 4 * 4 + e] + g * o[e];
        }
    }
    if (span.parts > 1) {
        const int64_t to = part_at(a, head, k_tile, part, wave);
        f32x4 *o = reinterpret_cast<f32x4 *>(a.part_o) + to * (DT * 4) * 64 + lane;
#pragma unroll
        for (int i = 0; i < DT * 4; ++i) o[i * 64] = quarter_of(acc[i % DT], i / DT);
        a.part_ml[to * 64 + lane] = make_float2(m, l);
        return;
    }
    if (!real) return;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        f32x4 x[DT];
#pragma unroll
        for (int c = 0; c < DT; ++c) x[c] = quarter_of(acc[c], k);
        put_quarter<D, F32O>(a, head, t.seq.row + token, head_of_row, k, x, l);
    }
}

// The parts of a tile joined, a workgroup for a quarter of its channels: every wave its 32 rows, lanes as in the products.
template <int D, bool F32O>
__global__ __launch_bounds__(THREADS) void join_prompts_kernel(const AttendArgs a)
{
    constexpr int DT = D / 32;
    const int32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int32_t head = blockIdx.x % a.s.heads, k_tile = blockIdx.x / a.s.heads, quarter = blockIdx.y;
    Tile t;
    if (!tile_at(a, k_tile, &t)) return;
    const int32_t tok0 = (int32_t)((uint32_t)t.first / (uint32_t)a.group), head0 = t.first - tok0 * a.group;
    const Span span = span_of(a, sight_of(a, t, tok0, head0, PROWS));
    if (span.parts <= 1) return;
    const int64_t from = part_at(a, head, k_tile, 0, wave);
    const float2 *ml = a.part_ml + from * 64 + lane;
    const f32x4 *o = reinterpret_cast<const f32x4 *>(a.part_o) + (from * 4 + quarter) * DT * 64 + lane;
    float top = -INFINITY, l = 0.0f;
    for (int32_t p = 0; p < span.parts; ++p) top = fmaxf(top, ml[p * WAVES * 64].x);
    if (top == -INFINITY) top = 0.0f;
    f32x4 x[DT];
#pragma unroll
    for (int c = 0; c < DT; ++c) x[c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int32_t p = 0; p < span.parts; ++p) {
        const float f = __builtin_amdgcn_exp2f(ml[p * WAVES * 64].x - top);
        l += f * ml[p * WAVES * 64].y;
#pragma unroll
        for (int c = 0; c < DT; ++c) x[c] += f * o[(p * WAVES * 4 * DT + c) * 64];
    }
    const int32_t n = wave * 32 + (lane & 31), token = tok0 + (int32_t)a.by_group.divide((uint32_t)(head0 + n));
    if (t.first + n < t.rows) put_quarter<D, F32O>(a, head, t.seq.row + token, head0 + n - (token - tok0) * a.group, quarter, x, l);
}

} // namespace

QllmKvPrompts qllm_kv_plan_prompts(const qllm_kv_batch &batch, int64_t heads, int64_t group, int64_t dim, int64_t tokens)
{
    QllmKvPrompts n;
    const int64_t rows = batch.rows * group, tiles = batch.n_seqs == 1 ? (rows + PROWS - 1) / PROWS : rows / PROWS + batch.n_seqs; // at most
    n.workgroups = tiles * heads;
    n.groups = n.workgroups <= 2 * 256 ? 2 : 1;
    n.parts = n.workgroups > 0 && n.workgroups <= 128 && tokens >= 1280 ? 256 / n.workgroups : 1;
    if (n.parts > 32) n.parts = 32;
    n.sums = n.parts > 1 ? n.workgroups * n.parts * PROWS * dim * (int64_t)sizeof(float) : 0;
    n.bytes = n.parts > 1 ? n.sums + n.workgroups * n.parts * WAVES * 64 * (int64_t)sizeof(float2) : 0;
    return n;
}

int32_t qllm_kv_launch_prompts(const AttendArgs &args, const QllmKvPrompts &n, int64_t dim, int32_t out_dtype, void *workspace, hipStream_t stream)
{
    AttendArgs a = args;
    a.parts = (int32_t)n.parts;
    a.part_o = static_cast<float *>(workspace);
    a.part_ml = reinterpret_cast<float2 *>(static_cast<uint8_t *>(workspace) + n.sums);
    const dim3 grid((unsigned)(n.workgroups * n.parts)), tiles((unsigned)n.workgroups, 4);
#define QLLM_PROMPTS(D, FO)                                                                                     \
    do {                                                                                                        \
        if (n.groups == 2) hipLaunchKernelGGL((prompts_kernel<D, FO, 2>), grid, dim3(2 * THREADS), 0, stream, a); \
        else hipLaunchKernelGGL((prompts_kernel<D, FO, 1>), grid, dim3(THREADS), 0, stream, a);                 \
        if (n.parts > 1) hipLaunchKernelGGL((join_prompts_kernel<D, FO>), tiles, dim3(THREADS), 0, stream, a);  \
    } while (0)
    if (dim == 128) {
        if (out_dtype == QLLM_F32) QLLM_PROMPTS(128, true);
        else QLLM_PROMPTS(128, false);
    } else {
        if (out_dtype == QLLM_F32) QLLM_PROMPTS(64, true);
        else QLLM_PROMPTS(64, false);
    }
#undef QLLM_PROMPTS
    return launched("cache attention of prompts: launch");
}
