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

struct Unfinished;
struct AttendArgs {
    Step s;
    const void *q;
    void *out;
    int64_t ldq, ldo;
    int32_t q_heads, group, window; // window 0: none
    float scale2;                   // scale * log2 e
    int32_t blocks;                 // workgroups of a kv head
    float *part_o;                  // their partial results, see partial_at
    float2 *part_ml;
    Unfinished *unfinished;   // [heads][blocks]
};

__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}

// 16 + code of nibble i (0..3) of both halves of w, as a pair of bf16.  The two constants are kept in registers, unknown to the
// compiler: only then are "and" and "or" one instruction (a literal for each makes them two).
struct Codes16 {
    uint32_t mask, sixteen;
    __device__ __forceinline__ Codes16()
    {
        asm("v_mov_b32 %0, 0x780078" : "=v"(mask));
        asm("v_mov_b32 %0, 0x41804180" : "=v"(sixteen));
    }
    template <int I>
    __device__ __forceinline__ uint32_t pair(uint32_t w) const
    {
        const uint32_t t = I == 0 ? w << 3 : w >> (4 * I - 3);
        return (t & mask) | sixteen;
    }
    // 8 codes of a dword as a matrix-core operand: elements are codes 0, 4, 1, 5, 2, 6, 3, 7
    __device__ __forceinline__ bf16x8 operand(uint32_t w) const
    {
        return __builtin_bit_cast(bf16x8, u32x4{pair<0>(w), pair<1>(w), pair<2>(w), pair<3>(w)});
    }
};

// A row tile of a workgroup: rows first .. first + 15 of a sequence's n * group rows.
struct Tile {
    Seq seq;
    int32_t first, rows;
};

// What rows see: tokens all_lo .. all_hi some of them, each_lo .. each_hi every one.
struct Sight {
    int32_t limit, all_lo, all_hi, each_lo, each_hi;
};

__device__ __forceinline__ int32_t lo_at(const AttendArgs &a, int32_t pos) { return a.window > 0 && pos - a.window + 1 > 0 ? pos - a.window + 1 : 0; }
__device__ __forceinline__ int32_t hi_at(int32_t limit, int32_t pos) { return pos < limit ? pos : limit - 1; }
__device__ __forceinline__ int32_t limit_of(const AttendArgs &a, const Seq &q)
{
    const int32_t cap = a.s.table_ld << a.s.page_shift;
    return q.line < 0 ? 0 : (q.len < cap ? q.len : cap);
}

__device__ __forceinline__ Sight sight_of(const AttendArgs &a, const Tile &t)
{
    Sight v;
    v.limit = limit_of(a, t.seq);
    const int32_t last_row = t.first + ROWS < t.rows ? t.first + ROWS - 1 : t.rows - 1;
    const int32_t p_first = t.seq.len - t.seq.n + t.first / a.group, p_last = t.seq.len - t.seq.n + last_row / a.group;
    v.all_lo = lo_at(a, p_first), v.all_hi = hi_at(v.limit, p_last);
    v.each_lo = lo_at(a, p_last), v.each_hi = hi_at(v.limit, p_first);
    return v;
}

// The work of a kv head is one long line of steps: sequence after sequence, tile after tile, `steps` of 32 tokens for each tile
// (what its sequence's rows see together; at least one, for rows that see nothing get their zeros too).  The workgroups of the
// head share the line out evenly, whatever the lengths: one may end in the middle of a tile and the next go on there.
struct Work {
    int32_t tiles, first, steps; // of a sequence; its first step is number `first` of the cache line
    // (a bound that only a row_start that does not ascend can reach: 2^20 of these still add up)
    __device__ __forceinline__ int64_t all() const { return min((int64_t)tiles * steps, (int64_t)1 << 42); }
};

__device__ __forceinline__ Work work_of(const AttendArgs &a, const Seq &q)
{
    Work w;
    w.tiles = (int32_t)(((int64_t)q.n * a.group + ROWS - 1) / ROWS);
    const int32_t lo = lo_at(a, q.len - q.n), hi = hi_at(limit_of(a, q), q.len - 1);
    w.first = lo / STEP;
    w.steps = hi < lo ? 1 : hi / STEP + 1 - w.first;
    return w;
}

__device__ __forceinline__ int64_t lane64(int64_t x, int32_t lane) // lane `lane`'s x, the same in every lane and known to be
{
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int32_t)((uint64_t)x >> 32), lane) << 32 |
                     (uint32_t)__builtin_amdgcn_readlane((int32_t)x, lane));
}

// The line as one wave sees it: 64 sequences at a time, one a lane.  Up to 64 are read from memory once.
struct Line {
    Seq mine;      // sequence base + lane
    int64_t upto;  // where it ends
    int64_t total; // the whole line
    int32_t base;

    __device__ __forceinline__ void look(const AttendArgs &a, int32_t from, int64_t before)
    {
        const int32_t lane = threadIdx.x & 63, i = from + lane;
        base = from;
        mine = Seq{0, 0, -1, 0};
        if (i < a.s.n_seqs) mine = seq_of(a.s, i);
        upto = work_of(a, mine).all(); // none without rows
        if (i >= a.s.n_seqs) upto = 0;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int64_t y = __shfl_up(upto, o);
            if (lane >= o) upto += y;
        }
        upto += before;
    }
    __device__ __forceinline__ explicit Line(const AttendArgs &a)
    {
        total = 0;
        for (int32_t from = 0; from < a.s.n_seqs; from += 64) {
            look(a, from, total);
            total = lane64(upto, 63);
        }
        if (total >= (int64_t)1 << 50) total = 0; // see Work::all
    }
    // The sequence that step `at` < total belongs to; *begin: where that begins.
    __device__ __forceinline__ int32_t find(const AttendArgs &a, int64_t at, int64_t *begin)
    {
        int64_t before = 0;
        for (int32_t from = 0; from < a.s.n_seqs; from += 64) {
            if (a.s.n_seqs > 64) look(a, from, before);
            const int32_t skipped = __popcll(__ballot(upto <= at)); // sequences that end at or before it
            if (skipped < 64) {
                *begin = skipped ? lane64(upto, skipped - 1) : before;
                return from + skipped;
            }
            before = lane64(upto, 63);
        }
        return a.s.n_seqs;
    }
    __device__ __forceinline__ Seq seq(const AttendArgs &a, int32_t i)
    {
        if (i < base || i >= base + 64) look(a, i, 0); // only its sequences are asked for from now on
        const int32_t k = i - base;
        return Seq{__builtin_amdgcn_readlane(mine.row, k), __builtin_amdgcn_readlane(mine.n, k), __builtin_amdgcn_readlane(mine.line, k),
                   __builtin_amdgcn_readlane(mine.len, k)};
    }
};

// How many workgroups share the line: none gets less than LEAST steps while another has some.  Share b begins at total * b / of.
constexpr int LEAST = 16;
__device__ __forceinline__ int32_t sharers(const AttendArgs &a, int64_t total)
{
    const int64_t most = (total + LEAST - 1) / LEAST;
    return most < a.blocks ? (int32_t)most : a.blocks;
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

// What a wave asks of memory for one step: codes of its keys (tokens 16 h + r, channels D / 4 g ..) and values (tokens of
// element e, channels D / 16 r ..), and one token's alpha and beta, of the keys in lanes 0..31, of the values in the others.
template <int D>
struct Loaded {
    uint32_t k[2][D / 32], v[8], beta;
    float alpha;
    int32_t t0; // its first token, -1: nothing
};

template <int D>
__device__ __forceinline__ void ask(const Step &s, int32_t head, int32_t lane, int32_t page, int32_t t0, Loaded<D> &x)
{
    const int32_t P = 1 << s.page_shift, r = lane & 15, g = lane >> 4, in_page = t0 & (P - 1);
    const uint8_t *part = s.pages + page * s.page_bytes + (int64_t)head * P * (D + 16);
    const uint8_t *kc = part + (int64_t)in_page * (D / 2), *vc = kc + (int64_t)P * (D / 2);
    x.t0 = t0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint8_t *src = kc + (16 * h + r) * (D / 2) + D / 8 * g;
        if (D == 128) {
            const uint4 w = *reinterpret_cast<const uint4 *>(src);
            x.k[h][0] = w.x, x.k[h][1] = w.y, x.k[h][D / 32 - 2] = w.z, x.k[h][D / 32 - 1] = w.w;
        } else {
            const uint2 w = *reinterpret_cast<const uint2 *>(src);
            x.k[h][0] = w.x, x.k[h][1] = w.y;
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint8_t *src = vc + (16 * (e >> 2) + 4 * g + (e & 3)) * (D / 2) + D / 32 * r;
        x.v[e] = D == 128 ? *reinterpret_cast<const uint32_t *>(src) : *reinterpret_cast<const uint16_t *>(src);
    }
    const uint32_t *par = reinterpret_cast<const uint32_t *>(part + (int64_t)P * D) + (lane >> 5) * 2 * P + in_page + (lane & 31);
    x.alpha = __uint_as_float(par[0]);
    x.beta = par[P];
}

// A workgroup leaves at most two tiles unfinished: the one it begins with (slot 0) and the one it ends with (slot 1).  Per row:
// running maximum and sum, and dim unnormalised sums.
struct Unfinished { // a tile whose first steps a workgroup has and whose last it has not; parts 0: there is none
    int32_t parts, slot, row, first, rows, pad[3];
};
__device__ __forceinline__ int64_t partial_at(const AttendArgs &a, int32_t head, int32_t block, int32_t slot, int32_t row)
{
    return (((int64_t)head * a.blocks + block) * 2 + slot) * ROWS + row;
}

template <int D, bool F32O>
__device__ __forceinline__ void put_out(const AttendArgs &a, const Tile &t, int32_t head, int32_t row, int32_t c, float y)
{
    const int32_t tok = row / a.group;
    const int64_t at = (int64_t)(t.seq.row + tok) * a.ldo + (int64_t)(head * a.group + row - tok * a.group) * D + c;
    if (F32O) static_cast<float *>(a.out)[at] = y;
    else static_cast<uint16_t *>(a.out)[at] = (uint16_t)pack_bf16(y, 0.0f);
}

__device__ __forceinline__ float quotient(float o, float sum) { return sum > 0.0f ? o / sum : (sum == 0.0f ? 0.0f : sum); } // a NaN stays

template <int D, bool F32Q, bool F32O>
__global__ __launch_bounds__(WAVES * 64, F32Q ? 2 : 3) void attend_kernel(const AttendArgs a)
{
    constexpr int PARTS = F32Q ? 3 : 1;
    constexpr int KS = D / 32, DT = D / 16; // steps of 32 channels; tiles of 16 channels (one channel of each lane row)
    __shared__ float mrg_m[WAVES][ROWS], mrg_l[WAVES][ROWS], mrg_o[WAVES][ROWS][D + 4];
    // a token's parameters, worked out by one lane and read by sixteen: a key's factor and 16 + beta, a value's alpha and - (16 + beta)
    __shared__ __attribute__((aligned(16))) float2 params[WAVES][64];

    const Step &s = a.s;
    const int32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int32_t head = blockIdx.y;
    Line line(a);
    const int32_t of = sharers(a, line.total), block = blockIdx.x;
    Unfinished left = {};
    if (block >= of) {
        if (threadIdx.x == 0) a.unfinished[head * a.blocks + block] = left;
        return;
    }
    const int64_t begin = line.total * block / of, end = line.total * (block + 1) / of;
    const Codes16 codes;
    const float factor = lane < 32 ? a.scale2 : 1.0f, sign = lane < 32 ? 1.0f : -1.0f, exact = lane < 32 ? INFINITY : 256.0f;

    int64_t at = begin, seq_begin = 0;
    int32_t i_seq = line.find(a, begin, &seq_begin);
    while (at < end && i_seq < s.n_seqs) {
    Tile t;
    t.seq = line.seq(a, i_seq);
    const Work work_here = work_of(a, t.seq);
    if (at - seq_begin >= work_here.all()) { // on to the next sequence
        seq_begin += work_here.all(), ++i_seq;
        continue;
    }
    const int64_t number = (at - seq_begin) / work_here.steps;
    const int32_t skip = (int32_t)(at - seq_begin - number * work_here.steps);
    const int32_t take = work_here.steps - skip < end - at ? work_here.steps - skip : (int32_t)(end - at);
    t.first = (int32_t)number * ROWS, t.rows = t.seq.n * a.group;
    const Sight v = sight_of(a, t);
    const int32_t step_begin = work_here.first + skip;
    const int32_t step_end = v.all_hi < 0 || step_begin + take <= v.all_hi / STEP + 1 ? step_begin + take : v.all_hi / STEP + 1;
    const bool whole = take == work_here.steps;
    const int32_t slot = at == begin ? 0 : 1;
    if (skip == 0 && !whole) { // the shares up to the one in which the tile's last step lies
        const int64_t last = at + work_here.steps - 1;
        int32_t b = (int32_t)(last * of / line.total);
        if (b + 1 < of && line.total * (b + 1) / of <= last) ++b;
        left = Unfinished{b - block + 1, slot, t.seq.row, t.first, t.rows, {}};
    }
    at += take;

    // this lane's row (a column of the transposed products) and the tokens it sees: lo .. hi
    const int32_t row = t.first + r, token = row / a.group;
    const bool real = row < t.rows;
    const int32_t pos = t.seq.len - t.seq.n + token, hi = real ? hi_at(v.limit, pos) : -1, lo = lo_at(a, pos);

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
    float m = -INFINITY, l = 0.0f; // running maximum; this lane's part of the sum of p

    const auto work = [&](const Loaded<D> &x) {
        const float zero = sign * ((float)(int32_t)x.beta + 16.0f);
        params[wave][lane] = make_float2(x.alpha * factor, zero);
        const bool far = __any(fabsf(zero) > exact); // some - (16 + beta) of a value has more than the 8 bits of a bf16
        __builtin_amdgcn_wave_barrier();
        float sc[8], va[8], vz[8]; // scores, the values' alpha and - (16 + beta), of tokens 16 h + 4 g + i
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            f32x4 d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = PARTS - 1; i >= 0; --i)
#pragma unroll
                for (int k = 0; k < KS; ++k) d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes.operand(x.k[h][k]), qo[i][k], d, 0, 0, 0);
            const float4 *kp = reinterpret_cast<const float4 *>(&params[wave][16 * h + 4 * g]), *vp = kp + STEP / 2;
            const float4 k0 = kp[0], k1 = kp[1], v0 = vp[0], v1 = vp[1];
            const float ka[4] = {k0.x, k0.z, k1.x, k1.z}, kb[4] = {k0.y, k0.w, k1.y, k1.w};
            va[4 * h] = v0.x, va[4 * h + 1] = v0.z, va[4 * h + 2] = v1.x, va[4 * h + 3] = v1.z;
            vz[4 * h] = v0.y, vz[4 * h + 1] = v0.w, vz[4 * h + 2] = v1.y, vz[4 * h + 3] = v1.w;
#pragma unroll
            for (int i = 0; i < 4; ++i) sc[4 * h + i] = ka[i] * __builtin_fmaf(-kb[i], qsum, d[i]);
        }
        if (x.t0 < v.each_lo || x.t0 + STEP - 1 > v.each_hi) { // some row does not see some token; what lies there may be anything
            int32_t t0 = x.t0 + 4 * g;
            asm volatile("" : "+v"(t0)); // keeps the comparisons in here
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int32_t tok = t0 + 16 * (i >> 2) + (i & 3);
                const bool seen = tok >= lo && tok <= hi;
                sc[i] = seen ? sc[i] : -INFINITY;
                va[i] = seen ? va[i] : 0.0f;
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
            m = now, l *= f;
#pragma unroll
            for (int i = 0; i < DT; ++i) acc[i] *= f;
        }
        const float base = m == -INFINITY ? 0.0f : m;
        float part_p[8][PARTS];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float p = __builtin_amdgcn_exp2f(sc[i] - base);
            l += p;
            split<PARTS>(p * va[i], part_p[i]);
        }
        bf16x8 pw[PARTS];
#pragma unroll
        for (int j = 0; j < PARTS; ++j)
            pw[j] = __builtin_bit_cast(bf16x8, u32x4{pack_bf16(part_p[0][j], part_p[1][j]), pack_bf16(part_p[2][j], part_p[3][j]),
                                                     pack_bf16(part_p[4][j], part_p[5][j]), pack_bf16(part_p[6][j], part_p[7][j])});
        uint32_t low[4], high[4]; // codes 0..3 and 4..7 of two neighbouring tokens
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            low[e] = __builtin_amdgcn_perm(x.v[2 * e + 1], x.v[2 * e], 0x05040100u);
            high[e] = __builtin_amdgcn_perm(x.v[2 * e + 1], x.v[2 * e], 0x07060302u);
        }
        // (16 + c) - (16 + beta) in two products: the sums stay as small as the values are, whatever the number of tokens
        const auto high_halves = [&] { // of - (16 + beta): the number itself where it has 8 bits
            u32x4 y;
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = __builtin_amdgcn_perm(__float_as_uint(vz[2 * e + 1]), __float_as_uint(vz[2 * e]), 0x07060302u);
            return __builtin_bit_cast(bf16x8, y);
        };
        const bf16x8 zero0 = high_halves();
        const auto tile = [&](int i, bf16x8 c) {
#pragma unroll
            for (int j = PARTS - 1; j >= 0; --j) {
                acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(zero0, pw[j], acc[i], 0, 0, 0);
                acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(c, pw[j], acc[i], 0, 0, 0);
            }
        };
        const auto four = [&](const uint32_t (&w)[4], int at) {
            tile(at + 0, __builtin_bit_cast(bf16x8, u32x4{codes.pair<0>(w[0]), codes.pair<0>(w[1]), codes.pair<0>(w[2]), codes.pair<0>(w[3])}));
            tile(at + 1, __builtin_bit_cast(bf16x8, u32x4{codes.pair<1>(w[0]), codes.pair<1>(w[1]), codes.pair<1>(w[2]), codes.pair<1>(w[3])}));
            tile(at + 2, __builtin_bit_cast(bf16x8, u32x4{codes.pair<2>(w[0]), codes.pair<2>(w[1]), codes.pair<2>(w[2]), codes.pair<2>(w[3])}));
            tile(at + 3, __builtin_bit_cast(bf16x8, u32x4{codes.pair<3>(w[0]), codes.pair<3>(w[1]), codes.pair<3>(w[2]), codes.pair<3>(w[3])}));
        };
        four(low, 0);
        if (D == 128) four(high, DT - 4);
        if (far) { // values far from zero for their range: what the high halves leave out
#pragma unroll
            for (int k = 0; k < 2; ++k) {
#pragma unroll
                for (int e = 0; e < 8; ++e) vz[e] -= __uint_as_float(__float_as_uint(vz[e]) & 0xffff0000u);
                const bf16x8 rest = high_halves();
#pragma unroll
                for (int i = 0; i < DT; ++i)
#pragma unroll
                    for (int j = PARTS - 1; j >= 0; --j) acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(rest, pw[j], acc[i], 0, 0, 0);
            }
        }
    };

    // The loads of a step are on their way while the step before is worked on.  Nothing in between may wait for memory or hang on
    // a condition that the compiler cannot see through: the page numbers of up to 64 steps are fetched beforehand, one a lane,
    // and a step without a page reads page 0 and drops it.
    const auto ask_for = [&](int32_t page, int32_t st, Loaded<D> &x) { ask<D>(s, head, lane, page < 0 ? 0 : page, st * STEP, x); };
    for (int32_t first = step_begin + wave; first < step_end; first += 64 * WAVES) {
        const int32_t mine = first + lane * WAVES;
        const int32_t pages = mine < step_end ? page_of(s, t.seq.line, mine * STEP) : -1;
        const int32_t left = (step_end - first + WAVES - 1) / WAVES, count = left < 64 ? left : 64;
        Loaded<D> x[2];
        int32_t page = __builtin_amdgcn_readlane(pages, 0);
        ask_for(page, first, x[0]);
        for (int32_t n = 0; n < count; n += 2) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int32_t next = n + i + 1 < count ? __builtin_amdgcn_readlane(pages, (n + i + 1) & 63) : -1;
                ask_for(next, first + (n + i + 1) * WAVES, x[1 - i]);
                if (page >= 0) work(x[i]);
                page = next;
            }
        }
    }

    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    // accumulator i of tile c is channel (D / 16) (4 g + i) + c of this lane's row
    if (g == 0) mrg_m[wave][r] = m, mrg_l[wave][r] = l;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < DT; ++c) mrg_o[wave][r][DT * (4 * g + i) + c] = acc[c][i];
    __syncthreads();
    for (int32_t i = threadIdx.x; i < ROWS * D; i += WAVES * 64) {
        const int32_t n = i / D, c = i % D, rw = t.first + n;
        if (rw >= t.rows) break;
        float top = -INFINITY, sum = 0.0f, o = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) top = fmaxf(top, mrg_m[w][n]);
        const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float f = __builtin_amdgcn_exp2f(mrg_m[w][n] - base);
            sum += f * mrg_l[w][n];
            o += f * mrg_o[w][n][c];
        }
        if (whole) {
            put_out<D, F32O>(a, t, head, rw, c, quotient(o, sum));
        } else {
            const int64_t at = partial_at(a, head, block, slot, n);
            a.part_o[at * D + c] = o;
            if (c == 0) a.part_ml[at] = make_float2(top, sum);
        }
    }
    __syncthreads(); // before the next tile's results
    }
    if (threadIdx.x == 0) a.unfinished[head * a.blocks + block] = left;
}

// The parts of unfinished tiles joined, a workgroup for each that may have begun one: a row's parts are dealt out to as many
// waves as JOIN_WAVES have for each row.
constexpr int JOIN_WAVES = 16;
template <int D, bool F32O>
__global__ __launch_bounds__(JOIN_WAVES * 64) void join_kernel(const AttendArgs a)
{
    __shared__ float sums[JOIN_WAVES], os[JOIN_WAVES][D];
    const int32_t head = blockIdx.y, block = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const Unfinished u = a.unfinished[head * a.blocks + block];
    const int32_t parts = u.parts;
    if (parts == 0) return;
    Tile t;
    t.seq.row = u.row, t.first = u.first, t.rows = u.rows;
    const int32_t rows = t.rows - t.first < ROWS ? t.rows - t.first : ROWS;
    const int32_t lanes_of_rows = rows <= 1 ? 1 : 1 << (32 - __clz(rows - 1)), per_row = JOIN_WAVES / lanes_of_rows;
    const int32_t n = wave % lanes_of_rows, chunk = wave / lanes_of_rows;
    float top = -INFINITY, sum = 0.0f, o[D / 64] = {};
    const auto partial = [&](int32_t p) { return partial_at(a, head, block + p, p == 0 ? u.slot : 0, n); };
    if (n < rows) {
        for (int32_t p = lane; p < parts; p += 64) top = fmaxf(top, a.part_ml[partial(p)].x);
#pragma unroll
        for (int x = 32; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor(top, x));
        const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll 4
        for (int32_t p = chunk; p < parts; p += per_row) {
            const int64_t from = partial(p);
            const float2 ml = a.part_ml[from];
            const float f = __builtin_amdgcn_exp2f(ml.x - base);
            sum += f * ml.y;
#pragma unroll
            for (int c = 0; c < D / 64; ++c) o[c] += f * a.part_o[from * D + 64 * c + lane];
        }
    }
    if (lane == 0) sums[wave] = sum;
#pragma unroll
    for (int c = 0; c < D / 64; ++c) os[wave][64 * c + lane] = o[c];
    __syncthreads();
    if (wave < rows) { // row `wave`
        float all = 0.0f;
        for (int32_t k = 0; k < per_row; ++k) all += sums[wave + k * lanes_of_rows];
#pragma unroll
        for (int c = 0; c < D / 64; ++c) {
            float y = 0.0f;
            for (int32_t k = 0; k < per_row; ++k) y += os[wave + k * lanes_of_rows][64 * c + lane];
            put_out<D, F32O>(a, t, head, t.first + wave, 64 * c + lane, quotient(y, all));
        }
    }
}

int32_t check(const qllm_kv_cache *cache, const qllm_kv_batch *batch, int64_t q_heads)
{
    if (q_heads <= 0 || q_heads > (1 << 16) || q_heads % cache->heads || cache->heads > 65535) return QLLM_ERR_SHAPE;
    if (batch->rows * (q_heads / cache->heads) + batch->n_seqs > INT32_MAX) return QLLM_ERR_SHAPE;
    return QLLM_OK;
}

// Workgroups of a kv head: as many as the card holds at once (three on each of 256 CUs), but none for less than LEAST steps.
int32_t blocks_of(const qllm_kv_cache *cache, const qllm_kv_batch *batch, int64_t q_heads)
{
    constexpr int64_t RESIDENT = 768;
    const int64_t group = q_heads / cache->heads;
    const int64_t tiles = batch->row_start ? batch->rows * group / ROWS + batch->n_seqs : batch->n_seqs * ((group + ROWS - 1) / ROWS);
    const int64_t most = tiles * (batch->table_ld * cache->page_tokens / STEP) / LEAST + 1; // below 2^62
    const int64_t blocks = cache->heads < RESIDENT ? RESIDENT / cache->heads : 1;
    return (int32_t)(blocks < most ? blocks : most);
}

} // namespace

extern "C" int64_t qllm_kv_attention_workspace_bytes(const qllm_kv_cache *cache, const qllm_kv_batch *batch, int64_t q_heads)
{
    Step s;
    int32_t rc = prepare_step(cache, batch, false, &s);
    if (rc == QLLM_OK) rc = check(cache, batch, q_heads);
    if (rc != QLLM_OK) return rc;
    return cache->heads * blocks_of(cache, batch, q_heads) * (2 * ROWS * (cache->dim + 2) * (int64_t)sizeof(float) + (int64_t)sizeof(Unfinished));
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
    a.blocks = blocks_of(cache, batch, q_heads);
    const int64_t parts = cache->heads * a.blocks;
    a.unfinished = static_cast<Unfinished *>(workspace);
    a.part_ml = reinterpret_cast<float2 *>(a.unfinished + parts);
    a.part_o = reinterpret_cast<float *>(a.part_ml + parts * 2 * ROWS);
    const dim3 grid((unsigned)a.blocks, (unsigned)cache->heads);
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
    rc = launched("cache attention: launch");
    if (rc != QLLM_OK || a.blocks == 1) return rc; // one workgroup a head finishes what it begins
    const dim3 cuts((unsigned)a.blocks, (unsigned)cache->heads);
    if (cache->dim == 128 && out_dtype == QLLM_F32) hipLaunchKernelGGL((join_kernel<128, true>), cuts, dim3(JOIN_WAVES * 64), 0, stream, a);
    else if (cache->dim == 128) hipLaunchKernelGGL((join_kernel<128, false>), cuts, dim3(JOIN_WAVES * 64), 0, stream, a);
    else if (out_dtype == QLLM_F32) hipLaunchKernelGGL((join_kernel<64, true>), cuts, dim3(JOIN_WAVES * 64), 0, stream, a);
    else hipLaunchKernelGGL((join_kernel<64, false>), cuts, dim3(JOIN_WAVES * 64), 0, stream, a);
    return launched("cache attention: parts joined");
}
