// Causal attention over the 4-bit key/value cache: the kernel for single tokens and few rows, which is bound by memory, and the
// entry points (kv_attend.h has the formulas).  64 single tokens of 32 heads behind 2000 each read 590 MB, 118 us of 125 at 5.0 TB/s
// (a large copy: 5.2); sixteen of 8 heads behind 1000 to 8000 85 MB, 24 us and 5 more to join; one of 8 heads behind 131000 151 MB,
// 34 us and 5.  A wave has whole steps of loads in flight while it works on another (VGPRs for three workgroups a CU); with one, or
// with four workgroups and half a step, 142 us for the first.
#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include "kv_attend.h"

namespace {

using namespace qllm_kv_detail;

constexpr int ROWS = 16, STEP = 32, WAVES = 4; // rows of a tile, tokens of a step, waves of a workgroup
// The work of a kv head is one long line of steps: sequence after sequence, tile after tile, `steps` for each tile: first BESIDE
// empty ones, the time that a tile takes whatever its length (its queries, the first loads, the waves' results put together), then
// one for every 32 tokens (of what its sequence's rows see together).  The workgroups of the head share the line out evenly,
// whatever the lengths: one may end in the middle of a tile and the next go on there.  (Chunks of 0 to 260 rows mixed with single
// tokens, float32, BESIDE 0, 4, 8, 16: 55, 52, 46, 48 us; single tokens behind 3000 to 20000: no difference.)
constexpr int BESIDE = 8;
struct Work {
    int32_t tiles, first, steps; // of a sequence; its first step with tokens is number `first` of the cache line
};

__device__ __forceinline__ Work work_of(const AttendArgs &a, const Seq &q)
{
    Work w;
    const int32_t rows = q.n * a.group; // checked on the host
    w.tiles = rows > a.few ? 0 : (int32_t)(((uint32_t)rows + ROWS - 1) / ROWS);
    const int32_t lo = lo_at(a, q.len - q.n), hi = hi_at(limit_of(a, q), q.len - 1);
    w.first = lo / STEP;
    w.steps = BESIDE + (hi < lo ? 0 : hi / STEP + 1 - w.first);
    return w;
}

// The line, 64 sequences at a time, one a lane.  Up to LISTED are read from memory once and kept in LDS: by every wave for itself
// where they are 64 (all write the same there, before they read), else by the workgroup's waves in turn.  The host checks that a
// line stays below 2^31 steps; sums saturate, for a row_start that does not ascend.  (256 single tokens behind 1000, 8 heads of 8: 84 us,
// 91 us with every wave reading all sequences again and again.)
constexpr int LISTED = 512;
struct Listed {
    Seq seq;
    int32_t upto; // where it ends in its 64 sequences' part of the line
};
struct Line {
    Listed *list;      // [LISTED]
    int32_t *part;     // [LISTED / 64] steps of 64 sequences
    int32_t total;

    static __device__ __forceinline__ Listed look(const AttendArgs &a, int32_t from)
    {
        const int32_t lane = threadIdx.x & 63, i = from + lane;
        Listed x;
        x.seq = Seq{0, 0, -1, 0};
        if (i < a.s.n_seqs) x.seq = seq_of(a.s, i);
        const Work w = work_of(a, x.seq); // without rows: no tiles
        x.upto = w.tiles * w.steps;
        for (int32_t o = 1; o < 64 && o < a.s.n_seqs; o <<= 1) {
            const int32_t y = __shfl_up(x.upto, o);
            if (lane >= o) x.upto = __builtin_elementwise_add_sat(x.upto, y);
        }
        return x;
    }
    static __device__ __forceinline__ int32_t last_of(const AttendArgs &a, int32_t from) { return a.s.n_seqs - from < 64 ? a.s.n_seqs - from - 1 : 63; }

    __device__ __forceinline__ Line(const AttendArgs &a, Listed *room, int32_t *parts) : list(room), part(parts), total(0)
    {
        const int32_t lane = threadIdx.x & 63, n = a.s.n_seqs;
        if (n <= 64) {
            const Listed x = look(a, 0);
            list[lane] = x;
            total = __builtin_amdgcn_readlane(x.upto, last_of(a, 0));
            part[0] = total;
            __builtin_amdgcn_wave_barrier();
        } else if (n <= LISTED) {
            for (int32_t from = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * 64; from < n; from += WAVES * 64) {
                const Listed x = look(a, from);
                list[from + lane] = x;
                part[from / 64] = __builtin_amdgcn_readlane(x.upto, last_of(a, from));
            }
            __syncthreads();
            for (int32_t from = 0; from < n; from += 64) total = __builtin_elementwise_add_sat(total, part[from / 64]);
        } else {
            for (int32_t from = 0; from < n; from += 64) total = __builtin_elementwise_add_sat(total, __builtin_amdgcn_readlane(look(a, from).upto, last_of(a, from)));
        }
        total = __builtin_amdgcn_readfirstlane(total);
        if (total == INT32_MAX) total = 0;
    }
    // The sequence that step `at` < total belongs to; *begin: where that begins.
    __device__ __forceinline__ int32_t find(const AttendArgs &a, int32_t at, int32_t *begin) const
    {
        const int32_t lane = threadIdx.x & 63, n = a.s.n_seqs;
        int32_t before = 0;
        for (int32_t from = 0; from < n; from += 64) {
            int32_t upto = 0, steps;
            if (n <= LISTED) {
                steps = __builtin_amdgcn_readfirstlane(part[from / 64]);
            } else {
                upto = look(a, from).upto;
                steps = __builtin_amdgcn_readlane(upto, last_of(a, from));
            }
            if (at - before >= steps) {
                before += steps;
                continue;
            }
            if (n <= LISTED) upto = list[from + lane].upto;
            const int32_t skipped = __popcll(__ballot(from + lane < n && upto <= at - before)); // sequences that end at or before it
            *begin = before + (skipped ? __builtin_amdgcn_readlane(upto, skipped - 1) : 0);
            return from + skipped;
        }
        return n;
    }
    __device__ __forceinline__ Seq seq(const AttendArgs &a, int32_t i) const
    {
        const Seq q = a.s.n_seqs <= LISTED ? list[i].seq : seq_of(a.s, i);
        return Seq{__builtin_amdgcn_readfirstlane(q.row), __builtin_amdgcn_readfirstlane(q.n), __builtin_amdgcn_readfirstlane(q.line),
                   __builtin_amdgcn_readfirstlane(q.len)};
    }
};

// How many workgroups share the line (none gets less than LEAST steps while another has some), and where share b begins: any
// rising function of b that all workgroups evaluate alike will do, so one product in double does.  LEAST 16, 24, 32 for one
// token behind 480: 17, 12, 12 us (one workgroup a head needs no join); sixteen behind 500: 21, 15, 21; behind 4000: 18, 17, 18.
constexpr int LEAST = 24;
struct Shares {
    int32_t total, of;
    double each;
    __device__ __forceinline__ Shares(const AttendArgs &a, int32_t steps)
    {
        total = steps;
        of = total / LEAST + (total % LEAST != 0);
        if (of > a.blocks) of = a.blocks;
        each = (double)total / (double)(of > 0 ? of : 1);
    }
    __device__ __forceinline__ int32_t begin(int32_t b) const { return b >= of ? total : __builtin_amdgcn_readfirstlane((int32_t)(each * (double)b)); }
    __device__ __forceinline__ int32_t share_of(int32_t step) const // the share that step `step` lies in
    {
        int32_t b = __builtin_amdgcn_readfirstlane((int32_t)((double)step / each));
        while (b > 0 && begin(b) > step) --b; // one off at most
        while (b + 1 < of && begin(b + 1) <= step) ++b;
        return b;
    }
};

// What a wave asks of memory for one step: codes of its keys (tokens 16 h + r, channels D / 4 g ..) and values (tokens of
// element e, channels D / 16 r ..), and one token's alpha and beta, of the keys in lanes 0..31, of the values in the others.
// Addresses are a base for the wave and 32-bit offsets for the lanes.
template <int D>
struct Codes {
    uint32_t k[2][D / 32], v[8];
    float alpha;
    int32_t beta;
};
template <int D>
struct Loads {
    uint32_t key_at, value_at, param_at; // of the lane

    __device__ __forceinline__ Loads(int32_t lane, int32_t P)
    {
        const uint32_t r = lane & 15, g = lane >> 4;
        key_at = r * (D / 2) + D / 8 * g;
        value_at = 4 * g * (D / 2) + D / 32 * r;
        param_at = ((lane >> 5) * 2 * P + (lane & 31)) * 4;
    }
    __device__ __forceinline__ void ask(const Step &s, int32_t head, int32_t page, int32_t t0, Codes<D> &x) const
    {
        const int32_t P = 1 << s.page_shift, in_page = t0 & (P - 1);
        const uint8_t *part = s.pages + (page < 0 ? 0 : page) * s.page_bytes + (int64_t)head * P * (D + 16);
        const uint8_t *keys = part + in_page * (D / 2), *values = keys + P * (D / 2), *alphas = part + P * D + in_page * 4;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint8_t *src = keys + key_at + 16 * h * (D / 2);
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
            const uint8_t *src = values + value_at + (16 * (e >> 2) + (e & 3)) * (D / 2);
            x.v[e] = D == 128 ? *reinterpret_cast<const uint32_t *>(src) : *reinterpret_cast<const uint16_t *>(src);
        }
        x.alpha = *reinterpret_cast<const float *>(alphas + param_at);
        x.beta = *reinterpret_cast<const int32_t *>(alphas + 4 * P + param_at);
    }
};

// A workgroup leaves at most two tiles unfinished: the one it begins with (slot 0) and the one it ends with (slot 1).  Per row:
// running maximum and sum, and dim unnormalised sums (partial_at).
// Sequence i's tiles are numbered from row_start[i] * group / ROWS + i on: at least as many numbers as it has tiles, in order.
__device__ __forceinline__ int32_t number_of(const AttendArgs &a, int32_t i)
{
    return a.s.row_start ? (int32_t)((uint32_t)(row_of(a.s, i) * a.group) / ROWS) + i : i * ((a.group + ROWS - 1) / ROWS);
}
__device__ __forceinline__ int64_t partial_at(const AttendArgs &a, int32_t head, int32_t block, int32_t slot, int32_t row)
{
    return (((int64_t)head * a.blocks + block) * 2 + slot) * ROWS + row;
}

// Channel c of row n of a tile whose first row is head head0 of row q_row of the step's tensors
template <int D, bool F32O>
__device__ __forceinline__ void put_out(const AttendArgs &a, int32_t head, int32_t q_row, int32_t head0, int32_t n, int32_t c, float y)
{
    const int32_t tok = (int32_t)a.by_group.divide((uint32_t)(head0 + n));
    const int64_t at = (int64_t)(q_row + tok) * a.ldo + (head * a.group + head0 + n - tok * a.group) * D + c;
    if (F32O) static_cast<float *>(a.out)[at] = y;
    else static_cast<uint16_t *>(a.out)[at] = (uint16_t)pack_bf16(y, 0.0f);
}

template <int D, bool F32Q, bool F32O>
__global__ __launch_bounds__(WAVES * 64, F32Q ? 2 : 3) void attend_kernel(const AttendArgs a)
{
    constexpr int PARTS = F32Q ? 3 : 1, WPARTS = F32Q ? 3 : 2; // of the queries, of the weights
    constexpr int KS = D / 32, DT = D / 16; // steps of 32 channels; tiles of 16 channels (one channel of each lane row)
    __shared__ float mrg_m[WAVES][ROWS], mrg_l[WAVES][ROWS], mrg_o[WAVES][ROWS][D + 4];
    // a token's parameters, worked out by one lane and read by sixteen: a key's factor and 16 + beta, a value's alpha and - (16 + beta)
    __shared__ __attribute__((aligned(16))) float2 params[WAVES][64];
    __shared__ Listed listed[LISTED];
    __shared__ int32_t parts[LISTED / 64];

    const Step &s = a.s;
    const int32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int32_t head = blockIdx.y;
    const Line line(a, listed, parts);
    const Shares shares(a, line.total);
    const int32_t block = blockIdx.x;
    const int32_t begin = shares.begin(block), end = shares.begin(block + 1);
    const Codes16 codes;
    const float factor = lane < 32 ? a.scale2 : 1.0f, sign = lane < 32 ? 1.0f : -1.0f, exact = lane < 32 ? INFINITY : 256.0f;

    int32_t at = begin, seq_begin = 0, i_seq = 0;
    if (at < end) i_seq = line.find(a, begin, &seq_begin);
    while (at < end && i_seq < s.n_seqs) {
    Tile t;
    t.seq = line.seq(a, i_seq);
    const Work work_here = work_of(a, t.seq);
    if (at - seq_begin >= work_here.tiles * work_here.steps) { // on to the next sequence
        seq_begin += work_here.tiles * work_here.steps, ++i_seq;
        continue;
    }
    const int32_t number = (int32_t)((uint32_t)(at - seq_begin) / (uint32_t)work_here.steps);
    const int32_t skip = at - seq_begin - number * work_here.steps;
    const int32_t take = work_here.steps - skip < end - at ? work_here.steps - skip : end - at;
    t.first = number * ROWS, t.rows = t.seq.n * a.group;
    const int32_t tok0 = (int32_t)((uint32_t)t.first / (uint32_t)a.group), head0 = t.first - tok0 * a.group; // of the tile's first row
    const Sight v = sight_of(a, t, tok0, head0, ROWS);
    const int32_t step_begin = work_here.first + (skip > BESIDE ? skip - BESIDE : 0), last = work_here.first + skip + take - BESIDE;
    const int32_t step_end = v.all_hi < 0 || last <= v.all_hi / STEP + 1 ? last : v.all_hi / STEP + 1;
    const bool whole = take == work_here.steps;
    const int32_t slot = at == begin ? 0 : 1;
    if (skip == 0 && threadIdx.x == 0 && a.numbers) // numbers 0: every workgroup finishes what it begins
        a.unfinished[(int64_t)head * a.numbers + number_of(a, i_seq) + number] = Unfinished{
            whole ? 1 : shares.share_of(at + work_here.steps - 1) - block + 1, block, slot, t.seq.row + tok0, head0, t.rows - t.first < ROWS ? t.rows - t.first : ROWS, {}};
    at += take;

    // page numbers of up to 64 steps of this wave, one a lane
    const auto pages_from = [&](int32_t first) {
        const int32_t mine = first + lane * WAVES;
        return mine < step_end ? page_of(s, t.seq.line, mine * STEP) : -1;
    };
    int32_t pages = pages_from(step_begin + wave);

    // this lane's row (a column of the transposed products) and the tokens it sees: lo .. hi
    const int32_t row = t.first + r, token = tok0 + (int32_t)a.by_group.divide((uint32_t)(head0 + r)), head_of_row = head0 + r - (token - tok0) * a.group;
    const bool real = row < t.rows;
    const int32_t pos = t.seq.len - t.seq.n + token, hi = real ? hi_at(v.limit, pos) : -1, lo = lo_at(a, pos);

    // queries: element e of step k of lane group g is channel (D / 4) g + 8 k + {0, 4, 1, 5, 2, 6, 3, 7}[e]
    bf16x8 qo[PARTS][KS];
    float qsum = 0.0f;
    // float32: - 24 times the sums of the queries' first parts over a step of channels, and of the other parts over all.  A matrix
    // operation on bf16 codes gives the exact sum rounded once, the accumulator's share included, in 0.92 to 1.00 of its results, and is off
    // by three steps of the largest addend at most in the others: what cancels inside of one costs next to no bits.
    float centre[F32Q ? KS : 1], rest = 0.0f;
    {
        const int64_t from = (int64_t)(t.seq.row + token) * a.ldq + (head * a.group + head_of_row) * D + D / 4 * g;
        if (!F32Q && a.q_vec) {
            uint4 w[KS];
#pragma unroll
            for (int k = 0; k < KS; ++k) w[k] = make_uint4(0, 0, 0, 0);
            if (real) {
#pragma unroll
                for (int k = 0; k < KS; ++k) w[k] = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(a.q) + from + 8 * k);
            }
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const uint32_t d[4] = {w[k].x, w[k].y, w[k].z, w[k].w};
#pragma unroll
                for (int e = 0; e < 4; ++e) qsum += __uint_as_float(d[e] << 16) + __uint_as_float(d[e] & 0xffff0000u);
                qo[0][k] = __builtin_bit_cast(bf16x8, u32x4{__builtin_amdgcn_perm(d[2], d[0], 0x05040100u), __builtin_amdgcn_perm(d[2], d[0], 0x07060302u),
                                                            __builtin_amdgcn_perm(d[3], d[1], 0x05040100u), __builtin_amdgcn_perm(d[3], d[1], 0x07060302u)});
            }
        } else {
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                float x[8], sum0 = 0.0f;
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = 0.0f;
                if (F32Q && real && a.q_vec) {
                    const float4 *src = reinterpret_cast<const float4 *>(static_cast<const float *>(a.q) + from + 8 * k);
                    const float4 w = src[0], y = src[1];
                    x[0] = w.x, x[1] = y.x, x[2] = w.y, x[3] = y.y, x[4] = w.z, x[5] = y.z, x[6] = w.w, x[7] = y.w;
                } else if (real) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = load1<F32Q>(a.q, from + 8 * k + (e >> 1) + 4 * (e & 1));
                }
                if (F32Q) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float high = __uint_as_float(__float_as_uint(x[e]) & 0xffff0000u);
                        sum0 += high, rest += x[e] - high;
                    }
                    sum0 += __shfl_xor(sum0, 16);
                    sum0 += __shfl_xor(sum0, 32);
                    centre[k] = -24.0f * sum0, qsum += sum0;
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) qsum += x[e];
                }
                bf16x8 part[PARTS];
                split8<PARTS>(x, part);
#pragma unroll
                for (int i = 0; i < PARTS; ++i) qo[i][k] = part[i];
            }
        }
        float &part_sum = F32Q ? rest : qsum;
        part_sum += __shfl_xor(part_sum, 16);
        part_sum += __shfl_xor(part_sum, 32);
        if (F32Q) qsum += rest, rest *= -24.0f;
    }

    f32x4 acc[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.0f; // running maximum; this lane's part of the sum of p

    const auto work = [&](const Codes<D> &x, int32_t t0, int32_t page) {
            const float zero = sign * ((float)x.beta + 16.0f);
            params[wave][lane] = make_float2(x.alpha * factor, F32Q && lane < 32 ? (float)x.beta - 8.0f : zero);
            const bool far = __any(fabsf(zero) > exact); // some - (16 + beta) of a value has more than the 8 bits of a bf16
            __builtin_amdgcn_wave_barrier();
            const float4 *par = reinterpret_cast<const float4 *>(&params[wave][4 * g]); // tokens 16 h + 4 g + i at 8 h + i / 2, values' behind
            float sc[8];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                f32x4 d = f32x4{1.f, 1.f, 1.f, 1.f} * rest;
#pragma unroll
                for (int i = PARTS - 1; i >= (F32Q ? 1 : 0); --i)
#pragma unroll
                    for (int k = 0; k < KS; ++k) d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes.operand(x.k[h][k]), qo[i][k], d, 0, 0, 0);
                if (F32Q) { // about one rounding for 32 channels, of a sum of (c - 8) q: 16 + c and what is taken off meet in one operation
#pragma unroll
                    for (int k = 0; k < KS; ++k)
                        d += __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes.operand(x.k[h][k]), qo[0][k], f32x4{1.f, 1.f, 1.f, 1.f} * centre[k], 0, 0, 0);
                }
                const float4 k0 = par[8 * h], k1 = par[8 * h + 1];
                const float ka[4] = {k0.x, k0.z, k1.x, k1.z}, kb[4] = {k0.y, k0.w, k1.y, k1.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) sc[4 * h + i] = ka[i] * __builtin_fmaf(-kb[i], qsum, d[i]);
            }
            float va[8];
            bf16x8 zeros; // - (16 + beta) of the values: the high halves, the number itself where it has 8 bits
            {
                float vz[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float4 v0 = par[16 + 8 * (i >> 1) + (i & 1)];
                    va[2 * i] = v0.x, vz[2 * i] = v0.y, va[2 * i + 1] = v0.z, vz[2 * i + 1] = v0.w;
                }
                u32x4 y;
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = __builtin_amdgcn_perm(__float_as_uint(vz[2 * e + 1]), __float_as_uint(vz[2 * e]), 0x07060302u);
                zeros = __builtin_bit_cast(bf16x8, y);
            }
            if (t0 < v.each_lo || t0 + STEP - 1 > v.each_hi || page < 0) { // some row does not see some token; what lies there may be anything
                int32_t mine = t0 + 4 * g;
                asm volatile("" : "+v"(mine)); // keeps the comparisons in here
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int32_t tok = mine + 16 * (i >> 2) + (i & 3);
                    const bool seen = tok >= lo && tok <= hi && page >= 0;
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
            float w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float p = __builtin_amdgcn_exp2f(sc[i] - base);
                l += p;
                w[i] = p * va[i];
            }
            // in bf16 parts, which leave out 2^-16 of a weight at most for bf16 queries (one part, 2^-8, makes a bf16 output's error
            // 1.4 times as large and saves 3 % of the time) and hold 24 bits for float32
            bf16x8 pw[WPARTS];
            split8<WPARTS>(w, pw);
            uint32_t low[4], high[4]; // codes 0..3 and 4..7 of two neighbouring tokens
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                low[e] = __builtin_amdgcn_perm(x.v[2 * e + 1], x.v[2 * e], 0x05040100u);
                high[e] = __builtin_amdgcn_perm(x.v[2 * e + 1], x.v[2 * e], 0x07060302u);
            }
            // (16 + c) - (16 + beta) in two products: the sums stay as small as the values are, whatever the number of tokens.
            // float32, the weights' first parts: 16 tokens' codes and zero points in one operation, which rounds about once, what it adds to
            // the accumulator; the other parts are 2^-8 of it.
            const auto tile = [&](int i, bf16x8 c) {
#pragma unroll
                for (int j = WPARTS - 1; j >= (F32Q ? 1 : 0); --j) {
                    acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(zeros, pw[j], acc[i], 0, 0, 0);
                    acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(c, pw[j], acc[i], 0, 0, 0);
                }
                if (F32Q) {
                    const u32x4 w = __builtin_bit_cast(u32x4, c), z = __builtin_bit_cast(u32x4, zeros), p = __builtin_bit_cast(u32x4, pw[0]);
#pragma unroll
                    for (int h = 0; h < 4; h += 2)
                        acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, u32x4{w[h], w[h + 1], z[h], z[h + 1]}),
                                                                         __builtin_bit_cast(bf16x8, u32x4{p[h], p[h + 1], p[h], p[h + 1]}), acc[i], 0, 0, 0);
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
            if (far) { // values far from zero for their range: what the high halves leave out, 16 bits in two more parts
                float vz[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float4 v0 = par[16 + 8 * (i >> 1) + (i & 1)];
                    vz[2 * i] = v0.y, vz[2 * i + 1] = v0.w;
                }
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    u32x4 y;
#pragma unroll
                    for (int e = 0; e < 8; ++e) vz[e] -= __uint_as_float(__float_as_uint(vz[e]) & 0xffff0000u);
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[e] = __builtin_amdgcn_perm(__float_as_uint(vz[2 * e + 1]), __float_as_uint(vz[2 * e]), 0x07060302u);
                    const bf16x8 rest = __builtin_bit_cast(bf16x8, y);
#pragma unroll
                    for (int i = 0; i < DT; ++i)
#pragma unroll
                        for (int j = WPARTS - 1; j >= 0; --j) acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(rest, pw[j], acc[i], 0, 0, 0);
                }
            }
    };

    // The loads of a step are on their way while the step before is worked on.  Nothing in between waits for memory and no condition
    // stands around them: the page numbers are there beforehand, and a step without a page reads page 0 and sees nothing of it.
    const Loads<D> from(lane, 1 << s.page_shift);
    for (int32_t first = step_begin + wave; first < step_end;) {
        const int32_t left_of = (step_end - first + WAVES - 1) / WAVES, count = left_of < 64 ? left_of : 64;
        Codes<D> x[2];
        int32_t page = __builtin_amdgcn_readlane(pages, 0);
        from.ask(s, head, page, first * STEP, x[0]);
        for (int32_t n = 0; n < count;) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int32_t next = n + 1 < count ? __builtin_amdgcn_readlane(pages, n + 1) : -1, t0 = (int32_t)((uint32_t)(first + n * WAVES) * STEP);
                from.ask(s, head, next, (int32_t)((uint32_t)t0 + WAVES * STEP), x[1 - i]);
                if (n < count) work(x[i], t0, page);
                page = next, ++n;
            }
        }
        first += 64 * WAVES;
        if (first < step_end) pages = pages_from(first);
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
        const int32_t n = i / D, c = i % D;
        if (t.first + n >= t.rows) break;
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
            put_out<D, F32O>(a, head, t.seq.row + tok0, head0, n, c, quotient(o, sum));
        } else {
            const int64_t at = partial_at(a, head, block, slot, n);
            a.part_o[at * D + c] = o;
            if (c == 0) a.part_ml[at] = make_float2(top, sum);
        }
    }
    __syncthreads(); // before the next tile's results
    }
}

// The parts of unfinished tiles joined, a workgroup for (some rows of) each tile: a wave for a row of few parts, JOIN_WAVES / 2
// for a row of many.  A part of a row takes D / 4 lanes; every read of a batch is on its way before the first is looked at.
constexpr int JOIN_WAVES = 8, JOIN_FEW = 12;
template <int D, bool F32O>
__global__ __launch_bounds__(JOIN_WAVES * 64) void join_kernel(const AttendArgs a)
{
    constexpr int AT_ONCE = 64 / (D / 4), BATCH = 6;
    __shared__ float tops[JOIN_WAVES], sums[JOIN_WAVES], os[JOIN_WAVES][D];
    const int32_t head = blockIdx.y, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int32_t number = blockIdx.x;
    if (a.s.row_start) { // not every number is a tile's
        const int32_t i = last_not_above(a.s.n_seqs, number, [&](int32_t k) { return (int64_t)number_of(a, k); });
        const int32_t k = number - number_of(a, i);
        if (k < 0 || k >= work_of(a, seq_of(a.s, i)).tiles) return;
    }
    const Unfinished u = a.unfinished[(int64_t)head * a.numbers + number];
    // (the comparisons with the launch's sizes are for a row_start that does not ascend)
    if (u.parts <= 1 || u.block < 0 || u.block >= a.blocks || u.parts > a.blocks - u.block || u.q_row < 0 || u.head0 < 0 || u.head0 >= a.group ||
        u.rows > ROWS || (int64_t)u.q_row * a.group + u.head0 + u.rows > (int64_t)a.s.rows * a.group)
        return;
    const int32_t per_row = u.parts <= JOIN_FEW ? 1 : JOIN_WAVES / 2, at_once = JOIN_WAVES / per_row; // waves of a row, rows of a pass
    const int32_t sub = lane / (D / 4), c = lane % (D / 4) * 4;
    for (int32_t row0 = blockIdx.z * at_once; row0 < u.rows; row0 += gridDim.z * at_once) {
        const int32_t n = row0 + wave / per_row, step = per_row * AT_ONCE;
        float top = -INFINITY, sum = 0.0f;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
        for (int32_t p0 = wave % per_row * AT_ONCE + sub; n < u.rows && p0 < u.parts; p0 += step * BATCH) {
            float2 ml[BATCH];
            f32x4 x[BATCH];
#pragma unroll
            for (int k = 0; k < BATCH; ++k) {
                const int32_t p = p0 + k * step;
                ml[k] = make_float2(-INFINITY, 0.0f), x[k] = f32x4{0.f, 0.f, 0.f, 0.f};
                if (p < u.parts) {
                    const int64_t from = partial_at(a, head, u.block + p, p == 0 ? u.slot & 1 : 0, n);
                    ml[k] = a.part_ml[from];
                    x[k] = *reinterpret_cast<const f32x4 *>(a.part_o + from * D + c);
                }
            }
            float now = top;
#pragma unroll
            for (int k = 0; k < BATCH; ++k) now = fmaxf(now, ml[k].x);
            const float base = now == -INFINITY ? 0.0f : now, f0 = __builtin_amdgcn_exp2f(top - base);
            sum *= f0, o *= f0, top = now;
#pragma unroll
            for (int k = 0; k < BATCH; ++k) {
                const float f = __builtin_amdgcn_exp2f(ml[k].x - base);
                sum += f * ml[k].y, o += f * x[k];
            }
        }
        // the lanes of a wave, then the waves of a row
        float best = top;
#pragma unroll
        for (int k = D / 4; k < 64; k <<= 1) best = fmaxf(best, __shfl_xor(best, k));
        const float f = __builtin_amdgcn_exp2f(top - (best == -INFINITY ? 0.0f : best));
        sum *= f, o *= f;
#pragma unroll
        for (int k = D / 4; k < 64; k <<= 1) {
            sum += __shfl_xor(sum, k);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], k);
        }
        if (lane == 0) tops[wave] = best, sums[wave] = sum;
        if (sub == 0) *reinterpret_cast<f32x4 *>(&os[wave][c]) = o;
        __syncthreads();
        for (int32_t i = threadIdx.x; i < at_once * D; i += JOIN_WAVES * 64) {
            const int32_t k = i / D, ch = i % D, row = row0 + k;
            if (row >= u.rows) break;
            float all = -INFINITY, total = 0.0f, y = 0.0f;
            for (int w = k * per_row; w < (k + 1) * per_row; ++w) all = fmaxf(all, tops[w]);
            if (all == -INFINITY) all = 0.0f;
            for (int w = k * per_row; w < (k + 1) * per_row; ++w) {
                const float g = __builtin_amdgcn_exp2f(tops[w] - all);
                total += g * sums[w], y += g * os[w][ch];
            }
            put_out<D, F32O>(a, head, u.q_row, u.head0, row, ch, quotient(y, total));
        }
        __syncthreads(); // before the next rows
    }
}

int32_t check(const qllm_kv_cache *cache, const qllm_kv_batch *batch, int64_t q_heads)
{
    if (q_heads <= 0 || q_heads > (1 << 15) || q_heads % cache->heads) return QLLM_ERR_SHAPE;
    const int64_t rows = batch->rows * (q_heads / cache->heads);
    const int64_t tiles = rows / ROWS + batch->n_seqs, steps = batch->table_ld * cache->page_tokens / STEP + BESIDE;
    return tiles < (1 << 23) && tiles * steps < INT32_MAX ? QLLM_OK : QLLM_ERR_SHAPE; // (a grid of tiles has less than 2^32 threads)
}

// Whether the prompts kernel takes sequences of more than FEW_ROWS rows: few tiles of 128 rows leave most of the card to wait for
// one way through the tokens, beyond what its sharing of them makes good; this kernel's time grows with tiles and tokens alike.
// One sequence, tiles x tokens, this kernel's us first (D 128): 8 x 4000 30 and 30, 8 x 16000 40 and 49, 16 x 1000 26 and 31,
// 16 x 4000 34 and 30, 16 x 16000 58 and 47, 32 x 1000 30 and 31, 32 x 4000 40 and 32, 64 x 4000 63 and 38, 128 x 4000 101 and 55,
// 128 x 16000 323 and 160; 32 x 300 27 and 20, 16 x 64 20 and 14.  With several sequences this kernel runs beside it, some 5 us if
// it finds nothing: 8 x 64 rows behind 2000, 32 tiles, 37 and 35 + 5; 8 x 128, 64 tiles, 48 and 38 + 4.
// FEW_ROWS: sequences x rows, 8 heads, 2000 tokens: 32 x 32 47 and 47, 32 x 64 71 and 48, 32 x 128 119 and 53.
// (A grid of 2^32 threads would be refused by the runtime.)
constexpr int32_t FEW_ROWS = 32;
bool prompts_pay(const qllm_kv_cache *cache, const qllm_kv_batch *batch, int64_t q_heads, int32_t q_dtype)
{
    const int64_t rows = batch->rows * (q_heads / cache->heads), tiles = rows / 128 * cache->heads, tokens = batch->table_ld * cache->page_tokens;
    const int64_t least = batch->n_seqs == 1 ? 16 : 48;
    return q_dtype == QLLM_BF16 && batch->row_start && (tokens <= 640 || (tiles >= least && tiles * tokens >= 2000 * least)) &&
           rows > batch->n_seqs * FEW_ROWS && (rows / 128 + batch->n_seqs) * cache->heads < (1 << 24);
}
QllmKvPrompts plan_prompts(const qllm_kv_cache *cache, const qllm_kv_batch *batch, int64_t q_heads)
{
    return qllm_kv_plan_prompts(*batch, cache->heads, q_heads / cache->heads, cache->dim, batch->table_ld * cache->page_tokens);
}

// Workgroups of a kv head: as many as the card holds at once (on each of 256 CUs three, two for float32 queries, whose parts take
// registers: 768 there 42.9 against 39.1 us for sixteen single tokens behind 5000), but none for less than LEAST steps.
struct Launch {
    int64_t numbers, blocks; // of tiles (see number_of); of workgroups
    int64_t marks, parts;    // bytes of the workspace for each kind
};
Launch plan(const qllm_kv_cache *cache, const qllm_kv_batch *batch, int64_t q_heads, int32_t q_dtype)
{
    const int64_t resident = q_dtype == QLLM_F32 ? 2 * 256 : 3 * 256;
    const int64_t group = q_heads / cache->heads;
    Launch n;
    n.numbers = batch->row_start ? batch->rows * group / ROWS + batch->n_seqs : batch->n_seqs * ((group + ROWS - 1) / ROWS);
    const int64_t most = n.numbers * (batch->table_ld * cache->page_tokens / STEP + BESIDE) / LEAST + 1; // below 2^31
    const int64_t blocks = cache->heads < resident ? resident / cache->heads : 1;
    n.blocks = blocks < most ? blocks : most;
    n.marks = n.blocks > 1 ? cache->heads * n.numbers * (int64_t)sizeof(Unfinished) : 0;
    n.parts = n.blocks > 1 ? cache->heads * n.blocks * 2 * ROWS : 0;
    return n;
}

} // namespace

extern "C" int64_t qllm_kv_attention_workspace_bytes(const qllm_kv_cache *cache, const qllm_kv_batch *batch, int64_t q_heads)
{
    Step s;
    int32_t rc = prepare_step(cache, batch, false, &s);
    if (rc == QLLM_OK) rc = check(cache, batch, q_heads);
    if (rc != QLLM_OK) return rc;
    const Launch n = plan(cache, batch, q_heads, QLLM_BF16); // no less than for float32
    const int64_t bytes = n.marks + n.parts * (cache->dim + 2) * (int64_t)sizeof(float);
    if (!prompts_pay(cache, batch, q_heads, QLLM_BF16)) return 256 + bytes;
    const int64_t prompts = plan_prompts(cache, batch, q_heads).bytes; // before the others: the same place
    return 256 + (bytes > prompts ? bytes : prompts);
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
    if (ldq < q_heads * cache->dim || ldo < q_heads * cache->dim || window < 0 || !isfinite(scale * LOG2E)) return QLLM_ERR_SHAPE;
    if ((reinterpret_cast<uintptr_t>(q) & (q_dtype == QLLM_F32 ? 3u : 1u)) || (reinterpret_cast<uintptr_t>(out) & (out_dtype == QLLM_F32 ? 3u : 1u)))
        return QLLM_ERR_ALIGN;
    if (!workspace || workspace_bytes < qllm_kv_attention_workspace_bytes(cache, batch, q_heads)) return QLLM_ERR_WORKSPACE;
    if (reinterpret_cast<uintptr_t>(workspace) & 15u) return QLLM_ERR_ALIGN;
    if (batch->rows == 0 || batch->n_seqs == 0) return QLLM_OK;
    a.q = q, a.out = out, a.ldq = ldq, a.ldo = ldo;
    a.q_heads = (int32_t)q_heads, a.group = (int32_t)(q_heads / cache->heads);
    a.by_group = qllm_detail::quotient_by((uint32_t)a.group);
    a.q_vec = ((reinterpret_cast<uintptr_t>(q) | (uintptr_t)(ldq * (q_dtype == QLLM_F32 ? 4 : 2))) & 15u) == 0;
    a.out_vec = ((reinterpret_cast<uintptr_t>(out) | (uintptr_t)(ldo * (out_dtype == QLLM_F32 ? 4 : 2))) & (out_dtype == QLLM_F32 ? 15u : 7u)) == 0;
    a.window = window > INT32_MAX ? 0 : (int32_t)window;
    a.scale2 = scale * LOG2E;
    // Sequences of many rows are the prompts kernel's, the others this one's.  (One sequence: all of it goes to one of them.)
    hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
    (void)hipGetLastError();
    a.few = INT32_MAX;
    if (a.scale2 != 0.0f && prompts_pay(cache, batch, q_heads, q_dtype)) { // (it divides by the scale)
        a.few = batch->n_seqs == 1 ? 0 : FEW_ROWS;
        rc = qllm_kv_launch_prompts(a, plan_prompts(cache, batch, q_heads), cache->dim, out_dtype, workspace, stream);
        if (rc != QLLM_OK || batch->n_seqs == 1) return rc;
    }
    const Launch n = plan(cache, batch, q_heads, q_dtype);
    a.blocks = (int32_t)n.blocks, a.numbers = n.blocks > 1 ? (int32_t)n.numbers : 0;
    a.unfinished = static_cast<Unfinished *>(workspace);
    a.part_o = reinterpret_cast<float *>(static_cast<uint8_t *>(workspace) + n.marks);
    a.part_ml = reinterpret_cast<float2 *>(a.part_o + n.parts * cache->dim);
    const dim3 grid((unsigned)a.blocks, (unsigned)cache->heads);
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
    // one token each: few tiles, perhaps of many parts, two rows of which a workgroup takes; else many tiles, most of them whole
    const int64_t rows = a.group < ROWS ? a.group : ROWS;
    const dim3 cuts((unsigned)n.numbers, (unsigned)cache->heads, batch->row_start ? 1 : (unsigned)((rows + 1) / 2));
    if (cache->dim == 128 && out_dtype == QLLM_F32) hipLaunchKernelGGL((join_kernel<128, true>), cuts, dim3(JOIN_WAVES * 64), 0, stream, a);
    else if (cache->dim == 128) hipLaunchKernelGGL((join_kernel<128, false>), cuts, dim3(JOIN_WAVES * 64), 0, stream, a);
    else if (out_dtype == QLLM_F32) hipLaunchKernelGGL((join_kernel<64, true>), cuts, dim3(JOIN_WAVES * 64), 0, stream, a);
    else hipLaunchKernelGGL((join_kernel<64, false>), cuts, dim3(JOIN_WAVES * 64), 0, stream, a);
    return launched("cache attention: parts joined");
}
