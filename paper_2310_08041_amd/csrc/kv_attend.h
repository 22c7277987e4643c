// Internal to libqllm: what the two attention kernels over the 4-bit cache share.
//
// For a kv head the queries of its group of query heads are rows of one matrix: row r of a sequence's n rows x G heads is token
// r / G, head r % G.  Codes are integers, so with k = alpha (c - beta) the score of a token is
//     scale alpha (q . (16 + c) - (16 + beta) sum q),
// the first product on the matrix cores: 16 + c is an exact bf16 whose bits are 0x4180 | c << 3, two vector instructions for a
// pair of codes.  In the same way sum_t p_t v_t = sum_t (p_t alpha_t)(16 + c_t) - sum_t (p_t alpha_t)(16 + beta_t), with p_t alpha_t
// in bf16 parts, the same in both sums, which are taken together on the matrix cores.  The scores are
// formed transposed (tokens x rows): their accumulator then is, register for register, the operand that meets the values, and
// nothing crosses lanes in between.
#ifndef QLLM_KV_ATTEND_H
#define QLLM_KV_ATTEND_H

#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include "fused_common.h"
#include "kv_common.h"

namespace qllm_kv_detail {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr float LOG2E = 1.44269504088896341f;
constexpr float SLACK = 8.0f; // the running maximum follows only when the scores pass it by this much: weights stay below 2^8

struct Unfinished { // how a tile is to be joined: its parts (1: nothing to join), the workgroup of the first and the slot there,
    int32_t parts, block, slot, q_row, head0, rows, pad[2]; // its first row, head head0 of row q_row, and how many
};
struct AttendArgs {
    Step s;
    const void *q;
    void *out;
    int64_t ldq, ldo;
    int32_t q_heads, group, window; // window 0: none
    float scale2;                   // scale * log2 e
    int32_t q_vec, out_vec;         // queries in 16-byte pieces; four outputs at a time
    qllm_detail::QuotientBy by_group; // for numbers below group + 128
    int32_t blocks;                 // workgroups of a kv head
    float *part_o;                  // their partial results, see partial_at
    float2 *part_ml;
    int32_t few;                    // sequences of more rows than this are left to the kernel for prompts
    int32_t numbers;                // of tiles, see number_of
    Unfinished *unfinished;         // [heads][numbers]
    int32_t parts;                  // of a prompts tile's tokens, at most
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

// A row tile of a workgroup: rows from `first` on of a sequence's n * group rows (row r: token r / group, query head r % group).
struct Tile {
    Seq seq;
    int32_t first, rows;
};

// What rows see: tokens all_lo .. all_hi some of them, each_lo .. each_hi every one.
struct Sight {
    int32_t limit, all_lo, all_hi, each_lo, each_hi;
};

__device__ __forceinline__ int32_t lo_at(const AttendArgs &a, int32_t pos) { return first_seen(pos, a.window); }
__device__ __forceinline__ int32_t hi_at(int32_t limit, int32_t pos) { return pos < limit ? pos : limit - 1; }
__device__ __forceinline__ int32_t limit_of(const AttendArgs &a, const Seq &q)
{
    const int32_t cap = a.s.table_ld << a.s.page_shift;
    return q.line < 0 ? 0 : (q.len < cap ? q.len : cap);
}

__device__ __forceinline__ Sight sight_of(const AttendArgs &a, const Tile &t, int32_t tok0, int32_t head0, int32_t most)
{
    Sight v;
    v.limit = limit_of(a, t.seq);
    const int32_t rows = t.rows - t.first < most ? t.rows - t.first : most;
    const int32_t p_first = t.seq.len - t.seq.n + tok0, p_last = p_first + (int32_t)a.by_group.divide((uint32_t)(head0 + rows - 1));
    v.all_lo = lo_at(a, p_first), v.all_hi = hi_at(v.limit, p_last);
    v.each_lo = lo_at(a, p_last), v.each_hi = hi_at(v.limit, p_first);
    return v;
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

// Eight of them: the high halves as they are, what they leave out in the next part, rounded in the last.
template <int PARTS>
__device__ __forceinline__ void split8(float (&x)[8], bf16x8 (&part)[PARTS])
{
#pragma unroll
    for (int j = 0; j < PARTS; ++j) {
        u32x4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t x0 = __float_as_uint(x[2 * e]), x1 = __float_as_uint(x[2 * e + 1]);
            y[e] = j == PARTS - 1 ? pack_bf16(x[2 * e], x[2 * e + 1]) : __builtin_amdgcn_perm(x1, x0, 0x07060302u);
            x[2 * e] -= __uint_as_float(x0 & 0xffff0000u), x[2 * e + 1] -= __uint_as_float(x1 & 0xffff0000u);
        }
        part[j] = __builtin_bit_cast(bf16x8, y);
    }
}

__device__ __forceinline__ float quotient(float o, float sum) { return sum > 0.0f ? o / sum : (sum == 0.0f ? 0.0f : sum); } // a NaN stays

} // namespace qllm_kv_detail

// The kernel for prompts (kv_prompts.hip): sequences of more than a.few rows, bf16 queries.
struct QllmKvPrompts {
    int64_t workgroups, parts, groups; // as many as there may be tiles; each tile's tokens shared by `parts` of them, of `groups` of waves
    int64_t sums, bytes;               // of the workspace for the parts' sums, and altogether
};
QllmKvPrompts qllm_kv_plan_prompts(const qllm_kv_batch &batch, int64_t heads, int64_t group, int64_t dim, int64_t tokens);
int32_t qllm_kv_launch_prompts(const qllm_kv_detail::AttendArgs &a, const QllmKvPrompts &n, int64_t dim, int32_t out_dtype, void *workspace, hipStream_t stream);

#endif
