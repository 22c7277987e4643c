// Low-rank adapters of many requests beside a shared projection: out = y + scale_a (x A_a^T) B_a^T, each row with its own a.
//
// What it has to move is x of the rows, the factors of the adapters that are named, y in and out; the operations are few
// (2 rank (C + O) a row), so it is bound by memory, and for a few rows by latency.
//   adapter_plan_kernel    once a step: the rows sorted by adapter, in tiles of up to 64 rows of one adapter
//   down_kernel            h = x A^T of a tile over a slice of C, fp32, a part of the sum per slice
//   join_kernel            where the slices of many rows are to be added: their sum
//   up_kernel              out = y + (scale h) B^T of a tile over a block of columns
// No sum uses atomics, and a row's sums do not depend on its place in a tile: equal calls give equal bits.
#include <hip/hip_runtime.h>

#include <stdint.h>

#include "fused_common.h"
#include "qllm_block.h"
#include "rows.h"

using namespace qllm_detail;

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int TILE = 64;             // rows of a tile
constexpr int PLAN_HEAD_WORDS = 4;   // {tiles, rows, adapters of the pool, -}
constexpr int PLAN_THREADS = 1024;
constexpr int MOST_ADAPTERS = 8192;
constexpr int64_t MOST_ROWS = 1 << 24, MOST_SEQS = 1 << 20;

inline int64_t most_tiles(int64_t rows, int64_t n_adapters)
{
    const int64_t groups = n_adapters + 1; // those without one are a group too
    return rows / TILE + (rows < groups ? rows : groups);
}
// words: head, rows in order, tiles of {adapter, first place in the order, rows, -}
inline int64_t order_words(int64_t rows) { return (rows + 3) / 4 * 4; }
inline int64_t plan_words(int64_t rows, int64_t n_adapters) { return PLAN_HEAD_WORDS + order_words(rows) + 4 * most_tiles(rows, n_adapters); }

// ---- the plan: rows counted per adapter, the adapters' places in the order summed up, the sequences put there.  In which order the
// sequences of one adapter come (an atomic decides) is no part of any result.
__global__ __launch_bounds__(PLAN_THREADS) void adapter_plan_kernel(int32_t rows, int32_t n_seqs, const int32_t *row_start,
                                                                   const int32_t *adapter, int32_t n_adapters, int32_t most, int32_t *plan)
{
    __shared__ uint32_t next[MOST_ADAPTERS + 1]; // rows of an adapter, then the next free place of its own; group n_adapters: none
    __shared__ uint32_t part_rows[PLAN_THREADS / 64], part_tiles[PLAN_THREADS / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int groups = n_adapters + 1;
    int32_t *order = plan + PLAN_HEAD_WORDS;
    int4 *tiles = reinterpret_cast<int4 *>(order + (rows + 3) / 4 * 4);
    for (int g = tid; g < groups; g += PLAN_THREADS) next[g] = 0;
    __syncthreads();
    auto group_of = [&](int i) {
        const int32_t a = adapter[i];
        return a >= 0 && a < n_adapters ? a : n_adapters;
    };
    auto first_row = [&](int i) { return row_start ? min(max(row_start[i], 0), rows) : min(i, rows); };
    // counts saturate, so that sequences which overlap cannot run one over
    for (int i = tid; i < n_seqs; i += PLAN_THREADS) {
        const int n = first_row(i + 1) - first_row(i);
        if (n > 0) {
            uint32_t *count = &next[group_of(i)];
            if (atomicAdd(count, (uint32_t)n) > (1u << 25)) atomicMin(count, 1u << 25);
        }
    }
    __syncthreads();
    // where each group begins: every thread sums a run of groups, then the threads' sums are summed
    const int run = (groups + PLAN_THREADS - 1) / PLAN_THREADS, g0 = tid * run, g1 = min(g0 + run, groups);
    uint32_t n_rows = 0, n_tiles = 0;
    for (int g = g0; g < g1; ++g) {
        const uint32_t n = min(next[g], (uint32_t)rows);
        n_rows = min(n_rows + n, (uint32_t)rows), n_tiles += (n + TILE - 1) / TILE;
    }
    uint32_t before_rows = n_rows, before_tiles = n_tiles;
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t r = __shfl_up(before_rows, d, 64), t = __shfl_up(before_tiles, d, 64);
        if (lane >= d) before_rows += r, before_tiles += t;
    }
    if (lane == 63) part_rows[wave] = before_rows, part_tiles[wave] = before_tiles;
    before_rows -= n_rows, before_tiles -= n_tiles;
    __syncthreads();
    uint32_t all_tiles = 0;
    for (int w = 0; w < PLAN_THREADS / 64; ++w) {
        if (w < wave) before_rows += part_rows[w], before_tiles += part_tiles[w];
        all_tiles += part_tiles[w];
    }
    for (int g = g0; g < g1; ++g) {
        const uint32_t n = min(next[g], (uint32_t)rows);
        next[g] = before_rows;
        for (uint32_t at = 0; at < n; at += TILE, ++before_tiles)
            if (before_tiles < (uint32_t)most) tiles[before_tiles] = make_int4(g, (int32_t)min(before_rows + at, (uint32_t)rows), (int32_t)min(n - at, (uint32_t)TILE), 0);
        before_rows += n;
    }
    if (tid == 0) *reinterpret_cast<int4 *>(plan) = make_int4((int32_t)min(all_tiles, (uint32_t)most), rows, n_adapters, 0);
    __syncthreads();
    if (!row_start) {
        for (int i = tid; i < min(n_seqs, rows); i += PLAN_THREADS) {
            const uint32_t at = atomicAdd(&next[group_of(i)], 1u);
            if (at < (uint32_t)rows) order[at] = i;
        }
        return;
    }
    for (int i = wave; i < n_seqs; i += PLAN_THREADS / 64) { // a sequence a wave
        const int row = first_row(i), n = first_row(i + 1) - row;
        if (n <= 0) continue;
        uint32_t at = 0;
        if (lane == 0) at = atomicAdd(&next[group_of(i)], (uint32_t)n);
        at = __builtin_amdgcn_readfirstlane(at);
        for (int j = lane; j < n; j += 64)
            if (at + j < (uint32_t)rows) order[at + j] = row + j;
    }
}

struct ApplyArgs {
    const void *x, *A, *B, *y;
    void *out;
    int64_t ldx, ldy, ldo, C, O;
    const float *scale;
    const int32_t *ranks, *plan;
    float *h; // [slices][rows in the plan's order][parts * rank]
    int32_t rows, n_adapters, rank, wide, slices, blocks_per_slice; // wide: parts * rank; blocks of 64 channels
    int32_t n_parts, part_end[QLLM_ADAPTER_PARTS], block_end[QLLM_ADAPTER_PARTS]; // columns, blocks of columns, summed up
};

struct Tile {
    int32_t adapter, first, count, rank; // count 0: none
};
__device__ __forceinline__ Tile tile_of(const ApplyArgs &a, uint32_t t)
{
    const int4 head = *reinterpret_cast<const int4 *>(a.plan);
    Tile tile{0, 0, 0, 0};
    if (head.y != a.rows || head.z != a.n_adapters || t >= (uint32_t)head.x) return tile;
    const int4 w = reinterpret_cast<const int4 *>(a.plan + PLAN_HEAD_WORDS + (a.rows + 3) / 4 * 4)[t];
    if (w.x < 0 || w.x > a.n_adapters || w.y < 0 || w.y >= a.rows || w.z <= 0) return tile;
    tile.adapter = w.x, tile.first = w.y, tile.count = min(min(w.z, TILE), a.rows - w.y);
    if (w.x < a.n_adapters) tile.rank = a.ranks ? min(max(a.ranks[w.x], 0), a.rank) : a.rank;
    return tile;
}
// the row at a place of the order, -1 where there is none
__device__ __forceinline__ int32_t row_at(const ApplyArgs &a, int32_t place)
{
    const int32_t row = a.plan[PLAN_HEAD_WORDS + place];
    return row >= 0 && row < a.rows ? row : -1;
}

// Sixteen neighbouring channels of one row of x or A, a lane's share of a block of 64 (four lanes a row).
template <typename T>
struct Sixteen {
    Eight<T> e[2];
    __device__ __forceinline__ void load(const T *p, int n)
    {
        e[0].load(p, n);
        e[1].load(p + 8, n - 8);
    }
};

// ---- h = x A^T.  Lane l of a wave holds channels 16 (l / 16) .. + 15 of a block of 64 of row l mod 16 of either operand (the order of
// the channels is the same in both, so any will do): whole 128-byte lines of bf16.  The block's waves take the slice's blocks in turn.
template <typename XT, typename WT, int MT, int NT>
__device__ __forceinline__ void down_tile(const ApplyArgs &a, const Tile &tile, int first_rank, float *part)
{
    constexpr bool HALF = sizeof(XT) == 2 && sizeof(WT) == 2;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r16 = lane & 15, quarter = lane >> 4;
    const XT *x[MT];
    const WT *w[NT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const int32_t row = row_at(a, tile.first + min(m * 16 + r16, tile.count - 1));
        x[m] = static_cast<const XT *>(a.x) + (int64_t)max(row, 0) * a.ldx + 16 * quarter;
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int at = min(first_rank + n * 16 + r16, a.wide - 1), p = at / a.rank, r = min(at - p * a.rank, tile.rank - 1);
        w[n] = static_cast<const WT *>(a.A) + ((int64_t)tile.adapter * a.wide + p * a.rank + r) * a.C + 16 * quarter;
    }
    f32x4 acc[MT][NT];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[m][n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const int64_t begin = (int64_t)blockIdx.y * a.blocks_per_slice * 64, end = min(begin + (int64_t)a.blocks_per_slice * 64, a.C);
    for (int64_t c = begin + 64 * wave; c < end; c += 64 * 4) {
        Sixteen<XT> xe[MT];
        Sixteen<WT> we[NT];
        const int left = (int)min(a.C - c - 16 * quarter, (int64_t)16);
#pragma unroll
        for (int m = 0; m < MT; ++m) xe[m].load(x[m] + c, left);
#pragma unroll
        for (int n = 0; n < NT; ++n) we[n].load(w[n] + c, left);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if constexpr (HALF) {
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
                        acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, we[n].e[h].q), __builtin_bit_cast(bf16x8, xe[m].e[h].q), acc[m][n], 0, 0, 0);
            } else {
                float xv[MT][8], wv[NT][8];
#pragma unroll
                for (int m = 0; m < MT; ++m) xe[m].e[h].widen(xv[m]);
#pragma unroll
                for (int n = 0; n < NT; ++n) we[n].e[h].widen(wv[n]);
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int m = 0; m < MT; ++m)
#pragma unroll
                        for (int n = 0; n < NT; ++n) acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x4f32(wv[n][j], xv[m][j], acc[m][n], 0, 0, 0);
            }
        }
    }
    // the waves' parts meet in LDS: [wave][row][rank]; lane l has ranks 4 (l / 16) .. + 3 of row l mod 16
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n) *reinterpret_cast<f32x4 *>(part + ((wave * MT + m) * 16 + r16) * (NT * 16) + n * 16 + 4 * quarter) = acc[m][n];
    __syncthreads();
    float *h = a.h + ((int64_t)blockIdx.y * a.rows + tile.first) * a.wide + first_rank;
    for (int i = threadIdx.x; i < MT * 16 * NT * 4; i += 256) {
        const int row = i / (NT * 4), r4 = i - row * (NT * 4);
        if (row >= tile.count || first_rank + 4 * r4 >= a.wide) continue;
        f32x4 s = *reinterpret_cast<const f32x4 *>(part + row * (NT * 16) + 4 * r4);
#pragma unroll
        for (int v = 1; v < 4; ++v) s += *reinterpret_cast<const f32x4 *>(part + (v * MT * 16 + row) * (NT * 16) + 4 * r4);
        *reinterpret_cast<f32x4 *>(h + (int64_t)row * a.wide + 4 * r4) = s;
    }
}

template <typename XT, typename WT, int NT>
__global__ __launch_bounds__(256) void down_kernel(const ApplyArgs a)
{
    __shared__ __align__(16) float part[4 * TILE * NT * 16];
    const Tile tile = tile_of(a, blockIdx.x);
    if (tile.count == 0 || tile.rank == 0) return;
    const int first_rank = blockIdx.z * NT * 16;
    if (tile.count <= 16) down_tile<XT, WT, 1, NT>(a, tile, first_rank, part);
    else down_tile<XT, WT, 4, NT>(a, tile, first_rank, part);
}

// ---- the slices' sums
__global__ __launch_bounds__(256) void join_kernel(float *h, int64_t words4, int32_t slices)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= words4) return;
    f32x4 *at = reinterpret_cast<f32x4 *>(h) + i;
    f32x4 s = at[0];
    for (int k = 1; k < slices; ++k) s += at[k * words4];
    at[0] = s;
}

// ---- out = y + (scale h) B^T.  The columns are the rows of the matrix operation and the tile's rows its columns: lane l gets 16
// neighbouring columns (4 of each of 4 operations) of row l mod 16, whose reads and writes of y are whole lines.
// h goes through LDS, with bf16 weights as PARTS bf16 numbers that add up to it, one after the other along the sum.
template <typename WT, typename YT, int MT>
__device__ __forceinline__ void up_tile(const ApplyArgs &a, const Tile &tile, int p, int column, int end, void *staged, int32_t *rows_of)
{
    constexpr bool HALF = sizeof(WT) == 2;
    constexpr int PARTS = HALF ? (sizeof(YT) == 2 ? 2 : 3) : 1;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r16 = lane & 15, quarter = lane >> 4;
    const int octets = a.rank / 8, steps = HALF ? (PARTS * octets + 3) / 4 : (a.rank + 15) / 16;
    const int stride = HALF ? steps * 32 + 8 : steps * 16 + 4; // elements of a row in LDS
    uint16_t *hb = static_cast<uint16_t *>(staged);
    float *hf = static_cast<float *>(staged);
    if (tid < MT * 16) rows_of[tid] = tid < tile.count ? row_at(a, tile.first + tid) : -1;
    const float scale = tile.rank == 0 ? 0.0f : a.scale ? a.scale[tile.adapter] : 1.0f;
    const int cells = HALF ? a.rank / 4 : steps * 4; // of 4 ranks, a row
    for (int i = tid; i < MT * 16 * cells; i += 256) {
        const int m = i / cells, r = 4 * (i - m * cells);
        f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
        if (m < tile.count && r < tile.rank) {
            const float *h = a.h + (int64_t)(tile.first + m) * a.wide + p * a.rank + r;
            for (int k = 0; k < a.slices; ++k) s += *reinterpret_cast<const f32x4 *>(h + (int64_t)k * a.rows * a.wide);
#pragma unroll
            for (int j = 0; j < 4; ++j) s[j] = r + j < tile.rank ? s[j] * scale : 0.0f;
        }
        if constexpr (HALF) {
#pragma unroll
            for (int part = 0; part < PARTS; ++part) {
                const uint32_t lo = to_bf16(s[0], s[1]), hi = to_bf16(s[2], s[3]);
                *reinterpret_cast<uint2 *>(hb + m * stride + part * a.rank + r) = make_uint2(lo, hi);
                s[0] -= __uint_as_float(lo << 16), s[1] -= __uint_as_float(lo & 0xffff0000u);
                s[2] -= __uint_as_float(hi << 16), s[3] -= __uint_as_float(hi & 0xffff0000u);
            }
        } else {
            *reinterpret_cast<f32x4 *>(hf + m * stride + r) = s;
        }
    }
    if constexpr (HALF) { // what the last operation reads past the parts
        const int pad = steps * 4 - PARTS * octets;
        for (int i = tid; i < MT * 16 * pad; i += 256)
            *reinterpret_cast<uint4 *>(hb + (i / pad) * stride + PARTS * a.rank + 8 * (i % pad)) = make_uint4(0, 0, 0, 0);
    }
    __syncthreads();

    const WT *B = static_cast<const WT *>(a.B) + (int64_t)tile.adapter * a.O * a.rank;
    for (int o0 = column + 64 * wave; o0 < end; o0 += 256) {
        f32x4 acc[MT][4];
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int t = 0; t < 4; ++t) acc[m][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        const int oc = o0 + 16 * quarter, left = end - oc;
        Eight<YT> ye[MT][2];
        if (tile.count > 0) {
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const int32_t row = rows_of[m * 16 + r16];
                const YT *y = static_cast<const YT *>(a.y) + (int64_t)max(row, 0) * a.ldy + oc;
                ye[m][0].load(y, row < 0 ? 0 : left);
                ye[m][1].load(y + 8, row < 0 ? 0 : left - 8);
            }
        }
        if (tile.rank > 0) {
            for (int k = 0; k < steps; ++k) {
                if constexpr (HALF) {
                    const int octet = 4 * k + quarter, r = 8 * (octet % octets);
                    const bool there = octet < PARTS * octets && r < tile.rank;
                    bf16x8 hv[MT];
#pragma unroll
                    for (int m = 0; m < MT; ++m) hv[m] = *reinterpret_cast<const bf16x8 *>(hb + (m * 16 + r16) * stride + 32 * k + 8 * quarter);
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        const int o = min(o0 + 16 * (r16 >> 2) + 4 * t + (r16 & 3), end - 1);
                        u32x4 b = {0, 0, 0, 0};
                        if (there) b = *reinterpret_cast<const u32x4 *>(reinterpret_cast<const uint16_t *>(B) + (int64_t)o * a.rank + r);
                        if (r + 8 > tile.rank)
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                if (r + 2 * j >= tile.rank) b[j] = 0;
                                else if (r + 2 * j + 1 >= tile.rank) b[j] &= 0xffffu;
                            }
#pragma unroll
                        for (int m = 0; m < MT; ++m) acc[m][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, b), hv[m], acc[m][t], 0, 0, 0);
                    }
                } else {
                    const int r = 16 * k + 4 * quarter;
                    f32x4 hv[MT];
#pragma unroll
                    for (int m = 0; m < MT; ++m) hv[m] = *reinterpret_cast<const f32x4 *>(hf + (m * 16 + r16) * stride + r);
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        const int o = min(o0 + 16 * (r16 >> 2) + 4 * t + (r16 & 3), end - 1);
                        f32x4 b = {0.0f, 0.0f, 0.0f, 0.0f};
                        if (r < tile.rank) b = *reinterpret_cast<const f32x4 *>(reinterpret_cast<const float *>(B) + (int64_t)o * a.rank + r);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float bj = r + j < tile.rank ? b[j] : 0.0f;
#pragma unroll
                            for (int m = 0; m < MT; ++m) acc[m][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(bj, hv[m][j], acc[m][t], 0, 0, 0);
                        }
                    }
                }
            }
        }
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const int32_t row = rows_of[m * 16 + r16];
            if (row < 0) continue;
            YT *out = static_cast<YT *>(a.out) + (int64_t)row * a.ldo + oc;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                float v[8];
                ye[m][half].widen(v);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] += acc[m][2 * half + j / 4][j % 4];
                if (tile.rank > 0) ye[m][half].round(v);
                ye[m][half].store(out + 8 * half, left - 8 * half);
            }
        }
    }
}

constexpr int COLUMNS = 256; // a workgroup's at a time

template <typename WT, typename YT>
__global__ __launch_bounds__(256) void up_kernel(const ApplyArgs a)
{
    extern __shared__ __align__(16) uint8_t staged[];
    __shared__ int32_t rows_of[TILE];
    const int blocks = a.block_end[a.n_parts - 1], block = (int)(blockIdx.x % (uint32_t)blocks);
    const Tile tile = tile_of(a, blockIdx.x / (uint32_t)blocks);
    if (tile.count == 0 || (tile.rank == 0 && a.out == a.y)) return;
    int p = 0, b = block, from = 0;
    for (int k = 0; k + 1 < QLLM_ADAPTER_PARTS; ++k)
        if (p == k && k + 1 < a.n_parts && block >= a.block_end[k]) p = k + 1, b = block - a.block_end[k], from = a.part_end[k];
    const int column = from + b * COLUMNS, end = min(column + COLUMNS, a.part_end[p]);
    if (tile.count <= 16) up_tile<WT, YT, 1>(a, tile, p, column, end, staged, rows_of);
    else up_tile<WT, YT, 4>(a, tile, p, column, end, staged, rows_of);
}

int32_t launched(const char *what)
{
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return QLLM_OK;
    qllm_note_hip_error(what, hipGetErrorName(e));
    return QLLM_ERR_HIP;
}

bool misses(const void *p, int64_t to) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(to - 1)) != 0; }

int32_t check_sizes(const qllm_adapters *w, int64_t rows)
{
    if (!w) return QLLM_ERR_NULL;
    if (rows < 0 || rows >= MOST_ROWS || w->n_adapters <= 0 || w->n_adapters > MOST_ADAPTERS) return QLLM_ERR_SHAPE;
    if (w->C <= 0 || w->C >= (1 << 24) || w->O <= 0 || w->O >= (1 << 24)) return QLLM_ERR_SHAPE;
    if (w->rank <= 0 || w->rank > 256 || w->rank % 8 != 0 || w->n_parts < 1 || w->n_parts > QLLM_ADAPTER_PARTS) return QLLM_ERR_SHAPE;
    int64_t sum = 0;
    for (int p = 0; p < w->n_parts; ++p) {
        if (w->part_O[p] <= 0 || w->part_O[p] > w->O) return QLLM_ERR_SHAPE;
        sum += w->part_O[p];
    }
    return sum == w->O ? QLLM_OK : QLLM_ERR_SHAPE;
}

// The slices of C: as many as fill the card with tiles (the most there can be), none shorter than a turn of the four waves.
void slices_of(const qllm_adapters *w, int64_t rows, int32_t *slices, int32_t *blocks_per_slice)
{
    const int64_t blocks = (w->C + 63) / 64, turns = (blocks + 3) / 4, groups = (w->n_parts * w->rank + 63) / 64;
    const int64_t tiles = most_tiles(rows, w->n_adapters) * groups;
    const int64_t want = tiles > 0 ? (1024 + tiles - 1) / tiles : 1, most = want < turns ? want : turns;
    const int64_t each = (turns + most - 1) / most;
    *blocks_per_slice = (int32_t)(4 * each);
    *slices = (int32_t)((turns + each - 1) / each);
}

} // namespace

extern "C" int64_t qllm_adapter_plan_bytes(int64_t rows, int64_t n_adapters)
{
    if (rows < 0 || rows >= MOST_ROWS || n_adapters <= 0 || n_adapters > MOST_ADAPTERS) return QLLM_ERR_SHAPE;
    return plan_words(rows, n_adapters) * 4;
}

extern "C" int32_t qllm_adapter_plan(int64_t rows, int64_t n_seqs, const int32_t *row_start, const int32_t *adapter, int64_t n_adapters,
                                     void *plan, int64_t plan_bytes, void *hip_stream)
{
    const int64_t need = qllm_adapter_plan_bytes(rows, n_adapters);
    if (need < 0) return QLLM_ERR_SHAPE;
    if (n_seqs < 0 || n_seqs > MOST_SEQS || (!row_start && n_seqs > rows)) return QLLM_ERR_SHAPE;
    if (!plan || (n_seqs > 0 && !adapter)) return QLLM_ERR_NULL;
    if (misses(plan, 16) || misses(row_start, 4) || misses(adapter, 4)) return QLLM_ERR_ALIGN;
    if (plan_bytes < need) return QLLM_ERR_WORKSPACE;
    (void)hipGetLastError();
    hipLaunchKernelGGL(adapter_plan_kernel, dim3(1), dim3(PLAN_THREADS), 0, reinterpret_cast<hipStream_t>(hip_stream), (int32_t)rows, (int32_t)n_seqs,
                       row_start, adapter, (int32_t)n_adapters, (int32_t)most_tiles(rows, n_adapters), static_cast<int32_t *>(plan));
    return launched("adapter plan: launch");
}

extern "C" int64_t qllm_adapter_workspace_bytes(const qllm_adapters *w, int64_t rows)
{
    const int32_t rc = check_sizes(w, rows);
    if (rc != QLLM_OK) return rc;
    int32_t slices, each;
    slices_of(w, rows, &slices, &each);
    return slices * rows * w->n_parts * w->rank * (int64_t)sizeof(float);
}

namespace {

template <typename XT, typename WT>
void run_down(const ApplyArgs &a, unsigned tiles, hipStream_t stream)
{
    const int frags = (a.wide + 15) / 16;
    const dim3 grid(tiles, (unsigned)a.slices, (unsigned)((frags + 3) / 4));
    if (frags == 1) hipLaunchKernelGGL((down_kernel<XT, WT, 1>), grid, dim3(256), 0, stream, a);
    else if (frags == 2) hipLaunchKernelGGL((down_kernel<XT, WT, 2>), grid, dim3(256), 0, stream, a);
    else if (frags == 3) hipLaunchKernelGGL((down_kernel<XT, WT, 3>), grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((down_kernel<XT, WT, 4>), grid, dim3(256), 0, stream, a);
}

template <typename WT, typename YT>
int32_t run_up(const ApplyArgs &a, unsigned tiles, hipStream_t stream)
{
    constexpr int PARTS = sizeof(WT) == 2 ? (sizeof(YT) == 2 ? 2 : 3) : 1;
    const size_t lds = sizeof(WT) == 2 ? (size_t)TILE * ((PARTS * a.rank / 8 + 3) / 4 * 32 + 8) * 2 : (size_t)TILE * ((a.rank + 15) / 16 * 16 + 4) * 4;
    auto *kernel = up_kernel<WT, YT>;
    if (lds > 48 * 1024) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) {
            (void)hipGetLastError();
            qllm_note_hip_error("adapters: raising the LDS limit", hipGetErrorName(e));
            return QLLM_ERR_HIP;
        }
    }
    hipLaunchKernelGGL(kernel, dim3((unsigned)a.block_end[a.n_parts - 1] * tiles), dim3(256), lds, stream, a);
    return QLLM_OK;
}

} // namespace

extern "C" int32_t qllm_adapter_apply(const void *x, int32_t x_dtype, int64_t ldx, int64_t rows, const qllm_adapters *w, const void *plan,
                                      int64_t plan_bytes, const void *y, int64_t ldy, void *out, int64_t ldo, int32_t y_dtype,
                                      void *workspace, int64_t workspace_bytes, void *hip_stream)
{
    const int32_t rc = check_sizes(w, rows);
    if (rc != QLLM_OK) return rc;
    for (int32_t d : {x_dtype, y_dtype, w->w_dtype})
        if (d != QLLM_F32 && d != QLLM_BF16) return QLLM_ERR_DTYPE;
    if (ldx < w->C || ldy < w->O || ldo < w->O || (out == y && ldo != ldy)) return QLLM_ERR_SHAPE;
    if (rows == 0) return QLLM_OK;
    if (!x || !w->A || !w->B || !plan || !y || !out) return QLLM_ERR_NULL;
    const int64_t xs = x_dtype == QLLM_BF16 ? 2 : 4, ys = y_dtype == QLLM_BF16 ? 2 : 4;
    if (misses(x, xs) || misses(y, ys) || misses(out, ys) || misses(w->A, 16) || misses(w->B, 16) || misses(plan, 16) || misses(workspace, 16) ||
        misses(w->scale, 4) || misses(w->ranks, 4))
        return QLLM_ERR_ALIGN;
    if (plan_bytes < qllm_adapter_plan_bytes(rows, w->n_adapters)) return QLLM_ERR_WORKSPACE;
    if (!workspace || workspace_bytes < qllm_adapter_workspace_bytes(w, rows)) return QLLM_ERR_WORKSPACE;

    ApplyArgs a{};
    a.x = x, a.A = w->A, a.B = w->B, a.y = y, a.out = out;
    a.ldx = ldx, a.ldy = ldy, a.ldo = ldo, a.C = w->C, a.O = w->O;
    a.scale = w->scale, a.ranks = w->ranks, a.plan = static_cast<const int32_t *>(plan), a.h = static_cast<float *>(workspace);
    a.rows = (int32_t)rows, a.n_adapters = (int32_t)w->n_adapters, a.rank = (int32_t)w->rank, a.wide = (int32_t)(w->n_parts * w->rank);
    slices_of(w, rows, &a.slices, &a.blocks_per_slice);
    a.n_parts = w->n_parts;
    for (int p = 0; p < w->n_parts; ++p) {
        a.part_end[p] = (int32_t)w->part_O[p] + (p ? a.part_end[p - 1] : 0);
        a.block_end[p] = (int32_t)((w->part_O[p] + COLUMNS - 1) / COLUMNS) + (p ? a.block_end[p - 1] : 0);
    }
    const int64_t tiles = most_tiles(rows, w->n_adapters);
    if (tiles * a.block_end[a.n_parts - 1] > INT32_MAX) return QLLM_ERR_SHAPE;
    hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
    (void)hipGetLastError();
    const bool xb = x_dtype == QLLM_BF16, wb = w->w_dtype == QLLM_BF16, yb = y_dtype == QLLM_BF16;
    if (wb) xb ? run_down<uint16_t, uint16_t>(a, (unsigned)tiles, stream) : run_down<float, uint16_t>(a, (unsigned)tiles, stream);
    else xb ? run_down<uint16_t, float>(a, (unsigned)tiles, stream) : run_down<float, float>(a, (unsigned)tiles, stream);
    if (const int32_t e = launched("adapters, first product: launch")) return e;
    if (a.slices > 1 && rows > TILE) {
        const int64_t words4 = rows * a.wide / 4;
        hipLaunchKernelGGL(join_kernel, dim3((unsigned)((words4 + 255) / 256)), dim3(256), 0, stream, a.h, words4, a.slices);
        if (const int32_t e = launched("adapters, sums: launch")) return e;
        a.slices = 1;
    }
    int32_t done;
    if (wb) done = yb ? run_up<uint16_t, uint16_t>(a, (unsigned)tiles, stream) : run_up<uint16_t, float>(a, (unsigned)tiles, stream);
    else done = yb ? run_up<float, uint16_t>(a, (unsigned)tiles, stream) : run_up<float, float>(a, (unsigned)tiles, stream);
    return done != QLLM_OK ? done : launched("adapters, second product: launch");
}
