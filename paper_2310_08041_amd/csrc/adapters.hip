// Low-rank adapters of many requests beside a shared projection: out = y + scale_a (x A_a^T) B_a^T, each row with its own a.
//
// What it has to move is x of the rows, the factors of the adapters that are named, y in and out; the operations are few
// (2 rank (C + O) a row), so it is bound by memory, and for a few rows by latency.
//   adapter_plan_kernel    once a step: the rows sorted by adapter, in tiles of up to 64 rows of one adapter
//   down_kernel            h = x A^T of a tile over a slice of C, fp32, a part of the sum per slice
//   join_kernel            where the slices of many rows are to be added: their sum
//   up_kernel              out = y + (scale h) B^T of a tile over a block of columns
// Measured: 2048 rows, 28672 -> 8192, 64 ranks, float32 y 32 + 5 + 32 us (x at 3.7 TB/s, y in and out at 4.2); 4360 rows, 5120 -> 27648 bf16
// 18 + 5 + 110 (y at 4.4); one token 4096 -> 4096 3.5 + 5.5, four dependent trips to memory and the launch.
// No sum uses atomics, and a row's sums do not depend on its place in a tile: equal calls give equal bits.
#include <hip/hip_runtime.h>

#include <stdint.h>

#include "fused_common.h"
#include "lds_limit.h"
#include "qllm_block.h"
#include "rows.h"

using namespace qllm_detail;

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int TILE = 64;             // rows of a tile
constexpr int PLAN_HEAD_WORDS = 4;   // {tiles, rows, adapters of the pool, -}
constexpr int PLAN_THREADS = 1024;
constexpr int MOST_ADAPTERS = 8192, MOST_RANKS = 256;
constexpr int64_t MOST_ROWS = 1 << 24, MOST_SEQS = 1 << 20;
constexpr int64_t MOST_BLOCKS = 1 << 24; // of 256 lanes: a launch counts its lanes in 32 bits

inline int64_t most_tiles(int64_t rows, int64_t n_adapters)
{
    const int64_t groups = n_adapters + 1; // those without one are a group too
    return rows / TILE + (rows < groups ? rows : groups);
}
// words: head, tiles of {adapter, rows of the tiles before it, its rows, -}, then TILE rows for each tile, so that a workgroup asks for
// all it needs of the plan at once
inline int64_t plan_words(int64_t rows, int64_t n_adapters) { return PLAN_HEAD_WORDS + (4 + TILE) * most_tiles(rows, n_adapters); }

// ---- the plan: rows counted per adapter, the adapters' tiles numbered, the sequences put there.  In which order the
// sequences of one adapter come (an atomic decides) is no part of any result.
__global__ __launch_bounds__(PLAN_THREADS) void adapter_plan_kernel(int32_t rows, int32_t n_seqs, const int32_t *row_start,
                                                                   const int32_t *adapter, int32_t n_adapters, int32_t most, int32_t *plan)
{
    __shared__ uint32_t next[MOST_ADAPTERS + 1]; // rows of an adapter, then the next free place of its own; group n_adapters: none
    __shared__ uint32_t part_rows[PLAN_THREADS / 64], part_tiles[PLAN_THREADS / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int groups = n_adapters + 1;
    int4 *tiles = reinterpret_cast<int4 *>(plan + PLAN_HEAD_WORDS);
    int32_t *order = plan + PLAN_HEAD_WORDS + 4 * (int64_t)most;
    const int64_t places = (int64_t)most * TILE;
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
        next[g] = min(before_tiles, (uint32_t)most) * TILE;
        for (uint32_t at = 0; at < n; at += TILE, ++before_tiles)
            if (before_tiles < (uint32_t)most) tiles[before_tiles] = make_int4(g, (int32_t)min(before_rows + at, (uint32_t)rows), (int32_t)min(n - at, (uint32_t)TILE), 0);
        before_rows += n;
    }
    if (tid == 0) *reinterpret_cast<int4 *>(plan) = make_int4((int32_t)min(all_tiles, (uint32_t)most), rows, n_adapters, 0);
    __syncthreads();
    if (!row_start) {
        for (int i = tid; i < min(n_seqs, rows); i += PLAN_THREADS) {
            const uint32_t at = atomicAdd(&next[group_of(i)], 1u);
            if (at < places) order[at] = i;
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
            if ((int64_t)at + j < places) order[(int64_t)at + j] = row + j;
    }
}

struct ApplyArgs {
    const void *x, *A, *B, *y;
    void *out;
    int64_t ldx, ldy, ldo, C, O;
    const float *scale;
    const int32_t *ranks, *plan;
    float *h; // [slices][rows in the order of the tiles][parts * rank]
    int32_t rows, n_adapters, most, rank, wide, slices, blocks_per_slice; // most: tiles; wide: parts * rank; blocks of 64 channels
    QuotientBy by_rank, by_cells, by_slices, by_blocks; // the last two: m 0 where a launch is too large for the multiplication
    bool stream; // y and out past the caches, which B and h need
    int32_t n_parts, part_end[QLLM_ADAPTER_PARTS], columns, block_end[QLLM_ADAPTER_PARTS]; // columns, of a block, blocks, summed up
};

__device__ __forceinline__ uint32_t divide(uint32_t x, const QuotientBy &by) { return by.m || by.d == 1u ? by.divide(x) : x / by.d; }

struct Tile {
    int32_t adapter, first, count, rank; // count 0: none
    const int32_t *rows;
};
// tile t < most_tiles(...): its words are there to be read whatever they hold
__device__ __forceinline__ Tile tile_of(const ApplyArgs &a, uint32_t t)
{
    const int4 head = *reinterpret_cast<const int4 *>(a.plan), w = reinterpret_cast<const int4 *>(a.plan + PLAN_HEAD_WORDS)[t];
    Tile tile{0, 0, 0, 0, a.plan + PLAN_HEAD_WORDS + 4 * (int64_t)a.most + (int64_t)t * TILE};
    if (head.y != a.rows || head.z != a.n_adapters || t >= (uint32_t)head.x) return tile;
    if (w.x < 0 || w.x > a.n_adapters || w.y < 0 || w.y >= a.rows || w.z <= 0) return tile;
    tile.adapter = w.x, tile.first = w.y, tile.count = min(min(w.z, TILE), a.rows - w.y);
    if (w.x < a.n_adapters) tile.rank = a.ranks ? min(max(a.ranks[w.x], 0), a.rank) : a.rank;
    return tile;
}
__device__ __forceinline__ int32_t checked_row(const ApplyArgs &a, int32_t row) { return row >= 0 && row < a.rows ? row : -1; }

// A lane's share of a block of 32 H channels of one row of x or A, 128 bytes of x (four lanes a row): channels 8 q .. + 7 of each 32.
template <typename T, int H>
struct Share {
    Eight<T> e[H];
    __device__ __forceinline__ void load(const T *p, int n)
    {
#pragma unroll
        for (int h = 0; h < H; ++h) e[h].load(p + 32 * h, n - 32 * h);
    }
};

// ---- h = x A^T.  Lane l of a wave holds its share (q = l / 16) of row l mod 16 of either operand; the order of the channels is the
// same in both, so any will do.  The four waves take the slice's blocks in turn, the next one's loads in flight.  64 rows a wave read A
// once for all of them (32 rows a wave 46.9 us, 64 36.5, before the tile's slices lay next to each other).
template <typename XT, typename WT, int MT, int NT>
__device__ __forceinline__ void down_tile(const ApplyArgs &a, const Tile &tile, int slice, int first_rank, float *part)
{
    constexpr bool HALF = sizeof(XT) == 2 && sizeof(WT) == 2;
    constexpr int H = HALF ? 2 : 1, BLOCK = 32 * H; // the same for any MT: a row's sums do not depend on its tile's other rows
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r16 = lane & 15, quarter = lane >> 4;
    const XT *x[MT];
    const WT *w[NT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const int32_t row = checked_row(a, tile.rows[min(m * 16 + r16, tile.count - 1)]);
        x[m] = static_cast<const XT *>(a.x) + (int64_t)max(row, 0) * a.ldx + 8 * quarter;
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int at = min(first_rank + n * 16 + r16, a.wide - 1), p = (int)a.by_rank.divide((uint32_t)at), r = min(at - p * a.rank, tile.rank - 1);
        w[n] = static_cast<const WT *>(a.A) + ((int64_t)tile.adapter * a.wide + p * a.rank + r) * a.C + 8 * quarter;
    }
    f32x4 acc[MT][NT];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[m][n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const int C = (int)a.C, begin = slice * a.blocks_per_slice * 64, end = min(begin + a.blocks_per_slice * 64, C);
    Share<XT, H> xe[MT];
    Share<WT, H> we[NT];
    auto request = [&](int c) {
        if (c + BLOCK <= C) {
#pragma unroll
            for (int m = 0; m < MT; ++m) xe[m].load(x[m] + c, BLOCK);
#pragma unroll
            for (int n = 0; n < NT; ++n) we[n].load(w[n] + c, BLOCK);
        } else { // the row's last block
            const int left = C - c - 8 * quarter;
#pragma unroll
            for (int m = 0; m < MT; ++m) xe[m].load(x[m] + c, left);
#pragma unroll
            for (int n = 0; n < NT; ++n) we[n].load(w[n] + c, left);
        }
    };
    int c = begin + BLOCK * wave;
    if (c < end) request(c);
    for (; c < end; c += BLOCK * 4) {
        Share<XT, H> xn[MT];
        Share<WT, H> wn[NT];
#pragma unroll
        for (int m = 0; m < MT; ++m) xn[m] = xe[m];
#pragma unroll
        for (int n = 0; n < NT; ++n) wn[n] = we[n];
        if (c + BLOCK * 4 < end) request(c + BLOCK * 4);
#pragma unroll
        for (int h = 0; h < H; ++h) {
            if constexpr (HALF) {
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
                        acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, wn[n].e[h].q), __builtin_bit_cast(bf16x8, xn[m].e[h].q), acc[m][n], 0, 0, 0);
            } else {
                float xv[MT][8], wv[NT][8];
#pragma unroll
                for (int m = 0; m < MT; ++m) xn[m].e[h].widen(xv[m]);
#pragma unroll
                for (int n = 0; n < NT; ++n) wn[n].e[h].widen(wv[n]);
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
    float *h = a.h + ((int64_t)slice * a.rows + tile.first) * a.wide + first_rank;
    for (int i = threadIdx.x; i < MT * 16 * NT * 4; i += 256) {
        const int row = i / (NT * 4), r4 = i - row * (NT * 4);
        if (row >= tile.count || first_rank + 4 * r4 >= a.wide) continue;
        f32x4 s = *reinterpret_cast<const f32x4 *>(part + row * (NT * 16) + 4 * r4);
#pragma unroll
        for (int v = 1; v < 4; ++v) s += *reinterpret_cast<const f32x4 *>(part + (v * MT * 16 + row) * (NT * 16) + 4 * r4);
        *reinterpret_cast<f32x4 *>(h + (int64_t)row * a.wide + 4 * r4) = s;
    }
}

// Neighbouring workgroups, on XCDs in turn, are a tile's slices: with 8 slices, or 16, a slice's part of A is in one L2 alone.
template <typename XT, typename WT, int NT>
__global__ __launch_bounds__(256, 2) void down_kernel(const ApplyArgs a)
{
    __shared__ __align__(16) float part[4 * TILE * NT * 16];
    const uint32_t t = divide(blockIdx.x, a.by_slices);
    const int slice = (int)(blockIdx.x - t * a.by_slices.d);
    const Tile tile = tile_of(a, t);
    if (tile.count == 0 || tile.rank == 0) return;
    const int first_rank = blockIdx.y * NT * 16;
    if (tile.count <= 16) down_tile<XT, WT, 1, NT>(a, tile, slice, first_rank, part);
    else down_tile<XT, WT, 4, NT>(a, tile, slice, first_rank, part);
}

// ---- the slices' sums: JOINERS neighbouring lanes add up every JOINERS-th slice each, then theirs are added
// (by the second product itself for few rows and ranks: 64 rows on as many adapters would gain 1 us with it, 256 rows on 8 lose 2, on 2 8)
constexpr int JOINERS = 8, JOINED = 32, JOINED_ROWS = 16, JOINED_RANKS = 1024;
__device__ __forceinline__ f32x4 slices_of_lane(const float *h, int64_t stride, int slices, int joiner)
{
    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int k0 = joiner; k0 < slices; k0 += 4 * JOINERS) { // four loads in flight; what is past the last slice is read from it, and dropped
        f32x4 v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] = *reinterpret_cast<const f32x4 *>(h + min(k0 + u * JOINERS, slices - 1) * stride);
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (k0 + u * JOINERS < slices) s += v[u];
    }
    return s;
}
__device__ __forceinline__ f32x4 over_joiners(f32x4 s)
{
#pragma unroll
    for (int d = 1; d < JOINERS; d <<= 1) {
        f32x4 o;
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = __shfl_xor(s[j], d, 64);
        s += o;
    }
    return s;
}

__global__ __launch_bounds__(256) void join_kernel(float *h, int64_t words4, int32_t slices)
{
    const int64_t i = (int64_t)blockIdx.x * (256 / JOINERS) + threadIdx.x / JOINERS, at = i < words4 ? i : words4 - 1;
    const f32x4 s = over_joiners(slices_of_lane(h + 4 * at, 4 * words4, slices, threadIdx.x % JOINERS));
    if (i < words4 && threadIdx.x % JOINERS == 0) reinterpret_cast<f32x4 *>(h)[at] = s;
}

// ---- out = y + (scale h) B^T.  Rows are the rows of the matrix operation and four operations take the columns 4 n + t, t = 0 .. 3, so
// that lane l gets 4 neighbouring columns of 4 rows and 16 lanes a whole piece of a row of y: its reads and writes are whole lines.
// h goes through LDS, with bf16 weights as PARTS bf16 numbers that add up to it, behind one another in a row.
template <typename T, bool STREAM>
struct Four; // 4 neighbouring elements of a row of y; STREAM: past the caches
template <bool STREAM>
struct Four<float, STREAM> {
    u32x4 q;
    __device__ __forceinline__ void load(const float *p, int n)
    {
        if (n >= 4) {
            if constexpr (STREAM) q = __builtin_nontemporal_load(reinterpret_cast<const u32x4_at4 *>(p));
            else q = *reinterpret_cast<const u32x4_at4 *>(p);
        } else {
            q = u32x4{0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < 3; ++j)
                if (j < n) q[j] = __float_as_uint(p[j]);
        }
    }
    __device__ __forceinline__ void add(const float *v)
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) q[j] = __float_as_uint(__uint_as_float(q[j]) + v[j]);
    }
    __device__ __forceinline__ void store(float *p, int n) const
    {
        if (n >= 4) {
            if constexpr (STREAM) __builtin_nontemporal_store(q, reinterpret_cast<u32x4_at4 *>(p));
            else *reinterpret_cast<u32x4_at4 *>(p) = q;
        } else {
#pragma unroll
            for (int j = 0; j < 3; ++j)
                if (j < n) p[j] = __uint_as_float(q[j]);
        }
    }
};
template <bool STREAM>
struct Four<uint16_t, STREAM> {
    u32x2 q;
    __device__ __forceinline__ void load(const uint16_t *p, int n)
    {
        if (n >= 4) {
            if constexpr (STREAM) q = __builtin_nontemporal_load(reinterpret_cast<const u32x2_at2 *>(p));
            else q = *reinterpret_cast<const u32x2_at2 *>(p);
        } else {
            q = u32x2{0, 0};
#pragma unroll
            for (int j = 0; j < 3; ++j)
                if (j < n) q[j / 2] |= (uint32_t)p[j] << (16 * (j & 1));
        }
    }
    __device__ __forceinline__ void add(const float *v)
    {
#pragma unroll
        for (int k = 0; k < 2; ++k) q[k] = to_bf16(__uint_as_float(q[k] << 16) + v[2 * k], __uint_as_float(q[k] & 0xffff0000u) + v[2 * k + 1]);
    }
    __device__ __forceinline__ void store(uint16_t *p, int n) const
    {
        if (n >= 4) {
            if constexpr (STREAM) __builtin_nontemporal_store(q, reinterpret_cast<u32x2_at2 *>(p));
            else *reinterpret_cast<u32x2_at2 *>(p) = q;
        } else {
#pragma unroll
            for (int j = 0; j < 3; ++j)
                if (j < n) p[j] = (uint16_t)(q[j / 2] >> (16 * (j & 1)));
        }
    }
};

// Ranks that one step of the second product takes, and elements of a row of h in LDS.
template <typename WT>
constexpr int STEP = sizeof(WT) == 2 ? 32 : 16;
// Three bf16 numbers hold all 24 bits of h, whatever y's type: two leave out 2^-17 of each rank, which shows in a bf16 result where the
// ranks cancel (and in 1 of 10^3 outputs otherwise, as a rounding the other way).
template <typename WT>
constexpr int PARTS = sizeof(WT) == 4 ? 1 : 3;
template <typename WT>
__host__ __device__ __forceinline__ int staged_stride(int rank)
{
    return PARTS<WT> * ((rank + STEP<WT> - 1) / STEP<WT> * STEP<WT>) + (sizeof(WT) == 2 ? 8 : 4);
}

// A wave has MT groups of 16 rows and 64 columns at a time, the next columns' y and B in flight; the waves of a workgroup share out the
// tile's rows and then its columns.  WHOLE: no column of the last 64 is past the end.
template <typename WT, typename YT, int MT, bool WHOLE, bool STREAM>
__device__ __forceinline__ void up_tile(const ApplyArgs &a, const Tile &tile, int p, int column, int end, uint8_t *staged)
{
    constexpr bool HALF = sizeof(WT) == 2;
    constexpr int P = PARTS<WT>, S = STEP<WT>;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r16 = lane & 15, quarter = lane >> 4;
    const int sharers = tile.count <= 16 * MT ? 1 : 2; // groups of MT * 16 rows
    const int first = 16 * MT * (wave & (sharers - 1)), turns = 4 / sharers;
    const YT *y[MT][4];
    bool there[MT][4];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const int at = first + 16 * m + 4 * quarter;
        const int4 four = *reinterpret_cast<const int4 *>(tile.rows + at);
        const int32_t rows[4] = {four.x, four.y, four.z, four.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int32_t row = at + i < tile.count ? checked_row(a, rows[i]) : -1;
            there[m][i] = row >= 0;
            y[m][i] = static_cast<const YT *>(a.y) + (int64_t)max(row, 0) * a.ldy + column + 4 * r16;
        }
    }
    // B of 4 columns a lane in a step: ranks 8 q .. + 7 (bf16) or 4 q .. + 3 (fp32) of each
    const WT *B = static_cast<const WT *>(a.B) + ((int64_t)min(tile.adapter, a.n_adapters - 1) * a.O + column) * a.rank;
    const int steps = (tile.rank + S - 1) / S;
    auto load_b = [&](u32x4 *b, int at, int step) { // at: of the workgroup's columns
        const int r = step * S + quarter * (S / 4), o = at + 4 * r16;
        const uint32_t from = r < tile.rank ? r : 0;
#pragma unroll
        for (int t = 0; t < 4; ++t) b[t] = *reinterpret_cast<const u32x4 *>(B + (uint32_t)((WHOLE ? o + t : min(o + t, end - column - 1)) * a.rank + from));
    };
    auto mask_b = [&](u32x4 *b, int step) { // past the adapter's own ranks: zeros
        if (tile.rank >= (step + 1) * S) return;
        const int r = step * S + quarter * (S / 4);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int one = HALF ? r + 2 * j : r + j;
            const uint32_t keep = one >= tile.rank ? 0u : HALF && one + 1 >= tile.rank ? 0xffffu : 0xffffffffu;
#pragma unroll
            for (int t = 0; t < 4; ++t) b[t][j] &= keep;
        }
    };
    Four<YT, STREAM> ye[MT][4];
    // steps of B asked for with the columns: for prompts one, whose registers count more (5120 -> 27648 109 us, two 120, three 121), for single
    // tokens two (16 adapters of up to 64 ranks 8.5, one 9.6)
    constexpr int AHEAD = MT == 1 ? 2 : 1;
    u32x4 b[AHEAD][4];
    auto request = [&](int at) {
        const int left = WHOLE ? 64 : end - column - at - 4 * r16;
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) ye[m][i].load(y[m][i] + at, left);
#pragma unroll
        for (int step = 0; step < AHEAD; ++step)
            if (step < steps) load_b(b[step], at, step);
    };
    const int width = end - column;
    int at = 64 * (wave / sharers);
    if (at < width) request(at);

    // scale h into LDS, the tile's rows (what lies in others reaches only results that are not stored)
    const int padded = (a.rank + S - 1) / S * S, stride = staged_stride<WT>(a.rank);
    if (tile.rank > 0) {
        const float scale = a.scale ? a.scale[tile.adapter] : 1.0f;
        const int cells = padded / 4, all = tile.count * cells; // of 4 ranks, a row
        const float *h = a.h + (int64_t)tile.first * a.wide + p * a.rank;
        auto stage = [&](int i, f32x4 s) {
            const int row = (int)a.by_cells.divide((uint32_t)i), r = 4 * (i - row * cells);
#pragma unroll
            for (int j = 0; j < 4; ++j) s[j] = r + j < tile.rank ? s[j] * scale : 0.0f;
            if constexpr (HALF) {
                uint16_t *to = reinterpret_cast<uint16_t *>(staged) + row * stride + r;
#pragma unroll
                for (int part = 0; part < P; ++part) { // the upper 8 bits of what is left, which are never past the largest bf16
                    uint32_t upper[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) upper[j] = __float_as_uint(s[j]) & 0xffff0000u, s[j] -= __uint_as_float(upper[j]);
                    *reinterpret_cast<uint2 *>(to + part * padded) = make_uint2(upper[0] >> 16 | upper[1], upper[2] >> 16 | upper[3]);
                }
            } else {
                *reinterpret_cast<f32x4 *>(reinterpret_cast<float *>(staged) + row * stride + r) = s;
            }
        };
        auto cell = [&](int i) { // any i: that of a rank or row past the end is read at another place
            const int row = (int)a.by_cells.divide((uint32_t)i);
            return h + min(row, tile.count - 1) * a.wide + min(4 * (i - row * cells), a.rank - 4);
        };
        if (a.slices > 1) {
            constexpr int AT_ONCE = 4; // trips to h in flight
            for (int i0 = tid / JOINERS; i0 < all; i0 += AT_ONCE * (256 / JOINERS)) {
                f32x4 s[AT_ONCE];
#pragma unroll
                for (int k = 0; k < AT_ONCE; ++k)
                    if (k == 0 || i0 + k * (256 / JOINERS) < all) s[k] = slices_of_lane(cell(i0 + k * (256 / JOINERS)), (int64_t)a.rows * a.wide, a.slices, tid % JOINERS);
#pragma unroll
                for (int k = 0; k < AT_ONCE; ++k) {
                    if (k > 0 && i0 + k * (256 / JOINERS) >= all) continue; // the same for a cell's eight lanes
                    s[k] = over_joiners(s[k]);
                    if (tid % JOINERS == 0) stage(i0 + k * (256 / JOINERS), s[k]);
                }
            }
        } else {
            for (int i0 = tid; i0 < all; i0 += 256 * 4) {
                f32x4 s[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) s[k] = *reinterpret_cast<const f32x4 *>(cell(i0 + 256 * k));
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (i0 + 256 * k < all) stage(i0 + 256 * k, s[k]);
            }
        }
        __syncthreads();
    }
    const WT *mine = reinterpret_cast<const WT *>(staged) + (first + r16) * stride + quarter * (S / 4);
    for (; at < width; at += 64 * turns) {
        Four<YT, STREAM> yn[MT][4];
        u32x4 bn[AHEAD][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int step = 0; step < AHEAD; ++step) bn[step][i] = b[step][i];
#pragma unroll
            for (int m = 0; m < MT; ++m) yn[m][i] = ye[m][i];
        }
        if (at + 64 * turns < width) request(at + 64 * turns);
        f32x4 acc[MT][4];
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int t = 0; t < 4; ++t) acc[m][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        for (int step = 0; step < steps; ++step) {
            u32x4 now[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                now[t] = bn[0][t];
#pragma unroll
                for (int k = 1; k < AHEAD; ++k) bn[k - 1][t] = bn[k][t];
            }
            if (step + AHEAD < steps) load_b(bn[AHEAD - 1], at, step + AHEAD);
            mask_b(now, step);
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                if constexpr (HALF) {
#pragma unroll
                    for (int part = 0; part < P; ++part) {
                        const bf16x8 h = *reinterpret_cast<const bf16x8 *>(mine + m * 16 * stride + part * padded + S * step);
#pragma unroll
                        for (int t = 0; t < 4; ++t) acc[m][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(h, __builtin_bit_cast(bf16x8, now[t]), acc[m][t], 0, 0, 0);
                    }
                } else {
                    const f32x4 h = *reinterpret_cast<const f32x4 *>(mine + m * 16 * stride + S * step);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int t = 0; t < 4; ++t) acc[m][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(h[j], __uint_as_float(now[t][j]), acc[m][t], 0, 0, 0);
                }
            }
        }
        const int left = WHOLE ? 64 : width - at - 4 * r16;
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (!there[m][i]) continue;
                const float v[4] = {acc[m][0][i], acc[m][1][i], acc[m][2][i], acc[m][3][i]};
                if (tile.rank > 0) yn[m][i].add(v); // else a copy, bit for bit
                YT *out = static_cast<YT *>(a.out) + (y[m][i] - static_cast<const YT *>(a.y)) + at;
                if (a.ldo != a.ldy) out += (int64_t)checked_row(a, tile.rows[first + 16 * m + 4 * quarter + i]) * (a.ldo - a.ldy);
                yn[m][i].store(out, left);
            }
    }
}

template <typename WT, typename YT>
__global__ __launch_bounds__(256, 2) void up_kernel(const ApplyArgs a)
{
    extern __shared__ __align__(16) uint8_t staged[];
    const uint32_t t = divide(blockIdx.x, a.by_blocks);
    const int block = (int)(blockIdx.x - t * a.by_blocks.d);
    const Tile tile = tile_of(a, t);
    if (tile.count == 0 || (tile.rank == 0 && a.out == a.y)) return;
    int p = 0, b = block, from = 0;
    for (int k = 0; k + 1 < QLLM_ADAPTER_PARTS; ++k)
        if (p == k && k + 1 < a.n_parts && block >= a.block_end[k]) p = k + 1, b = block - a.block_end[k], from = a.part_end[k];
    const int column = from + b * a.columns, end = min(column + a.columns, a.part_end[p]);
    const int form = ((end - column) & 63) != 0 ? 0 : a.stream ? 2 : 1;
    if (tile.count <= 16) {
        if (form == 2) up_tile<WT, YT, 1, true, true>(a, tile, p, column, end, staged);
        else if (form == 1) up_tile<WT, YT, 1, true, false>(a, tile, p, column, end, staged);
        else up_tile<WT, YT, 1, false, false>(a, tile, p, column, end, staged);
    } else {
        if (form == 2) up_tile<WT, YT, 2, true, true>(a, tile, p, column, end, staged);
        else if (form == 1) up_tile<WT, YT, 2, true, false>(a, tile, p, column, end, staged);
        else up_tile<WT, YT, 2, false, false>(a, tile, p, column, end, staged);
    }
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
    if (w->rank <= 0 || w->rank > MOST_RANKS || w->rank % 8 != 0 || w->n_parts < 1 || w->n_parts > QLLM_ADAPTER_PARTS) return QLLM_ERR_SHAPE;
    int64_t sum = 0;
    for (int p = 0; p < w->n_parts; ++p) {
        if (w->part_O[p] <= 0 || w->part_O[p] > w->O) return QLLM_ERR_SHAPE;
        sum += w->part_O[p];
    }
    return sum == w->O ? QLLM_OK : QLLM_ERR_SHAPE;
}

// The fewest tiles that the rows can make: what a launch counts on to fill the card.
inline int64_t fewest_tiles(int64_t rows) { return rows > TILE ? (rows + TILE - 1) / TILE : 1; }

// The slices of C: two workgroups a CU, none shorter than a turn of the four waves (256 channels), for few rows two turns where that leaves
// 16 slices.  The second product adds up as many as JOINED itself, and up to 4 turns are shorter than another launch if its sums are few
// (28672 -> 8192, 16 ranks, 1 row 10.6 us, 56 slices and their sum 13.5, 16 rows on 16 adapters 12.2 : 16.3; of 64 ranks 16 rows on 2
// adapters 16.6 : 14.9; 200000 channels fp32, 25 turns, 39 : 21).
void slices_of(const qllm_adapters *w, int64_t rows, int32_t *slices, int32_t *blocks_per_slice)
{
    const int64_t turns = (w->C + 255) / 256, tiles = fewest_tiles(rows) * ((w->n_parts * w->rank + 63) / 64);
    const bool joins = rows <= JOINED_ROWS && rows * w->rank <= JOINED_RANKS / 2 && turns <= 4 * JOINED;
    const int64_t want = rows > TILE ? (512 + tiles - 1) / tiles : turns <= 32 ? 16 : joins && turns > 2 * JOINED ? JOINED : turns / 2;
    const int64_t most = want < turns ? want : turns, each = (turns + most - 1) / most;
    *blocks_per_slice = (int32_t)(4 * each);
    *slices = (int32_t)((turns + each - 1) / each);
}

// Columns of a workgroup of the second product: the multiple of 256 with the least work in a row, in rounds of three workgroups a CU (two are
// resident, and as they end at different times a round half as large again costs no more), each as long as its columns and about 300 more
// (the trips to the plan, to h, to the first y).  1700 rows x 4999 fp32 256 columns 20.9 us, 512 23.8; 4400 x 27648 bf16 256 columns
// 137, 1280 or 2048 120, 4096 156.  Up to 512 rows are taken for single tokens of many requests, whose workgroups are alike: rounds of two a
// CU, with as many tiles as there are halfway between the fewest and the most (256 rows on 12 adapters, 12288 columns, 512 columns 9.9 us,
// 256 11.3).
int32_t columns_of(const qllm_adapters *w, int64_t rows)
{
    const int64_t fewest = fewest_tiles(rows), tiles = rows <= 512 ? (fewest + most_tiles(rows, w->n_adapters)) / 2 : fewest;
    const int64_t slots = rows <= 512 ? 512 : 768;
    int64_t best = 256, least = INT64_MAX;
    for (int64_t columns = 256; columns <= 2048; columns += 256) {
        int64_t blocks = 0;
        for (int p = 0; p < w->n_parts; ++p) blocks += (w->part_O[p] + columns - 1) / columns;
        const int64_t cost = (tiles * blocks + slots - 1) / slots * (columns + 300);
        if (cost < least) least = cost, best = columns;
    }
    return (int32_t)best;
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
    // At least slices * rows, and never less for more rows: up to TILE rows slices <= turns; beyond, slices <= 512 / ceil(rows / TILE) + 1.
    const int64_t turns = (w->C + 255) / 256, few = turns * (rows < TILE ? rows : TILE), many = 512 * TILE + rows;
    const int64_t all = turns * rows < many ? turns * rows : many;
    return (few > all ? few : all) * w->n_parts * w->rank * (int64_t)sizeof(float);
}

namespace {

template <typename XT, typename WT>
void run_down(const ApplyArgs &a, unsigned tiles, hipStream_t stream)
{
    const int frags = (a.wide + 15) / 16;
    const dim3 grid(tiles * (unsigned)a.slices, (unsigned)((frags + 3) / 4));
    if (frags == 1) hipLaunchKernelGGL((down_kernel<XT, WT, 1>), grid, dim3(256), 0, stream, a);
    else if (frags == 2) hipLaunchKernelGGL((down_kernel<XT, WT, 2>), grid, dim3(256), 0, stream, a);
    else if (frags == 3) hipLaunchKernelGGL((down_kernel<XT, WT, 3>), grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((down_kernel<XT, WT, 4>), grid, dim3(256), 0, stream, a);
}

template <typename WT, typename YT>
int32_t run_up(const ApplyArgs &a, unsigned tiles, hipStream_t stream)
{
    const size_t lds = (size_t)TILE * staged_stride<WT>(a.rank) * sizeof(WT);
    auto *kernel = up_kernel<WT, YT>;
    if (lds > 48 * 1024) {
        const int32_t e = raise_lds_limit(reinterpret_cast<const void *>(kernel), TILE * staged_stride<WT>(MOST_RANKS) * (int)sizeof(WT), "adapters: raising the LDS limit");
        if (e != QLLM_OK) return e;
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
    a.most = (int32_t)most_tiles(rows, w->n_adapters), a.columns = columns_of(w, rows);
    slices_of(w, rows, &a.slices, &a.blocks_per_slice);
    a.n_parts = w->n_parts;
    for (int p = 0; p < w->n_parts; ++p) {
        a.part_end[p] = (int32_t)w->part_O[p] + (p ? a.part_end[p - 1] : 0);
        a.block_end[p] = (int32_t)((w->part_O[p] + a.columns - 1) / a.columns) + (p ? a.block_end[p - 1] : 0);
    }
    // Where rows and parts are whole lines (prompts through 5120 -> 27648 130 : 124 us); lines that two waves share are better met in the
    // caches (1700 rows of 4999 fp32 31 : 21).
    a.stream = !misses(y, 128) && !misses(out, 128) && (ldy * ys % 128 | ldo * ys % 128) == 0;
    for (int p = 0; p + 1 < w->n_parts; ++p) a.stream = a.stream && a.part_end[p] * ys % 128 == 0;
    const int64_t tiles = most_tiles(rows, w->n_adapters);
    if (tiles * a.block_end[a.n_parts - 1] >= MOST_BLOCKS) return QLLM_ERR_SHAPE;
    auto by = [](int64_t d, int64_t most) { // of numbers up to `most`
        QuotientBy q = quotient_by((uint32_t)d);
        if (most * d >= (1ll << 32)) q.m = 0;
        return q;
    };
    const int32_t step = w->w_dtype == QLLM_BF16 ? STEP<uint16_t> : STEP<float>;
    a.by_rank = quotient_by((uint32_t)w->rank), a.by_cells = quotient_by((uint32_t)((w->rank + step - 1) / step * step / 4));
    a.by_slices = by(a.slices, tiles * a.slices), a.by_blocks = by(a.block_end[a.n_parts - 1], tiles * a.block_end[a.n_parts - 1]);
    hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
    (void)hipGetLastError();
    const bool xb = x_dtype == QLLM_BF16, wb = w->w_dtype == QLLM_BF16, yb = y_dtype == QLLM_BF16;
    if (wb) xb ? run_down<uint16_t, uint16_t>(a, (unsigned)tiles, stream) : run_down<float, uint16_t>(a, (unsigned)tiles, stream);
    else xb ? run_down<uint16_t, float>(a, (unsigned)tiles, stream) : run_down<float, float>(a, (unsigned)tiles, stream);
    if (const int32_t e = launched("adapters, first product: launch")) return e;
    if (a.slices > 1 && (a.slices > JOINED || rows > JOINED_ROWS || rows * w->rank > JOINED_RANKS)) {
        const int64_t words4 = rows * a.wide / 4;
        hipLaunchKernelGGL(join_kernel, dim3((unsigned)((words4 * JOINERS + 255) / 256)), dim3(256), 0, stream, a.h, words4, a.slices);
        if (const int32_t e = launched("adapters, sums: launch")) return e;
        a.slices = 1;
    }
    int32_t done;
    if (wb) done = yb ? run_up<uint16_t, uint16_t>(a, (unsigned)tiles, stream) : run_up<uint16_t, float>(a, (unsigned)tiles, stream);
    else done = yb ? run_up<float, uint16_t>(a, (unsigned)tiles, stream) : run_up<float, float>(a, (unsigned)tiles, stream);
    return done != QLLM_OK ? done : launched("adapters, second product: launch");
}
