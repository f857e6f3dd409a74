// Attention of several new tokens of each sequence over the paged cache: causal with a window and first tokens that stay
// visible, or the nodes of a drafted tree.
//
// O = sum_t p_t V_t / sum_t p_t, p_t = 2^(s_t - m), s_t = scale log2(e) q . K_t, over the tokens that a row sees, with the running
// maximum and sum of the softmax, so that keys and values are read once for all rows of a workgroup.  Rows are (token, head) pairs of the
// heads that share a key-value head, in this order: many rows make it a matrix product (4 d operations for a row and token, bound by the matrix
// pipes), few rows a stream through the cache (bound by memory).
//
// (Batches of at most one row for each sequence go to muxq_attend.hip, where that is faster: single() below.  Very unequal numbers of rows are
// divided badly: form_of goes by the bound, as if each sequence had max_new rows.  512 tokens of one sequence beside 63 single ones over 500 to 8000, 32
// heads of 128 over 8: 524 us, 23 and 210 in two calls.)
//
// Keys and values of a tile of tokens go through LDS as fp16, 8-bit codes converted on the way (exactly).  Both products are
// 32 x 32 x 16 steps with the tokens, or the dimensions, as rows of the left operand and 32 rows of the problem as the columns of the right one: scores
// come out with a row per lane column, which is where the weights of the second product have to stand, so that they never leave their
// lanes.  The second product's left operand is the transposed values, which LDS turns while it reads (16 lanes, 4 tokens of 16 dimensions).
// Rows in LDS are 16 bytes longer for keys and 32 for values, so that neither kind of read meets the same banks twice.  In the form for many rows of
// fp16 memory writes to LDS itself, two tiles in turn, and pieces of rows change places instead: no registers hold a tile (1.07 against
// 1.11 ms for the 16384 tokens below).
//
// Weights are 2^(s - m + 8), rounded to fp16, and m follows the maximum only when a score is 7 above it, which is rare: up to
// 2^15, so that small ones keep their bits.  The rounding is the one that a matrix instruction asks for; sums take the weights as they were rounded, so
// that it falls out of a sum of equal values.  The scale of a key goes to its score, the scale of a value to its weight; weights and
// their sum are over a running power of two that the scales which a row sees do not pass.
//
// What bounds it and what it reaches:
//   16384 tokens within a window of 4096, 32 heads of 128 over 8 of keys, fp16: 1.09 ms, 885 TFLOP/s of the 1190 that a large product reaches.
//     The matrix pipes are busy 46 % of the cycles that a CU works, at 1.7 GHz of the 2.4 nominal; LDS is active 48 % of them.
//   13 prompts, 8192 tokens together, behind up to 1500, a window of 1024, in codes: 0.22 ms, 520 TFLOP/s: conversion and scales are as many vector
//     instructions as the softmax is (14 for a product, 6 over fp16); the matrix pipes are busy 26 % of the cycles.
//   64 trees of 32 nodes over up to 8192 tokens: 0.26 ms, 4.4 TB/s: loads on their way, 32 KB a workgroup and two workgroups a CU.
//   1024 tokens, 12 heads of 64: 16.6 us with the join; 8 nodes behind 37
//     tokens, 12 heads: 9.3 us: chains of loads (lengths, pages, keys), one tile after the other, and what a launch costs.
// Taken back: eight waves of 32 rows (1.10 ms against 1.12 then, but 254 against 230 us in codes), loads between the products (their
// registers spilled), streaming loads (the trees 2 % faster, prompts 10 % slower).
#include "muxq_block_kernels.h"

#include <algorithm>
#include <type_traits>

namespace muxq {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef s16x4 __attribute__((address_space(3))) *LdsQuad;

constexpr int kChunk = 32;                    // tiles whose pages stand in LDS at a time
constexpr int kLoose = 32;                    // tiles with infinite or NaN values that are remembered one by one
constexpr float kFloor = -__builtin_inff();
constexpr float kMostScale = 3.0e38f / (65504.0f * 65504.0f * 256.0f);          // of scores, below which those of finite queries and keys are finite

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// Four codes of a word as fp16 values, exactly: code + 128 in the low byte of 0x64.. is 1024 + code + 128.
__device__ __forceinline__ void codes_to_half(uint32_t w, uint32_t &lo, uint32_t &hi)
{
    const uint32_t u = w ^ 0x80808080u;
    const uint32_t a = __builtin_amdgcn_perm(0x64646464u, u, 0x07010700u), b = __builtin_amdgcn_perm(0x64646464u, u, 0x07030702u);
    const f16x2 bias = {(_Float16)1152.0f, (_Float16)1152.0f};
    lo = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, a) - bias);
    hi = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, b) - bias);
}

// 2^(m - top) of a part with maximum m and sum l, never quite 0, so that an infinity among the values stays one; one without
// weights counts nothing, unless NaN stands there.  (Where it has tokens, all of them with a score of -infinity, its sum is kNone: beside a
// part with weights that is nothing, and where no part has any it says that the softmax is 0 / 0, not an empty row.)
constexpr float kNone = 0x1p-60f;
__device__ __forceinline__ float weight_of(float m, float l, float top) { return m == kFloor ? l : fmaxf(exp2_(m - top), 1.1754944e-38f); }

// What the sum of the values is multiplied by in the end.
__device__ __forceinline__ float factor_of(float m, float l) { return m != kFloor ? 1.0f / l : l == 0.0f ? 0.0f : __builtin_nanf(""); }

// 16 bytes of each lane to LDS, one lane behind the other from `to` on, which is the same for all of them.  (Written out, so that reads of
// the other tile do not wait for it; wait_for_memory() does.)
__device__ __forceinline__ void to_lds(const char *from, char *to)
{
    const uint32_t at = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)to);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(at), "v"(from) : "memory", "m0");
}
__device__ __forceinline__ void wait_for_memory() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// How the work is divided: a workgroup to a sequence, key-value head, tile of rows and piece of `tiles` tiles of tokens.  Rows that
// see no more tiles than that are finished by their first piece; the others leave parts in the workspace.
struct Plan {
    int row_tiles, pieces, tiles;         // (the last piece has what is left)
    float *o;           // [row tile of all][piece][rows of a tile][d], unnormalised
    float2 *ml;         // [row tile of all][piece][rows of a tile]: m and the sum
};

// A number that all lanes need: through the scalar cache.
__device__ __forceinline__ int one(const int32_t *p)
{
    return *(const __attribute__((address_space(4))) int32_t *)(uintptr_t)p;
}

// What one workgroup's rows are and see.
template <int kTT>
struct Span {
    int s, kvh, first, n, len, ctx;           // rows first..first + n of the call, tokens before the first
    int row0, n_rows;                         // of the sequence's rows (token, head), fewer than 2^31
    int i_lo, i_hi, local0, t1;               // its tokens, the first row's place in the first of them, and the first token that none of its rows sees
    int sink_tiles, window_from, count;       // tiles that they see: the first ones, then from window_from on

    __device__ __forceinline__ bool find(const RowsArgs &a, int x, int seq, int row_tiles, int rows)
    {
        s = seq;
        const int tile = x / a.c.n_kv_heads;
        kvh = x - tile * a.c.n_kv_heads;
        const int from = one(a.starts + s), to = one(a.starts + s + 1), length = one(a.lengths + s);
        first = max(0, min(from, a.M));
        n = max(0, min(to, a.M)) - first;
        if (n < 1 || n > a.max_new) return false;
        row0 = (row_tiles - 1 - tile) * rows;          // the last tokens see most: they come first
        n_rows = min(rows, n * a.group - row0);
        if (n_rows <= 0) return false;
        len = max(0, min(length, a.max_length));
        ctx = len - n;
        i_lo = (int)((uint32_t)row0 / (uint32_t)a.group);
        local0 = row0 - i_lo * a.group;
        i_hi = (int)((uint32_t)(row0 + n_rows - 1) / (uint32_t)a.group);
        t1 = a.parents ? len : max(0, min(len, ctx + i_hi + 1));
        sink_tiles = window_from = 0;
        count = (t1 + kTT - 1) / kTT;
        if (a.window) {
            const int from = max(0, (int)max(-1ll, (long long)ctx + i_lo - a.window) + 1) / kTT, sinks = (min(a.sinks, t1) + kTT - 1) / kTT;
            if (from > sinks) sink_tiles = sinks, window_from = from, count = max(0, count - from) + sinks;
        }
        return true;
    }
    __device__ __forceinline__ int tile_of(int j) const { return j < sink_tiles ? j : window_from + j - sink_tiles; }
};

// A row: its place in the sequence, its head, and what it sees.
struct Row {
    int i, head, p, sinks;
    uint32_t window;
    uint64_t above;           // of a tree's nodes
    int ctx;

    __device__ __forceinline__ void find(const RowsArgs &a, int kvh, int n, int ctx_, int i_lo, int local)
    {
        const int more = (int)((uint32_t)local / (uint32_t)a.group);
        i = min(n - 1, i_lo + more);
        head = kvh * a.group + local - more * a.group;
        ctx = ctx_;
        p = ctx + i;
        window = a.window ? a.window : 0x80000000u;
        sinks = min(a.sinks, p + 1);
    }
    // which of the tokens t0..t0 + 31 it sees, a bit to each
    __device__ __forceinline__ uint32_t sees32(bool tree, int t0, int t1) const
    {
        uint32_t word;
        if (tree) {
            const int x = t0 - ctx;                   // the node of the first one
            word = below(-x);
            if (x > -32 && x < 64) word |= (uint32_t)(x < 0 ? above << -x : above >> x);
        } else {
            word = (below(p + 1 - t0) & ~below((int)max((long long)p - window + 1 - t0, -1ll))) | below(sinks - t0);
        }
        return word & below(t1 - t0);
    }
    // the n lowest bits
    static __device__ __forceinline__ uint32_t below(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1; }
    __device__ __forceinline__ bool sees(bool tree, int t) const
    {
        if (!tree) return (uint32_t)(p - t) < window || t < sinks;
        const int x = t - ctx;
        return t < ctx || ((uint32_t)x < 64u && (above >> x & 1));
    }
};

// The nodes above node i and itself.
__device__ __forceinline__ uint64_t nodes_above(const int32_t *parents, int i)
{
    uint64_t above = 0;
    for (;;) {
        above |= 1ull << i;
        const int up = parents[i];
        if (up < 0 || up >= i) return above;
        i = up;
    }
}

// Infinite and NaN values that the rows of a workgroup see, with weights of 1, or of 0 where the row's score is -infinity: all that counts for
// a sum in which there is one.  The tiles' values went into the products without them; here they decide what they stand for.  A row whose
// sum of weights is NaN, in any of the kWT waves that have it, stays NaN.
// (Finite queries and keys have finite scores, which need not be looked at.  One dimension infinite in all of 4096 tokens, 32 heads of 128: 30 ms,
// where a score for each row, dimension and token took 603.)
template <bool kInt8, int kTT, int kWR, int kWT>
__device__ void put_loose(const RowsArgs &a, const Span<kTT> &w, int j0, int j1, const int *tiles, int n_tiles,
                                                    const int32_t *parents, const float (*totals)[32], _Float16 *o, float *part)
{
    typedef typename std::conditional<kInt8, int8_t, _Float16>::type Value;
    typedef Value Four __attribute__((ext_vector_type(4)));
    typedef Value Eight __attribute__((ext_vector_type(8)));
    const int d = a.c.head_dim, quads = d / 4, shift = a.c.block_shift, mask = (1 << shift) - 1;
    const int local0 = w.local0, n_rows = w.n_rows, n = n_tiles > kLoose ? j1 - j0 : n_tiles;
    auto tile = [&](int x) { return w.tile_of(n_tiles > kLoose ? j0 + x : tiles[x]) * kTT; };
    bool open = !(fabsf(a.scale) < kMostScale);                  // whether there are keys with scores that may be infinite
    for (int x = threadIdx.x; x < n * kTT; x += blockDim.x) {
        const int t = tile(x / kTT) + x % kTT;
        const int page = t < w.t1 ? a.table[(long long)w.s * a.ld_table + (t >> shift)] : -1;
        if (page < 0 || page >= a.c.n_blocks) continue;
        if (kInt8) {
            open |= !(fabsf(a.scale) * fabsf(a.c.k_scale[(((long long)page * a.c.n_kv_heads + w.kvh) << shift) + (t & mask)]) < kMostScale);
        } else {
            const char *const key = a.c.k + (page * a.c.ld_block + w.kvh * a.c.ld_head + (t & mask) * a.c.ld_token) * 2;
            for (int y = 0; y < d; y += 8) {
                const u32x4 k = *(const u32x4 *)(key + y * 2);
                for (int z = 0; z < 4; ++z) open |= (k[z] & 0x7c00u) == 0x7c00u || (k[z] & 0x7c000000u) == 0x7c000000u;
            }
        }
    }
    open = __syncthreads_or(open);
    for (int item = threadIdx.x; item < n_rows * quads; item += blockDim.x) {
        const int quad = item / n_rows, r = item - quad * n_rows, e = quad * 4;
        float all = 0.0f;
        for (int x = 0; x < kWT; ++x) all += totals[x * kWR + (r >> 5)][r & 31];
        if (all != all) continue;
        Row row;
        row.find(a, w.kvh, w.n, w.ctx, w.i_lo, local0 + r);
        row.above = a.parents ? nodes_above(parents, row.i) : 0;
        const _Float16 *const q = a.q + (long long)(w.first + row.i) * a.ldq + (long long)row.head * d;
        f32x4 sum = {};
        bool look = open, asked = open;
        for (int x = 0; x < n; ++x) {
            const int t0 = tile(x);
            for (int t = t0; t < min(t0 + kTT, w.t1); ++t) {
                if (!row.sees(a.parents != nullptr, t)) continue;
                const int page = a.table[(long long)w.s * a.ld_table + (t >> shift)];
                if (page < 0 || page >= a.c.n_blocks) continue;
                const long long at = page * a.c.ld_block + w.kvh * a.c.ld_head + (t & mask) * a.c.ld_token;
                const long long at_s = (((long long)page * a.c.n_kv_heads + w.kvh) << shift) + (t & mask);
                f32x4 v = __builtin_convertvector(*(const Four *)((const Value *)a.c.v + at + e), f32x4);
                if (kInt8) v *= a.c.v_scale[at_s];
                const f32x4 zero = v - v;
                if (zero[0] == 0.0f && zero[1] == 0.0f && zero[2] == 0.0f && zero[3] == 0.0f) continue;
                float score = 0.0f;
                for (int y = 0; y < d && !asked; y += 8) {
                    const f16x8 x8 = *(const f16x8 *)(q + y), none = x8 - x8;
#pragma unroll
                    for (int z = 0; z < 8; ++z) look |= none[z] != (_Float16)0.0f;
                }
                asked = true;
                if (look) {
                    for (int y = 0; y < d; y += 8) {
                        const f16x8 x8 = *(const f16x8 *)(q + y);
                        const Eight k8 = *(const Eight *)((const Value *)a.c.k + at + y);
#pragma unroll
                        for (int z = 0; z < 8; ++z) score += (float)x8[z] * (float)k8[z];
                    }
                    score *= a.scale;
                    if (kInt8) score *= a.c.k_scale[at_s];
                }
                for (int y = 0; y < 4; ++y)
                    if (zero[y] != 0.0f) sum[y] += score == kFloor ? 0.0f * v[y] : v[y];
                if (sum[0] != sum[0] && sum[1] != sum[1] && sum[2] != sum[2] && sum[3] != sum[3]) x = n, t = w.t1;      // NaN stays
            }
        }
        for (int y = 0; y < 4; ++y)
            if (sum[y] - sum[y] != 0.0f) {
                if (part)
                    part[(long long)r * d + e + y] = sum[y];
                else
                    o[(long long)(w.first + row.i) * a.ldo + (long long)row.head * d + e + y] = (_Float16)sum[y];
            }
    }
}

// kD: the head's dimensions, padded; kWaves, kWR of them along the rows, 32 each, the others divide a tile's tokens; kTT: tokens of a tile.
template <int kD, bool kInt8, int kWaves, int kWR, int kTT>
__global__ __launch_bounds__(64 * kWaves, kD == 64 ? 3 : kD == 128 ? 2 : 1) void k_rows(RowsArgs a, Plan plan)
{
    constexpr int kThreads = 64 * kWaves, kWT = kWaves / kWR, kR = 32 * kWR, kNB = kTT / kWT / 32;          // waves along tokens; rows; blocks of 32 tokens of a wave
    // fp16 of many rows: memory writes to LDS by itself, into one of two tiles; its rows are not longer then, but their 16-byte pieces
    // change places by the row's number, for the same end.
    constexpr bool kDirect = !kInt8 && kWR == 4;
    constexpr int kKeyRow = kDirect ? 2 * kD : 2 * kD + 16, kValueRow = kDirect ? 2 * kD : 2 * kD + 32;                   // bytes of a row in LDS
    constexpr int kTile = kTT * (kKeyRow + kValueRow);
    constexpr int kCH = kInt8 ? kD / 16 : kD / 8, kTPP = kThreads / kCH, kP = kTT / kTPP;      // loads of a row, rows of a pass, passes
    constexpr bool kAllJoin = kWR == 1 && kD * 128 * kWaves <= kTT * (kKeyRow + kValueRow);       // all waves' parts fit the tile's LDS
    static_assert(kNB >= 1 && kP >= 1, "tile");
    __shared__ __align__(1024) char sh_k[kTile * (kDirect ? 2 : 1)];
    char *const sh_v = sh_k + kTT * kKeyRow;
    f32x4 *const sh_o = (f32x4 *)sh_k;
    __shared__ long long sh_at[kChunk * (kTT / 8)];           // where runs of rows stand, in bytes; 0 for those that are nowhere
    __shared__ int sh_page[kChunk * (kTT / 8)];               // their pages; -1: not in the cache, or behind all tokens
    __shared__ __align__(16) float sh_ks[kInt8 ? kTT : 4], sh_vs[kInt8 ? kTT : 4];
    __shared__ float sh_m[kWaves][32], sh_l[kWaves][32];
    __shared__ long long sh_row[32];
    __shared__ int sh_bad, sh_found, sh_n_loose, sh_loose[kLoose], sh_parents[kMaxNodes];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wr = wave % kWR, wt = wave / kWR, col = lane & 31, half = lane >> 5;
    const int d = a.c.head_dim, shift = a.c.block_shift, mask = (1 << shift) - 1;
    const bool tree = a.parents != nullptr;

    if (tid == 0) sh_found = sh_n_loose = sh_bad = 0;
    __syncthreads();
    Span<kTT> w;
    if (!w.find(a, blockIdx.x, blockIdx.y, plan.row_tiles, kR)) return;
    const int piece = blockIdx.z;
    const bool whole = w.count <= plan.tiles || plan.pieces == 1;
    const int j0 = whole ? 0 : piece * plan.tiles, j1 = whole || piece == plan.pieces - 1 ? w.count : min(w.count, j0 + plan.tiles);
    if (piece > 0 && (whole || j0 >= j1)) return;

    // the pages of tiles j0..j9, and whether one is missing (0 before)
    const int run_shift = min(shift, __builtin_ctz(kTPP)), e_shift = __builtin_ctz(kTT) - run_shift;      // runs of a tile: 1 << e_shift
    auto find_pages = [&](int j0, int j9) {
        for (int x = tid; x < (j9 - j0) << e_shift; x += kThreads) {
            const int t = w.tile_of(j0 + (x >> e_shift)) * kTT + ((x & ((1 << e_shift) - 1)) << run_shift);
            int page = -1;
            if (t < w.t1) {
                page = a.table[(long long)w.s * a.ld_table + (t >> shift)];
                if (page < 0 || page >= a.c.n_blocks) page = -1, sh_bad = 1;
            }
            sh_at[x] = page < 0 ? 0 : (page * a.c.ld_block + w.kvh * a.c.ld_head + (t & mask) * a.c.ld_token) * (kInt8 ? 1 : 2);
            sh_page[x] = page;
        }
    };

    if (kDirect && d != kD)              // dimensions that nothing is written to
        for (int x = tid; x < (int)sizeof(sh_k) / 16; x += kThreads) ((u32x4 *)sh_k)[x] = u32x4{};
    const int local0 = w.local0, n_rows = w.n_rows;
    Row row;
    row.find(a, w.kvh, w.n, w.ctx, w.i_lo, local0 + min(wr * 32 + col, n_rows - 1));
    // what the wave's rows see, from the first to the last of them
    const int p_lo = __builtin_amdgcn_readfirstlane(row.p), p_hi = __builtin_amdgcn_readlane(row.p, 31);
    const _Float16 *const q_row = a.q + (long long)(w.first + row.i) * a.ldq + (long long)row.head * d;

    // queries: the right operand of the first product; a negative scale turns their signs, one of 0 makes them 0
    f16x8 q[kD / 16];
#pragma unroll
    for (int x = 0; x < kD / 16; ++x) {
        const int e = 16 * x + 8 * half;
        q[x] = f16x8{};
        if (e < d) q[x] = *(const f16x8 *)(q_row + e);
    }
    // (all of the first loads on their way together)
    int parent = 0;
    if (tree && tid < w.n) parent = a.parents[w.first + tid];
    find_pages(j0, min(j1, j0 + kChunk));
    if (tree && tid < w.n) sh_parents[tid] = parent;
    if (a.scale <= 0.0f)
#pragma unroll
        for (int x = 0; x < kD / 16; ++x) q[x] = a.scale < 0.0f ? -q[x] : q[x] * (_Float16)0.0f;
    const float c = a.scale == 0.0f ? 1.0f : fminf(fabsf(a.scale) * 1.44269504088896f, 3.0e38f);

    float m, total;
    int cap;                         // of codes: weights and their sum are over 2^cap, which scales of values do not pass
    f32x4 l;                         // the weights' sum, in four parts
    f32x16 o[kD / 32];
    bool careful = false;

    // what a thread loads of a tile: of rows kTPP apart the same 16 bytes, of keys and of values
    const int lane_row = tid / kCH, piece_of = tid % kCH;
    const bool live = piece_of * (kInt8 ? 16 : 8) < d;
    // (rows of a run stand in one page and belong to one pass)
    // (in LDS the lane's piece is of other dimensions, by the row, where pieces change places)
    const int piece_k = kDirect ? piece_of ^ (lane_row & 7) : piece_of, piece_v = kDirect ? piece_of ^ ((lane_row & 3) << 1) : piece_of;
    const bool live_k = piece_k * 8 < d, live_v = piece_v * 8 < d;
    const long long lane_row_at = (long long)(lane_row & ((1 << run_shift) - 1)) * a.c.ld_token * 2;
    const long long lane_at_k = lane_row_at + piece_k * 16, lane_at_v = lane_row_at + piece_v * 16;
    const long long lane_at = ((long long)(lane_row & ((1 << run_shift) - 1)) * a.c.ld_token + (live ? piece_of : 0) * (kInt8 ? 16 : 8)) * (kInt8 ? 1 : 2);
    u32x4 k[kDirect ? 1 : kP], v[kDirect ? 1 : kP];
    float scale_k = 0.0f, scale_v = 0.0f;
    bool bad = false, edge = false;
    int jc = j0, t_next = 0, slot_next = 0;

    // Every lane loads, from the first page where its row is nowhere: such rows become zeros in store().
    auto load = [&](int j) {
        t_next = w.tile_of(j) * kTT, slot_next = (j - jc) << e_shift;
        edge = bad || t_next + kTT > w.t1;
#pragma unroll
        for (int x = 0; x < kP; ++x) {
            const long long at = sh_at[slot_next + ((x * kTPP + lane_row) >> run_shift)] + (kDirect ? 0 : lane_at);
            if constexpr (kDirect) {
                if (live_k) to_lds(a.c.k + (at + lane_at_k), sh_k + (j & 1) * kTile + (x * kWaves + wave) * 1024);
                if (live_v) to_lds(a.c.v + (at + lane_at_v), sh_v + (j & 1) * kTile + (x * kWaves + wave) * 1024);
            } else {
                k[x] = *(const u32x4 *)(a.c.k + at);
                v[x] = *(const u32x4 *)(a.c.v + at);
            }
        }
        if (kInt8 && tid < kTT) {
            const int page = max(0, sh_page[slot_next + (tid >> run_shift)]);
            const long long at = (((long long)page * a.c.n_kv_heads + w.kvh) << shift) + ((t_next + tid) & mask);
            scale_k = a.c.k_scale[at];
            scale_v = a.c.v_scale[at];
        }
    };
    // Of a tile that memory wrote to LDS: values of rows that are nowhere become 0, where care is taken infinite and NaN ones too.
    auto mend = [&](int j) {
        bool found = false;
        const int t0 = w.tile_of(j) * kTT, slot = (j - jc) << e_shift;
#pragma unroll
        for (int x = 0; x < kP; ++x) {
            const int in = x * kTPP + lane_row;
            u32x4 *const at = (u32x4 *)(sh_v + (j & 1) * kTile) + x * kThreads + tid;
            u32x4 y = *at;
            if (t0 + in >= w.t1 || sh_page[slot + (in >> run_shift)] < 0) {
                y = u32x4{};
            } else if (careful) {
#pragma unroll
                for (int z = 0; z < 4; ++z) {
                    const uint32_t was = y[z];
                    if ((was & 0x7c00u) == 0x7c00u) y[z] &= 0xffff0000u;
                    if ((was & 0x7c000000u) == 0x7c000000u) y[z] &= 0xffffu;
                    found |= y[z] != was;
                }
            }
            *at = y;
        }
        if (careful && __any(found)) sh_found = 1;
    };
    // the tile that is on its way to LDS; where care is taken without its infinite and NaN values
    auto store = [&]() {
        bool found = false;
        if (edge || d != kD) {
#pragma unroll
            for (int x = 0; x < kP; ++x) {
                const int in = x * kTPP + lane_row;
                if (!live || t_next + in >= w.t1 || sh_page[slot_next + (in >> run_shift)] < 0) k[x] = v[x] = u32x4{};
            }
            if (kInt8 && tid < kTT && (t_next + tid >= w.t1 || sh_page[slot_next + (tid >> run_shift)] < 0)) scale_k = scale_v = 0.0f;
        }
        if (!kInt8 && careful) {
#pragma unroll
            for (int x = 0; x < kP; ++x)
#pragma unroll
                for (int z = 0; z < 4; ++z) {
                    const uint32_t was = v[x][z];
                    if ((was & 0x7c00u) == 0x7c00u) v[x][z] &= 0xffff0000u;
                    if ((was & 0x7c000000u) == 0x7c000000u) v[x][z] &= 0xffffu;
                    found |= v[x][z] != was;
                }
        }
#pragma unroll
        for (int x = 0; x < kP; ++x) {
            u32x4 *const to_k = (u32x4 *)(sh_k + (x * kTPP + lane_row) * kKeyRow + piece_of * (kInt8 ? 32 : 16));
            u32x4 *const to_v = (u32x4 *)(sh_v + (x * kTPP + lane_row) * kValueRow + piece_of * (kInt8 ? 32 : 16));
            if constexpr (kInt8) {
                uint32_t y[8];
#pragma unroll
                for (int z = 0; z < 4; ++z) codes_to_half(k[x][z], y[2 * z], y[2 * z + 1]);
                to_k[0] = u32x4{y[0], y[1], y[2], y[3]}, to_k[1] = u32x4{y[4], y[5], y[6], y[7]};
#pragma unroll
                for (int z = 0; z < 4; ++z) codes_to_half(v[x][z], y[2 * z], y[2 * z + 1]);
                to_v[0] = u32x4{y[0], y[1], y[2], y[3]}, to_v[1] = u32x4{y[4], y[5], y[6], y[7]};
            } else {
                *to_k = k[x];
                *to_v = v[x];
            }
        }
        if (kInt8 && tid < kTT) {
            if (careful && !(scale_v - scale_v == 0.0f)) found = true, scale_v = 0.0f;
            sh_ks[tid] = scale_k * c;
            sh_vs[tid] = scale_v;
        }
        if (careful && __any(found)) sh_found = 1;
    };

    int turn_k[4], turn_v[2];           // where a lane's pieces of a row begin
    if constexpr (kDirect) {
#pragma unroll
        for (int x = 0; x < 4; ++x) turn_k[x] = ((2 * x + half) ^ (col & 7)) * 16;
#pragma unroll
        for (int x = 0; x < 2; ++x) turn_v[x] = ((4 * x + ((lane & 16) >> 3) + ((lane & 3) >> 1)) ^ ((lane >> 2 & 3) << 1)) * 16 + (lane & 1) * 8;
    }

    auto compute = [&](int j) {
        const int t0 = w.tile_of(j) * kTT + wt * (32 * kNB), slot = (j - jc) << e_shift;
        // nothing, or all of it, to be seen by the wave's rows
        const int t9 = t0 + 32 * kNB - 1;
        if (t0 >= w.t1 || wr * 32 >= n_rows) return;
        bool all = t9 < w.t1 && !bad;
        if (tree) {
            all = all && t9 < w.ctx;
        } else {
            if (t0 > p_hi || (a.window && (long long)t9 <= (long long)p_lo - a.window && t0 >= a.sinks)) return;
            all = all && t9 <= p_lo && (!a.window || (long long)t0 > (long long)p_hi - a.window || t9 < a.sinks);
        }
        f32x16 acc[kNB] = {};
        const int tile_at = kDirect ? (j & 1) * kTile : 0;
        const char *const keys = sh_k + tile_at + (wt * kNB * 32 + col) * kKeyRow + (kDirect ? 0 : half * 16);
        const char *const values = sh_v + tile_at + (wt * kNB * 32 + 4 * half + ((lane & 15) >> 2)) * kValueRow + (kDirect ? 0 : ((lane & 16) + 4 * (lane & 3)) * 2);
        // A block is 32 tokens: kQ products with its keys, kQ with its values, and 16 weights of a lane between them.  While a block is
        // weighed, the products with the keys of the next one and with the values of the last one go on; reads of LDS are kAhead products in
        // front of theirs.  (In the compiler's own order each product waits for its read, and the weights for all of them.)
        constexpr int kQ = kD / 16, kAhead = 4;
        typedef short s16x8 __attribute__((ext_vector_type(8)));
        f16x8 key[kAhead];
        s16x8 value[kAhead];
        uint32_t weights[2][8];
        f32x4 vs[4];
        auto ask_key = [&](int b, int x) {
            key[x % kAhead] = *(const f16x8 *)(keys + b * 32 * kKeyRow + (kDirect ? turn_k[x & 3] + (x >> 2) * 128 : x * 32));
        };
        auto ask_value = [&](int b, int x) {
            // rows 4 half + 0..3 of 16 tokens, and 8 rows on, 32 dimensions
            const int y = x % (kD / 32);
            const char *const at = values + (b * 32 + x / (kD / 32) * 16) * kValueRow + (kDirect ? turn_v[y & 1] + (y >> 1) * 128 : y * 64);
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsQuad)at), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsQuad)(at + 8 * kValueRow));
            value[x % kAhead] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        };
        auto score = [&](int b, int x) {
            acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(key[x % kAhead], q[x], acc[b], 0, 0, 0);
            if (x + kAhead < kQ) ask_key(b, x + kAhead);
        };
        auto add = [&](int b, int x) {
            const uint32_t *const p = weights[b & 1] + x / (kD / 32) * 4;
            o[x % (kD / 32)] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, value[x % kAhead]), __builtin_bit_cast(f16x8, u32x4{p[0], p[1], p[2], p[3]}),
                                                                     o[x % (kD / 32)], 0, 0, 0);
            if (x + kAhead < kQ) ask_value(b, x + kAhead);
        };
        float off = 0.0f;
        auto weigh = [&](int b, int x) {              // two of them
            float p[2];
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const int at = 2 * x + y;
                p[y] = exp2_(kInt8 ? acc[b][at] + off : __builtin_fmaf(acc[b][at], c, off));
                if constexpr (kInt8) {
                    l[at & 3] += p[y];
                    p[y] *= vs[at >> 2][at & 3];
                }
            }
            const f16x2 y = __builtin_convertvector(f32x2{p[0], p[1]}, f16x2);
            weights[b & 1][x] = __builtin_bit_cast(uint32_t, y);
            asm volatile("" : "+v"(weights[b & 1][x]));              // (here, not where the weight is needed)
            // their sum as they were rounded
            if constexpr (!kInt8) l[x & 3] = __builtin_amdgcn_fdot2(y, f16x2{(_Float16)1.0f, (_Float16)1.0f}, l[x & 3], false);
        };
        // everything so far times a power of two
        auto scale_all = [&](int b, float keep) {
            l *= keep;
#pragma unroll
            for (int x = 0; x < kD / 32; ++x) o[x] *= keep;
            if (b > 0)
#pragma unroll
                for (int x = 0; x < 8; ++x)
                    weights[(b - 1) & 1][x] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, weights[(b - 1) & 1][x]) * f16x2{(_Float16)keep, (_Float16)keep});
        };
#pragma unroll
        for (int x = 0; x < kAhead; ++x) ask_key(0, x);
#pragma unroll
        for (int x = 0; x < kQ; ++x) {
            score(0, x);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int b = 0; b < kNB; ++b) {
            const bool last = b == kNB - 1;
            if (!last)
#pragma unroll
                for (int x = 0; x < kAhead; ++x) ask_key(b + 1, x);
            if (b > 0 || last)
#pragma unroll
                for (int x = 0; x < kAhead; ++x) ask_value(b > 0 ? b - 1 : b, x);
            if constexpr (kInt8) {
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const f32x4 y = *(const f32x4 *)(sh_ks + (wt * kNB + b) * 32 + 8 * x + 4 * half);
#pragma unroll
                    for (int z = 0; z < 4; ++z) acc[b][4 * x + z] *= y[z];
                }
            }
            if (!all) {
                uint32_t word = row.sees32(tree, t0 + 32 * b, w.t1);
                if (bad)                              // pages are 8 tokens at least
#pragma unroll
                    for (int x = 0; x < 4; ++x)
                        if (sh_page[slot + ((wt * 32 * kNB + 32 * b + 8 * x) >> run_shift)] < 0) word &= ~(255u << 8 * x);
                word >>= 4 * half;
#pragma unroll
                for (int x = 0; x < 16; ++x)
                    if (!(word >> (8 * (x >> 2) + (x & 3)) & 1)) acc[b][x] = kFloor;
            }
            float top = kFloor;
#pragma unroll
            for (int x = 0; x < 16; ++x) top = fmaxf(top, acc[b][x]);
            if (!kInt8) top *= c;
            if (__any(top > m + 7.0f)) {                    // rare after the first tiles: a new maximum for the row, a whole number
                top = fmaxf(top, __shfl_xor(top, 32, 64));
                const float to = fmaxf(m, __builtin_ceilf(top)), keep = weight_of(m, l[0] + l[1] + (l[2] + l[3]), to);
                m = to;
                scale_all(b, keep);
            }
            if constexpr (kInt8) {
                float most = 0.0f;
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    vs[x] = *(const f32x4 *)(sh_vs + (wt * kNB + b) * 32 + 8 * x + 4 * half);
#pragma unroll
                    for (int z = 0; z < 4; ++z) most = fmaxf(most, fabsf(vs[x][z]));
                }
                if (__any(most > __uint_as_float((uint32_t)(cap + 127) << 23))) {          // rare: scales of values beyond 2^cap
                    if (!all) {                       // (one that the row does not see is nothing to it)
                        uint32_t word = row.sees32(tree, t0 + 32 * b, w.t1) >> 4 * half;
                        asm volatile("" : "+v"(word));
                        most = 0.0f;
#pragma unroll
                        for (int x = 0; x < 16; ++x) most = fmaxf(most, word >> (8 * (x >> 2) + (x & 3)) & 1 ? fabsf(vs[x >> 2][x & 3]) : 0.0f);
                    }
                    most = fmaxf(most, __shfl_xor(most, 32, 64));
                    const int to = max(cap, (int)(min(__float_as_uint(most) >> 23, 252u) + 1) - 127);
                    scale_all(b, exp2_((float)(cap - to)));
                    cap = to;
                }
            }
            off = m == kFloor ? 0.0f : 8.0f - m - (kInt8 ? (float)cap : 0.0f);
            // two weights after each product; the last block's second half beside the products with its first half
            if (!last) {
                const int n = b > 0 ? 2 * kQ : kQ;
#pragma unroll
                for (int x = 0; x < n; ++x) {
                    if (x < kQ) score(b + 1, x);
                    else add(b - 1, x - kQ);
#pragma unroll
                    for (int y = x * 8 / n; y < (x + 1) * 8 / n; ++y) weigh(b, y);
                    __builtin_amdgcn_sched_barrier(0);
                }
            } else {
                if (b > 0) {
#pragma unroll
                    for (int x = 0; x < kQ; ++x) {
                        add(b - 1, x);
#pragma unroll
                        for (int y = x * 8 / kQ; y < (x + 1) * 8 / kQ; ++y) weigh(b, y);
                        __builtin_amdgcn_sched_barrier(0);
                    }
#pragma unroll
                    for (int x = 0; x < kAhead; ++x) ask_value(b, x);
                } else {
#pragma unroll
                    for (int y = 0; y < 4; ++y) weigh(b, y);
                }
#pragma unroll
                for (int x = 0; x < kQ; ++x) {
                    add(b, x);
                    if (b == 0 && x < kQ / 2)
#pragma unroll
                        for (int y = 4 + x * 4 / (kQ / 2); y < 4 + (x + 1) * 4 / (kQ / 2); ++y) weigh(b, y);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
    };

    // An infinite or NaN value makes all rows of a tile NaN, also those that do not see it (0 times infinity): where a sum is, the
    // workgroup begins again, takes such values out and remembers where they are.
    for (;;) {
        m = kFloor, cap = -80;
        l = f32x4{};
#pragma unroll
        for (int x = 0; x < kD / 32; ++x) o[x] = f32x16{};
        for (jc = j0; jc < j1; jc += kChunk) {
            const int j9 = min(j1, jc + kChunk);
            if (jc > j0 || careful) {
                __syncthreads();                              // readers of the pages before
                if (tid == 0) sh_bad = 0;
                __syncthreads();
                find_pages(jc, j9);
            }
            __syncthreads();
            bad = __builtin_amdgcn_readfirstlane(sh_bad) != 0;
            load(jc);
            if (jc == j0) row.above = tree ? nodes_above(sh_parents, row.i) : 0;
            for (int j = jc; j < j9; ++j) {
                if constexpr (kDirect) {
                    wait_for_memory();
                    __syncthreads();                          // the tile is there, and the readers of the one before are through
                    if (edge || careful) {
                        mend(j);
                        __syncthreads();
                    }
                } else {
                    if (j > j0) __syncthreads();              // readers of the tile before
                    store();
                    __syncthreads();
                }
                if (careful && tid == 0 && sh_found) {
                    if (sh_n_loose < kLoose) sh_loose[sh_n_loose] = j;
                    ++sh_n_loose;
                    sh_found = 0;
                }
                if (j + 1 < j9) load(j + 1);
                compute(j);
            }
        }
        // the sum of a row's weights, of the wave's tokens
        total = (l[0] + l[1]) + (l[2] + l[3]);
        total += __shfl_xor(total, 32, 64);
        if constexpr (kInt8) {
            const float up = __uint_as_float((uint32_t)(cap + 127) << 23);
            total *= up;
#pragma unroll
            for (int x = 0; x < kD / 32; ++x) o[x] *= up;
        }
        if (total == 0.0f && row.p >= 0) {                    // no weights: are there tokens?
            bool seen = false;
            for (int j = j0; j < j1 && !seen; ++j) {
                const int t0 = w.tile_of(j) * kTT + wt * (32 * kNB);
                for (int t = t0; t < min(t0 + 32 * kNB, w.t1) && !seen; ++t)
                    if (row.sees(tree, t)) {
                        const int page = a.table[(long long)w.s * a.ld_table + (t >> shift)];
                        seen = page >= 0 && page < a.c.n_blocks;
                    }
            }
            if (seen) total = kNone;
        }
        float sum = 0.0f;
#pragma unroll
        for (int x = 0; x < kD / 32; ++x)
#pragma unroll
            for (int y = 0; y < 16; ++y) sum += fabsf(o[x][y]);
        if constexpr (kWT > 1) {
            // Waves with the same rows leave their parts in LDS, lane by lane, where all threads join them; or the first takes what the others
            // leave there, where it does not hold all.
            __syncthreads();                                  // readers of the last tile
            static_assert(kD / 8 * 64 * 16 * (kWaves - kWR) <= sizeof(sh_k), "the parts fit the tile");
            if (half == 0) sh_m[wave][col] = m, sh_l[wave][col] = total;
            if (half == 0 && wave == 0) sh_row[col] = (long long)(w.first + row.i) * a.ldo + (long long)row.head * d;
            if (kAllJoin || wt > 0)
#pragma unroll
                for (int x = 0; x < kD / 8; ++x)
                    sh_o[((wave - (kAllJoin ? 0 : kWR)) * (kD / 8) + x) * 64 + lane] = f32x4{o[x >> 2][4 * (x & 3)], o[x >> 2][4 * (x & 3) + 1], o[x >> 2][4 * (x & 3) + 2], o[x >> 2][4 * (x & 3) + 3]};
        }
        if (careful && kWT == 1) {
            if (half == 0) sh_l[wave][col] = total;
            break;
        }
        if (!careful && __any(!(sum <= 3.4e38f))) sh_found = 1;
        __syncthreads();
        if (careful || __builtin_amdgcn_readfirstlane(sh_found) == 0) break;
        careful = true;
        __syncthreads();
        if (tid == 0) sh_found = 0;
    }

    const long long part = ((((long long)w.s * a.c.n_kv_heads + w.kvh) * plan.row_tiles + blockIdx.x / a.c.n_kv_heads) * plan.pieces + piece) * kR;
    float *const part_o = whole ? nullptr : plan.o + part * d;
    float top = m;
    if constexpr (kAllJoin) {
        // (not unrolled: a short call is bound by the fetching of instructions)
#pragma unroll 1
        for (int item = tid; item < kD / 8 * 64; item += kThreads) {
            const int x = item >> 6, r = item & 31, e = 32 * (x >> 2) + 8 * (x & 3) + 4 * (item >> 5 & 1);
            if (r >= n_rows || e >= d) continue;
            float top = sh_m[0][r], total = 0.0f;
#pragma unroll
            for (int y = 1; y < kWaves; ++y) top = fmaxf(top, sh_m[y][r]);
            f32x4 sum = {};
#pragma unroll
            for (int y = 0; y < kWaves; ++y) {
                const float z = sh_l[y][r], f = weight_of(sh_m[y][r], z, top);
                total += f * z;
                sum += f * sh_o[y * (kD * 8) + item];
            }
            if (whole)
                *(f16x4 *)(a.o + sh_row[r] + e) = __builtin_convertvector(sum * factor_of(top, total), f16x4);
            else
                *(f32x4 *)(part_o + (long long)r * d + e) = sum;
            if (!whole && e == 0) plan.ml[part + r] = make_float2(top, top == kFloor && total > 0.0f ? kNone : total);
        }
    } else if constexpr (kWT > 1) {
        if (wt == 0) {
#pragma unroll
            for (int x = 1; x < kWT; ++x) top = fmaxf(top, sh_m[x * kWR + wr][col]);
            const float f = weight_of(m, total, top);
            total *= f;
#pragma unroll
            for (int x = 0; x < kD / 32; ++x) o[x] *= f;
#pragma unroll
            for (int x = 1; x < kWT; ++x) {
                const float z = sh_l[x * kWR + wr][col], f = weight_of(sh_m[x * kWR + wr][col], z, top);
                total += f * z;
#pragma unroll
                for (int y = 0; y < kD / 8; ++y) {
                    const f32x4 v = f * sh_o[(((x - 1) * kWR + wr) * (kD / 8) + y) * 64 + lane];
#pragma unroll
                    for (int z = 0; z < 4; ++z) o[y >> 2][4 * (y & 3) + z] += v[z];
                }
            }
        }
    }
    if (!kAllJoin && wt == 0 && wr * 32 + col < n_rows) {
        const int r = wr * 32 + col;
        const float inv = factor_of(top, total);
        _Float16 *const o_row = a.o + (long long)(w.first + row.i) * a.ldo + (long long)row.head * d;
#pragma unroll
        for (int x = 0; x < kD / 32; ++x)
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                const int e = 32 * x + 8 * y + 4 * half;
                const f32x4 z = {o[x][4 * y], o[x][4 * y + 1], o[x][4 * y + 2], o[x][4 * y + 3]};
                if (e >= d) continue;
                if (whole)
                    *(f16x4 *)(o_row + e) = __builtin_convertvector(z * inv, f16x4);
                else
                    *(f32x4 *)(part_o + (long long)r * d + e) = z;
            }
        if (!whole && half == 0) plan.ml[part + r] = make_float2(top, top == kFloor && total > 0.0f ? kNone : total);
    }
    if (!careful) return;
    __syncthreads();
    if (sh_n_loose > 0) {
        __threadfence_block();
        put_loose<kInt8, kTT, kWR, kWT>(a, w, j0, j1, sh_loose, sh_n_loose, sh_parents, sh_l, a.o, part_o);
    }
}

// The parts of rows that several workgroups have, joined by weights 2^(m - max m): a workgroup to a tile of rows, a thread four
// dimensions of a row.
constexpr int kJoinThreads = 256;

template <int kTT>
__global__ __launch_bounds__(kJoinThreads) void k_rows_join(RowsArgs a, Plan plan, int rows)
{
    Span<kTT> w;
    if (!w.find(a, blockIdx.x, blockIdx.y, plan.row_tiles, rows) || w.count <= plan.tiles) return;
    const int d = a.c.head_dim, quads = d / 4, pieces = min(plan.pieces, (w.count + plan.tiles - 1) / plan.tiles);
    const int local0 = w.local0, n_rows = w.n_rows;
    const long long part = (((long long)w.s * a.c.n_kv_heads + w.kvh) * plan.row_tiles + blockIdx.x / a.c.n_kv_heads) * plan.pieces * rows;
    for (int item = threadIdx.x + kJoinThreads * blockIdx.z; item < n_rows * quads; item += kJoinThreads * gridDim.z) {
        const int r = item / quads, e = (item - r * quads) * 4;
        // eight parts on their way at a time, the last one again where there are fewer (a maximum more does not change, a weight counts as 0)
        float top = kFloor, total = 0.0f;
        f32x4 sum = {};
        for (int x0 = 0; x0 < pieces; x0 += 8) {
            float2 ml[8];
            f32x4 v[8];
#pragma unroll
            for (int x = 0; x < 8; ++x) {
                const long long at = part + (long long)min(x0 + x, pieces - 1) * rows + r;
                ml[x] = plan.ml[at];
                v[x] = *(const f32x4 *)(plan.o + at * d + e);
            }
            float to = top;
#pragma unroll
            for (int x = 0; x < 8; ++x) to = fmaxf(to, ml[x].x);
            const float keep = weight_of(top, total, to);
            total *= keep;
            sum *= keep;
            top = to;
#pragma unroll
            for (int x = 0; x < 8; ++x)
                if (x0 + x < pieces) {
                    const float f = weight_of(ml[x].x, ml[x].y, top);
                    total += f * ml[x].y;
                    sum += f * v[x];
                }
        }
        if (top == kFloor && total > 0.0f) total = kNone;
        const int i = w.i_lo + (local0 + r) / a.group, head = w.kvh * a.group + (local0 + r) % a.group;
        *(f16x4 *)(a.o + (long long)(w.first + i) * a.ldo + (long long)head * d + e) = __builtin_convertvector(sum * factor_of(top, total), f16x4);
    }
}

size_t up256(size_t v) { return (v + 255) & ~(size_t)255; }

// How a call is divided.
struct Form {
    int rows, tile;                 // rows of a workgroup, tokens of a tile
    long long row_tiles, groups;    // of a sequence and head, and of all
    int pieces, tiles;
};

// Workgroups that fill the chip, of 32 rows and heads of more than 64 dimensions, whose two waves hold half as much, twice as many; tiles of a piece, at least.  (22 trees of 20
// nodes, 16 heads of 96, to 4571 tokens, codes: 78 us with 3 pieces each, 104 with 2; 5 of 15 nodes, 12 heads of 80, 4580 tokens, fp16: 38
// us with 9 pieces, 45 with 17, which cost more to join than they gain.)
constexpr int kFill = 512, kLeast = 4;

// Tiles of `tile` tokens that a workgroup's rows see at most, `span` tokens being its own.
long long tiles_seen(int max_length, int window, int sinks, long long span, int tile)
{
    const long long all = ((long long)max_length + tile - 1) / tile;
    return window ? std::min(all, ((long long)window + sinks + span + tile - 1) / tile + 4) : all;
}

Form form_of(int S, int n_heads, int n_kv_heads, int head_dim, int max_new, int max_length, int window, int sinks, bool tree)
{
    Form f;
    const int group = n_heads / n_kv_heads;
    const long long most = (long long)max_new * group, all = (long long)S * n_kv_heads;
    // Rows of a workgroup.  Wider tiles read keys and values less often and keep the matrix pipes busier, narrower ones are more workgroups, and waste
    // less at the edges of a window.  us with 32 / 64 / 128 rows, workgroups of 64 (of 128) rows in brackets:
    //   heads of 128, 12 of 512 tokens 19.2 / 16.7 / 19.4 [96 (48)]; 32 of 8, 1000 tokens 49.8 / 41.3 / 38.8 [504 (256)];
    //     a window of 256: 2 sequences of 1024, 16 heads 23 / 19.1 / 23.2 [512 (256)]; 32 of 8, 4096 codes 90 / 69 / 51 [2048 (1024)];
    //     trees of 32 nodes, 32 of 8, 4000 tokens: 4 of them 36.8 / 29.5 / 32.5 [64 (32)], 8 55 / 44 / 41, 64 375 / 257 / 198;
    //   heads of 64, 16 of 2048 tokens 31.2 / 32.9 / 36.8 [512 (256)], codes 37.6 / 44.7 / 50.9; of 4096 tokens 85.7 / 67.9 / 80.4 [1024 (512)];
    //     32 of 8, 8192 tokens - / 449 / 366 [4096 (2048)]; a window of 256: 12 of 512 tokens 11.1 / 13.6 / 15.9 [96 (48)],
    //     16 of 2048 21.0 / 13.6 / 18.7 [512 (256)], 16 of 8192 - / 35.8 / 34.0 [2048 (1024)], codes - / 43.1 / 48.7;
    //     trees of 64 nodes, 12 heads, 1000 tokens: 4 of them 15.4 / 14.1, 64 71 / 40; of 32 nodes, 32 of 8: 4 of them - / 14.0 / 15.5 [64 (32)], 64
    //     - / 47.9 / 38.5 [1024 (512)].
    auto groups = [&](int rows) { return all * ((most + rows - 1) / rows); };
    const bool narrow = window && window < max_length;
    f.rows = 32;
    if (head_dim > 64) {
        if (most > 32) f.rows = 64;
        if (most > 64 && groups(128) >= (tree ? 64 : narrow ? 512 : 128)) f.rows = 128;
    } else {
        if (most > 32 && (tree || groups(64) >= (narrow ? 192 : 768))) f.rows = 64;
        if (most > 64 && groups(128) >= (tree ? 256 : 1024)) f.rows = 128;
    }
    if (head_dim > 128) f.rows = 128;
    f.tile = head_dim > 128 ? 32 : f.rows == 32 && head_dim <= 64 ? 128 : 64;
    f.row_tiles = (most + f.rows - 1) / f.rows;
    f.groups = all * f.row_tiles;
    const long long tiles = tiles_seen(max_length, window, sinks, std::min((long long)max_new, (long long)f.rows / group + 2), f.tile);
    f.pieces = 1;
    f.tiles = (int)tiles;
    const long long twice = f.rows == 32 && head_dim > 64 ? std::min((2 * kFill + f.groups - 1) / f.groups, 8ll) : 1;
    // Heads to 64 dimensions: no more of them than the chip holds at a time, three a CU.  (24 single tokens over 1000, 20 heads, fp16: 27.7 us with 480
    // workgroups, 34.3 with 960; over 100 to 1000 21.8 and 27.0.  Wider heads, two a CU, gain as much where sequences are equally long, 40 trees over 4000
    // tokens 152 us and 184, but lose more where they are not, 130 and 95 over 400 to 4000.)
    const long long at_once = head_dim <= 64 ? std::max(3 * 256 / f.groups, 1ll) : kFill;
    const long long want = std::min({std::max((kFill + f.groups - 1) / f.groups, twice), at_once, tiles / kLeast});
    if (want > 1) {
        f.tiles = (int)((tiles + want - 1) / want);
        f.pieces = (int)((tiles + f.tiles - 1) / f.tiles);
    }
    return f;
}

// Whether a call goes to the attention of one new token.
bool single(int S, int n_heads, int n_kv_heads, int head_dim, int max_new, int max_length, int window, int sinks, bool tree)
{
    return !tree && max_new == 1 && attend_rows_fits(S, n_heads, n_kv_heads, head_dim, max_length, window, sinks);
}

size_t bytes_of(size_t parts, int head_dim) { return up256(parts * head_dim * 4) + up256(parts * 8); }

template <int kD, bool kInt8>
hipError_t launch_d(const RowsArgs &a, const Plan &plan, const Form &f, hipStream_t s)
{
    const dim3 grid((unsigned)(f.row_tiles * a.c.n_kv_heads), a.S, f.pieces);
    hipError_t e;
    if constexpr (kD == 256) {
        e = launch_kernel(k_rows<kD, kInt8, 4, 4, 32>, grid, dim3(256), 0, s, a, plan);
    } else {
        if (f.rows == 128)
            e = launch_kernel(k_rows<kD, kInt8, 4, 4, 64>, grid, dim3(256), 0, s, a, plan);
        else if (f.rows == 64)
            e = launch_kernel(k_rows<kD, kInt8, 4, 2, 64>, grid, dim3(256), 0, s, a, plan);
        else if constexpr (kD == 64)
            e = launch_kernel(k_rows<kD, kInt8, 4, 1, 128>, grid, dim3(256), 0, s, a, plan);
        else
            e = launch_kernel(k_rows<kD, kInt8, 2, 1, 64>, grid, dim3(128), 0, s, a, plan);
    }
    if (e != hipSuccess || f.pieces == 1) return e;
    const dim3 join((unsigned)(f.row_tiles * a.c.n_kv_heads), a.S, std::max(1, std::min(f.rows * a.c.head_dim / 4 / kJoinThreads, 8)));
    if (f.tile == 32) return launch_kernel(k_rows_join<32>, join, dim3(kJoinThreads), 0, s, a, plan, f.rows);
    if (f.tile == 64) return launch_kernel(k_rows_join<64>, join, dim3(kJoinThreads), 0, s, a, plan, f.rows);
    return launch_kernel(k_rows_join<128>, join, dim3(kJoinThreads), 0, s, a, plan, f.rows);
}

}  // namespace

size_t rows_workspace_need(int S, int n_heads, int n_kv_heads, int head_dim, int max_new, int max_length, int window, int sinks, bool tree)
{
    if (single(S, n_heads, n_kv_heads, head_dim, max_new, max_length, window, sinks, tree)) return 0;
    const Form f = form_of(S, n_heads, n_kv_heads, head_dim, max_new, max_length, window, sinks, tree);
    return f.pieces > 1 ? bytes_of((size_t)f.groups * f.pieces * f.rows, head_dim) : 0;
}

// Enough for every smaller call: where a call is cut, all its workgroups are fewer than 4 kFill.
size_t rows_workspace_bytes(int, int n_heads, int n_kv_heads, int head_dim, int max_new, int max_length, int window, int sinks, bool)
{
    const long long most = (long long)max_new * (n_heads / n_kv_heads);
    const int rows = head_dim > 128 || most > 64 ? 128 : most > 32 ? 64 : 32;
    if (tiles_seen(max_length, window, sinks, std::min(max_new, 130), head_dim > 128 ? 32 : 64) < 2 * kLeast) return 0;
    return bytes_of((size_t)4 * kFill * rows, head_dim);
}

hipError_t rows_prepare()
{
    hipFuncAttributes at;
    return hipFuncGetAttributes(&at, (const void *)k_rows<64, false, 4, 1, 128>);
}

hipError_t launch_rows(const RowsArgs &a, bool int8, hipStream_t s)
{
    const int d = a.c.head_dim;
    if (single(a.S, a.n_heads, a.c.n_kv_heads, d, a.max_new, a.max_length, a.window, a.sinks, a.parents != nullptr)) {
        AttendArgs b{};
        b.q = a.q, b.o = a.o, b.table = a.table, b.lengths = a.lengths, b.starts = a.starts;
        b.S = a.S, b.M = a.M, b.n_heads = a.n_heads, b.group = a.group, b.ldq = a.ldq, b.ldo = a.ldo, b.ld_table = a.ld_table;
        b.max_length = a.max_length, b.window = a.window, b.sinks = a.sinks;
        b.scale = std::min(std::max(a.scale, -2.0e38f), 2.0e38f);            // (times log2(e) it stays a number)
        b.c = a.c;
        return launch_attend_rows(b, int8, s);
    }
    const Form f = form_of(a.S, a.n_heads, a.c.n_kv_heads, d, a.max_new, a.max_length, a.window, a.sinks, a.parents != nullptr);
    if (f.row_tiles * a.c.n_kv_heads > (1 << 23) + a.c.n_kv_heads) return hipErrorInvalidValue;
    Plan plan{(int)f.row_tiles, f.pieces, f.tiles, nullptr, nullptr};
    if (f.pieces > 1) {
        const size_t parts = (size_t)f.groups * f.pieces * f.rows;
        plan.o = (float *)a.workspace;
        plan.ml = (float2 *)((char *)a.workspace + up256(parts * d * 4));
    }
    if (d <= 64) return int8 ? launch_d<64, true>(a, plan, f, s) : launch_d<64, false>(a, plan, f, s);
    if (d <= 128) return int8 ? launch_d<128, true>(a, plan, f, s) : launch_d<128, false>(a, plan, f, s);
    return int8 ? launch_d<256, true>(a, plan, f, s) : launch_d<256, false>(a, plan, f, s);
}

}  // namespace muxq
