// Attention of one new token over the paged cache.
//
// O = sum_t p_t V_t / sum_t p_t, p_t = 2^(s_t - m), s_t = scale log2(e) q . K_t, with the running maximum m and
// sum of the softmax, so that keys and values are read once.  What bounds it is that reading: 4 d operations to
// 4 d bytes (fp16) for one query.  Both products still go through the matrix pipes: with the keys as the left operand
// (16 tokens x 32 dimensions a step) and up to 16 queries that share the key-value head as the right one, the scores
// come out with a query per lane column, which is where the weights of the second product have to stand: weights
// go from one product to the next without leaving their lanes.  The second product has the
// transposed values as its left operand; a lane loads the rows of its 8 tokens in one run each and transposes them
// with byte permutes.  Lanes of a 16-lane row read one row of V (2 d bytes) together.
//
// Weights are fp16 in the second product, in two parts (p = hi + lo, each rounded towards zero): 22 bits, where
// one part would add an error as large as the output's rounding.  They are 2^(s - m + 8), and m follows the maximum only when a
// score is 7 above it, which is rare: up to 2^15, so that small ones keep their bits.  8-bit codes are exact in
// fp16; the scale of a key goes to its score, the scale of a value to its weight, over a running power of two.
//
// How it is divided (Plan below): short or many sequences have a workgroup of 8 waves each and key-value head, and no second
// launch; otherwise as many workgroups as the chip holds have equal shares, and a second launch joins what they cut through.
// Measured: 64 sequences of 131 to 8192 tokens, 8 key-value heads of 128, fp16, 1.09 GB: 183 us, 6.0 TB/s; one of 131071 tokens
// 95 us, 5.7 TB/s; 64 of 4096 to 8192, 8 heads of 128, 8-bit codes, 0.83 GB: 152 us, 5.5 TB/s; 24 sequences to 1024, 20 heads of 64, codes,
// 34 MB: 15.3 us, where a wave has 32 tokens on its way at a time, of 128 bytes in codes, and four such steps one after the other; one of
// 37 tokens 5.2 us (kernel trace).  Heads of 144 to 256 in fp16 without shares keep arrays in scratch memory: 64 sequences to 1000, 4
// heads of 256, 157 us, in codes 25.
#include "muxq_block_kernels.h"

#include <algorithm>

namespace muxq {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __fp16 fp16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kTile = 32;               // tokens of a wave's step
constexpr int kStep = 4 * kTile;        // tokens of a step of the 4 waves that have shares
constexpr int kBegin = 1;               // what beginning a sequence and head costs, in steps
constexpr int kPages = 4096;            // tokens whose pages stand in LDS at a time
constexpr int kMaxSeqs = 2048;          // sequences whose steps a workgroup counts for itself
constexpr float kFloor = -__builtin_inff();

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// Four codes of a word as fp16 values, exactly: code + 128 in the low byte of 0x64.. is 1024 + code + 128.
__device__ __forceinline__ void codes_to_half(uint32_t w, uint32_t &lo, uint32_t &hi)
{
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    const uint32_t u = w ^ 0x80808080u;
    const uint32_t a = __builtin_amdgcn_perm(0x64646464u, u, 0x07010700u), b = __builtin_amdgcn_perm(0x64646464u, u, 0x07030702u);
    const h2 bias = {(_Float16)1152.0f, (_Float16)1152.0f};
    lo = __builtin_bit_cast(uint32_t, __builtin_bit_cast(h2, a) - bias);
    hi = __builtin_bit_cast(uint32_t, __builtin_bit_cast(h2, b) - bias);
}

__device__ __forceinline__ f16x8 half8(uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    return __builtin_bit_cast(f16x8, u32x4{a, b, c, d});
}

// kOnce: past the caches.  Long caches are read once and gain a tenth by it (131072 tokens: 91 us against 100); short ones
// may be in the memory-side cache from the step before and lose a third (24 sequences to 2000: 26 us against 20).
template <typename V, bool kOnce>
__device__ __forceinline__ V load(const char *p)
{
    typedef uint32_t Word __attribute__((ext_vector_type(sizeof(V) / 4)));
    return __builtin_bit_cast(V, kOnce ? __builtin_nontemporal_load((const Word *)p) : *(const Word *)p);
}

// 2^(m - top) of a part with maximum m and sum l, never quite 0, so that an infinity among the values stays one; one without
// weights counts nothing, unless NaN stands there.  (Where it has tokens, all of them with a score of -infinity, its sum is kNone: beside a
// part with weights that is nothing, and where no part has any it says that the softmax is 0 / 0, not an empty row.)
constexpr float kNone = 0x1p-60f;
__device__ __forceinline__ float weight_of(float m, float l, float top) { return m == kFloor ? l : fmaxf(exp2_(m - top), 1.1754944e-38f); }

// What the sum of the values is multiplied by in the end.
__device__ __forceinline__ float factor_of(float m, float l) { return m != kFloor ? 1.0f / l : l == 0.0f ? 0.0f : __builtin_nanf(""); }

// How the work is divided.  groups == 0: a workgroup to a sequence and key-value head.  Otherwise `groups` workgroups
// have equal shares of all steps (kStep tokens of one key-value head, and kBegin steps before the first) in the order
// sequence, head, step (fewer workgroups where there are fewer steps);
// a share that begins or ends inside a sequence and head leaves its part of it in the workspace: the first
// piece of a share in slot 0, the last one in slot 1.
struct Plan {
    int groups;
    float *o;           // [groups][2][heads of a workgroup][d], unnormalised
    float2 *ml;         // [groups][2][heads of a workgroup]: m and the sum
    int4 *open;         // [groups]: {sequence, pair, pieces, slot of the first} that the share leaves open, pieces 0: none
};

// Heads of one key-value head that a workgroup takes: the columns of the products, and what the joining in LDS holds.
template <int kD>
constexpr int kHeads = kD == 256 ? 8 : 16;

// The values of tokens t0 to t1 that are infinite or NaN, four dimensions from e on, with weights of 1, or of 0 where the query's score is
// -infinity: all that counts for a sum in which there is one.  The matrix product makes NaN of it, since the low part of a weight, or all of
// it, may be 0 in 16 bits; a thread that finds NaN or an infinity goes through the tokens by itself.
template <bool kInt8>
__device__ __forceinline__ f32x4 loose_values(const AttendArgs &a, int s, int kvh, int head, int e, int t0, int t1)
{
    const int d = a.c.head_dim, shift = a.c.block_shift, mask = (1 << shift) - 1;
    const _Float16 *const q = a.q + (long long)s * a.ldq + (long long)head * d;
    f32x4 sum = {};
    for (int t = t0; t < t1; ++t) {
        const int page = a.table[(long long)s * a.ld_table + (t >> shift)];
        if (page < 0 || page >= a.c.n_blocks) continue;
        const long long row = page * a.c.ld_block + kvh * a.c.ld_head + (t & mask) * a.c.ld_token;
        const long long at_s = (((long long)page * a.c.n_kv_heads + kvh) << shift) + (t & mask);
        f32x4 v;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            if constexpr (kInt8)
                v[x] = (float)((const int8_t *)a.c.v)[row + e + x] * a.c.v_scale[at_s];
            else
                v[x] = (float)((const _Float16 *)a.c.v)[row + e + x];
        }
        const f32x4 zero = v - v;
        if (zero[0] == 0.0f && zero[1] == 0.0f && zero[2] == 0.0f && zero[3] == 0.0f) continue;
        float score = 0.0f;
        for (int i = 0; i < d; ++i)
            score += (float)q[i] * (kInt8 ? (float)((const int8_t *)a.c.k)[row + i] : (float)((const _Float16 *)a.c.k)[row + i]);
        score *= a.scale;
        if constexpr (kInt8) score *= a.c.k_scale[at_s];
#pragma unroll
        for (int x = 0; x < 4; ++x)
            if (zero[x] != 0.0f) sum[x] += score == kFloor ? 0.0f * v[x] : v[x];
        if (sum[0] != sum[0] && sum[1] != sum[1] && sum[2] != sum[2] && sum[3] != sum[3]) break;
    }
    return sum;
}

template <int kD, bool kInt8, bool kFull, int kWaves, bool kShares>
__global__ __launch_bounds__(64 * kWaves, kD == 64 ? 4 : kD == 128 || kWaves == 8 ? 2 : 1) void k_attend(AttendArgs a, Plan plan)
{
    constexpr int NS = kD / 32, VE = kD / 16, kThreads = 64 * kWaves;
    constexpr int KW = kInt8 ? NS / 2 : NS, VW = kInt8 ? VE / 4 : VE / 2;      // 16-byte pieces of a key row, words of a value row
    extern __shared__ __align__(16) char lds[];
    __shared__ float sh_m[kWaves][16], sh_l[kWaves][16];
    __shared__ int sh_bad, sh_sum[kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 15, g = lane >> 4;
    const int subs = (a.group + kHeads<kD> - 1) / kHeads<kD>, pairs = a.c.n_kv_heads * subs;
    const int d = a.c.head_dim, shift = a.c.block_shift, mask = (1 << shift) - 1;
    auto length_of = [&](int s) { return max(0, min(a.lengths[s], a.max_length)); };
    auto steps_of = [&](int s) {
        const int len = length_of(s);
        return len > 0 ? kBegin + (len + kStep - 1) / kStep : 0;
    };

    // The share: steps [at, end), `at` being step j of `n` of sequence s and pair `pair`.  Steps before a
    // sequence, of one pair, are counted in LDS.
    int s = blockIdx.y, pair = blockIdx.x, j = 0, n = 0;
    long long at = 0, end = 0;
    int *const sh_before = (int *)lds;
    char *const rest = lds + (kShares ? ((a.S + 4) / 4) * 16 : 0);
    long long total = 0;
    int groups = 0;
    if constexpr (kShares) {
        for (int i = blockIdx.x; i < a.S; i += plan.groups)             // idle places
            if (a.lengths[i] <= 0)
                for (int e = tid; e < a.n_heads * d; e += kThreads) a.o[(long long)i * a.ldo + e] = (_Float16)0.0f;
        const int per = (a.S + kThreads - 1) / kThreads;
        int sum = 0;
        for (int i = tid * per; i < min(a.S, (tid + 1) * per); ++i) sum += steps_of(i);
        int incl = sum;
        for (int x = 1; x < 64; x <<= 1) {
            const int y = __shfl_up(incl, x, 64);
            if (lane >= x) incl += y;
        }
        if (lane == 63) sh_sum[wave] = incl;
        __syncthreads();
        int before = incl - sum, all = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            if (w < wave) before += sh_sum[w];
            all += sh_sum[w];
        }
        for (int i = tid * per; i < min(a.S, (tid + 1) * per); ++i) {
            sh_before[i] = before;
            before += steps_of(i);
        }
        if (tid == 0) sh_before[a.S] = all;
        __syncthreads();
        total = (long long)all * pairs;
        groups = (int)min((long long)plan.groups, total);      // every share has a step
        if ((int)blockIdx.x >= groups) {
            if (tid == 0) plan.open[blockIdx.x] = int4{0, 0, 0, 0};
            return;
        }
        at = total * blockIdx.x / groups;
        end = total * (blockIdx.x + 1) / groups;
        int lo = 0, hi = a.S;                     // the last sequence whose steps begin at or before `at`
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            ((long long)sh_before[mid] * pairs <= at ? lo : hi) = mid;
        }
        s = lo;
        n = sh_before[s + 1] - sh_before[s];      // (at least one: `at` lies in it)
        const long long in = at - (long long)sh_before[s] * pairs;
        pair = (int)(in / n);
        j = (int)(in - (long long)pair * n);
    }

    for (int piece = 0;; ++piece) {
        const int kvh = pair / subs, sub = pair - kvh * subs;
        const int head0 = kvh * a.group + sub * kHeads<kD>, n_here = min(kHeads<kD>, a.group - sub * kHeads<kD>);
        const int len = length_of(s);
        int t0 = 0, t1 = len;
        bool whole = true;
        if constexpr (kShares) {
            const int steps = (int)min((long long)(n - j), end - at);
            t0 = min(len, max(0, j - kBegin) * kStep);
            t1 = min(len, max(0, j + steps - kBegin) * kStep);
            whole = steps == n;
            at += steps;
        } else if (len == 0) {                       // an idle place
            for (int i = tid; i < n_here * d; i += kThreads) a.o[(long long)s * a.ldo + (long long)head0 * d + i] = (_Float16)0.0f;
            return;
        }

        // queries: column `col` of the right operand, the dimensions in the left one's order
        f16x8 q[NS];
        const _Float16 *qrow = a.q + (long long)s * a.ldq + (long long)(head0 + min(col, n_here - 1)) * d;
#pragma unroll
        for (int st = 0; st < NS; ++st) {
            const int e = kInt8 ? 64 * (st >> 1) + 16 * g + 8 * (st & 1) : 32 * st + 8 * g;
            q[st] = f16x8{};
            if (col < n_here && (kFull || e < d)) q[st] = *(const f16x8 *)(qrow + e);
        }

        const float c = a.scale * 1.44269504088896f;
        float m = kFloor, l = 0.0f, cap = 0.0f, cap_inv = 0.0f;
        f32x4 o[VE] = {};
        // what is on its way: keys of tokens 16 t + col, values of tokens 16 t + 4 g + i, and their scales
        uint4 k[2][KW];
        uint32_t v[8][VW];
        float4 ks[2], vs[2];

        // where the pages from token `c0` on stand, in elements (with codes: their numbers); -1: not in the cache
        long long *const sh_off = (long long *)rest;
        int first = 0, c1 = 0;
        bool any_bad = false;
        auto is_masked = [&](int tok) { return any_bad || tok + kTile > c1; };
        auto load_k = [&](auto masked_c, int tok) {
            constexpr bool kMasked = decltype(masked_c)::value;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int kt = tok + 16 * t + col;
                long long at = sh_off[(kt >> shift) - first];
                const bool there = !kMasked || (at >= 0 && kt < c1);
                if (kInt8) at = at * a.c.ld_block + kvh * a.c.ld_head;
                const long long row = there ? at + (kt & mask) * a.c.ld_token : 0;
#pragma unroll
                for (int u = 0; u < KW; ++u) {
                    const int e = kInt8 ? 64 * u + 16 * g : 32 * u + 8 * g;
                    k[t][u] = uint4{0, 0, 0, 0};
                    if (kFull || e < d) k[t][u] = load<uint4, kShares>(a.c.k + (row + e) * (kInt8 ? 1 : 2));
                }
            }
        };
        auto load_v = [&](auto masked_c, int tok) {
            constexpr bool kMasked = decltype(masked_c)::value;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                // the lane's tokens are 16 t + 4 g + 0..3, in one page
                const int vt = tok + 16 * t + 4 * g;
                const long long page = sh_off[(vt >> shift) - first];
                const long long at = kInt8 ? page * a.c.ld_block + kvh * a.c.ld_head : page;
                if constexpr (kInt8) {
                    const long long at_s = (kMasked && page < 0) ? 0 : ((page * a.c.n_kv_heads + kvh) << shift) + (vt & mask);
                    ks[t] = *(const float4 *)(a.c.k_scale + at_s);
                    vs[t] = *(const float4 *)(a.c.v_scale + at_s);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const bool there = !kMasked || (page >= 0 && vt + i < c1);
                    const char *p = a.c.v + (there ? at + ((vt & mask) + i) * a.c.ld_token + VE * col : 0) * (kInt8 ? 1 : 2);
                    uint32_t *w = v[4 * t + i];
#pragma unroll
                    for (int x = 0; x < VW; ++x) w[x] = 0;
                    if (kFull || VE * col < d) {
                        if constexpr (VW == 1) {
                            w[0] = load<uint32_t, kShares>(p);
                        } else if constexpr (VW == 2) {
                            const uint2 y = load<uint2, kShares>(p);
                            w[0] = y.x, w[1] = y.y;
                        } else {
#pragma unroll
                            for (int x = 0; x < VW / 4; ++x) {
                                const uint4 y = load<uint4, kShares>(p + 16 * x);
                                w[4 * x] = y.x, w[4 * x + 1] = y.y, w[4 * x + 2] = y.z, w[4 * x + 3] = y.w;
                            }
                        }
                    }
                    if (kMasked && !there) {          // what stands there may be NaN: its weight of 0 does not clear it
#pragma unroll
                        for (int x = 0; x < VW; ++x) w[x] = 0;
                    }
                }
            }
        };
        auto ask_k = [&](int tok) {
            if (is_masked(tok)) load_k(std::true_type{}, tok); else load_k(std::false_type{}, tok);
        };
        auto ask_v = [&](int tok) {
            if (is_masked(tok)) load_v(std::true_type{}, tok); else load_v(std::false_type{}, tok);
        };

        for (int c0 = t0; c0 < t1; c0 = c1) {
            c1 = min(t1, c0 + kPages);
            first = c0 >> shift;
            const int pages = ((c1 - 1) >> shift) - first + 1;
            __syncthreads();                              // the last piece's readers
            if (tid == 0) sh_bad = 0;
            __syncthreads();
            for (int i = tid; i < pages + 4; i += kThreads) {
                long long where = -1;
                if (i < pages) {
                    const int page = a.table[(long long)s * a.ld_table + first + i];
                    if (page >= 0 && page < a.c.n_blocks)
                        where = kInt8 ? page : page * a.c.ld_block + kvh * a.c.ld_head;
                    else
                        sh_bad = 1;
                }
                sh_off[i] = where;
            }
            __syncthreads();
            any_bad = sh_bad != 0;

            // The keys of the next step are requested when this step's are in the matrix pipes, its values when this step's are: the
            // same registers, and something is always on its way.
            int tok = c0 + wave * kTile;
            if (tok < c1) {
                ask_k(tok);
                ask_v(tok);
            }
            for (; tok < c1; tok += kWaves * kTile) {
                const int next = tok + kWaves * kTile;
                f32x4 acc[2] = {};
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int u = 0; u < KW; ++u) {
                        if constexpr (!kInt8) {
                            acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, k[t][u]), q[u], acc[t], 0, 0, 0);
                        } else {
                            uint32_t h[8];
                            codes_to_half(k[t][u].x, h[0], h[1]);
                            codes_to_half(k[t][u].y, h[2], h[3]);
                            codes_to_half(k[t][u].z, h[4], h[5]);
                            codes_to_half(k[t][u].w, h[6], h[7]);
                            acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(half8(h[0], h[1], h[2], h[3]), q[2 * u], acc[t], 0, 0, 0);
                            acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(half8(h[4], h[5], h[6], h[7]), q[2 * u + 1], acc[t], 0, 0, 0);
                        }
                    }
                if (next < c1) ask_k(next);

                float p[8], w[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) p[j] = acc[j >> 2][j & 3] * c;
                if constexpr (kInt8) {
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        p[4 * t] *= ks[t].x, p[4 * t + 1] *= ks[t].y, p[4 * t + 2] *= ks[t].z, p[4 * t + 3] *= ks[t].w;
                        w[4 * t] = vs[t].x, w[4 * t + 1] = vs[t].y, w[4 * t + 2] = vs[t].z, w[4 * t + 3] = vs[t].w;
                    }
                }
                if (is_masked(tok)) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int kt = tok + 16 * (j >> 2) + 4 * g + (j & 3);
                        if (kt >= c1 || sh_off[(kt >> shift) - first] < 0) p[j] = kFloor, w[j] = 0.0f;
                    }
                }
                float top = fmaxf(fmaxf(fmaxf(p[0], p[1]), fmaxf(p[2], p[3])), fmaxf(fmaxf(p[4], p[5]), fmaxf(p[6], p[7])));
                if (__any(top > m + 7.0f)) {                    // rare after the first steps: a new maximum for the head
                    top = fmaxf(top, __shfl_xor(top, 16, 64));
                    top = fmaxf(top, __shfl_xor(top, 32, 64));
                    const float to = fmaxf(m, top), keep = weight_of(m, l, to);
                    m = to;
                    l *= keep;
#pragma unroll
                    for (int e = 0; e < VE; ++e) o[e] *= keep;
                }
                const float off = m == kFloor ? 0.0f : 8.0f - m;
#pragma unroll
                for (int j = 0; j < 8; ++j) p[j] = exp2_(p[j] + off);
                l += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
                if constexpr (kInt8) {
                    float most = fmaxf(fmaxf(fmaxf(w[0], w[1]), fmaxf(w[2], w[3])), fmaxf(fmaxf(w[4], w[5]), fmaxf(w[6], w[7])));
                    if (__any(most > cap)) {                    // scales of values over a power of two
                        most = fmaxf(most, __shfl_xor(most, 16, 64));
                        most = fmaxf(most, __shfl_xor(most, 32, 64));
                        const uint32_t ex = min(__float_as_uint(most) >> 23, 252u) + 1;
                        const float was = cap;
                        cap = fmaxf(cap, __uint_as_float(ex << 23));
                        cap_inv = __uint_as_float((254u - (__float_as_uint(cap) >> 23)) << 23);
                        const float keep = was * cap_inv;
#pragma unroll
                        for (int e = 0; e < VE; ++e) o[e] *= keep;
                    }
#pragma unroll
                    for (int j = 0; j < 8; ++j) p[j] *= w[j] * cap_inv;
                }
                uint32_t hi[4], lo[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const fp16x2 h = __builtin_amdgcn_cvt_pkrtz(p[2 * j], p[2 * j + 1]);
                    const fp16x2 r = __builtin_amdgcn_cvt_pkrtz(p[2 * j] - (float)h[0], p[2 * j + 1] - (float)h[1]);
                    hi[j] = __builtin_bit_cast(uint32_t, h);
                    lo[j] = __builtin_bit_cast(uint32_t, r);
                }
                const f16x8 ph = half8(hi[0], hi[1], hi[2], hi[3]), pl = half8(lo[0], lo[1], lo[2], lo[3]);
#pragma unroll
                for (int e = 0; e < VE; ++e) {
                    uint32_t x[4];
                    if constexpr (!kInt8) {
                        const uint32_t sel = (e & 1) ? 0x07060302u : 0x05040100u;
#pragma unroll
                        for (int j = 0; j < 4; ++j) x[j] = __builtin_amdgcn_perm(v[2 * j + 1][e >> 1], v[2 * j][e >> 1], sel);
                    } else {
                        // byte e of the words of two tokens and two more, then as codes_to_half
                        const uint32_t sel = 0x0c0c0400u + 0x0101u * (e & 3);
                        uint32_t y[2];
#pragma unroll
                        for (int j = 0; j < 2; ++j)
                            y[j] = __builtin_amdgcn_perm(v[4 * j + 1][e >> 2], v[4 * j][e >> 2], sel) |
                                   (__builtin_amdgcn_perm(v[4 * j + 3][e >> 2], v[4 * j + 2][e >> 2], sel) << 16);
                        codes_to_half(y[0], x[0], x[1]);
                        codes_to_half(y[1], x[2], x[3]);
                    }
                    const f16x8 vt = half8(x[0], x[1], x[2], x[3]);
                    o[e] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vt, ph, o[e], 0, 0, 0);
                    o[e] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vt, pl, o[e], 0, 0, 0);
                }
                if (next < c1) ask_v(next);
            }
        }

        // The waves' parts: m and l by head, then sum_w 2^(m_w - max m) o_w in LDS, [wave][head][d], the upper half of the waves
        // through the lower one's places.
        l += __shfl_xor(l, 16, 64);
        l += __shfl_xor(l, 32, 64);
        if (__any(l == 0.0f)) {                           // no weights: are there tokens?
            bool seen = false;
            for (int tok = t0 + wave * kTile; tok < t1; tok += kWaves * kTile) {
                const int kt = tok + (lane & (kTile - 1));
                if (kt >= t1) break;
                const int page = a.table[(long long)s * a.ld_table + (kt >> shift)];
                seen |= page >= 0 && page < a.c.n_blocks;
            }
            if (__any(seen) && l == 0.0f) l = kNone;
        }
        if (lane < 16) sh_m[wave][lane] = m, sh_l[wave][lane] = l;
        __syncthreads();
        float top = sh_m[0][col];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) top = fmaxf(top, sh_m[w][col]);
        const float f = weight_of(m, l, top) * (kInt8 ? cap : 1.0f);
#pragma unroll
        for (int e = 0; e < VE; ++e) o[e] *= f;
        float *const sh_o = (float *)rest;
        float *const mine = sh_o + ((wave & 3) * n_here + col) * kD;
        auto put = [&](bool add) {
            if (col >= n_here) return;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < VE; e += 4) {
                    f32x4 *at = (f32x4 *)(mine + VE * (4 * g + i) + e);
                    f32x4 x = {o[e][i], o[e + 1][i], o[e + 2][i], o[e + 3][i]};
                    if (add) x += *at;
                    *at = x;
                }
        };
        if constexpr (kWaves == 8) {
            if (wave >= 4) put(false);
            __syncthreads();
            if (wave < 4) put(true);
        } else {
            put(false);
        }
        __syncthreads();
        for (int i = tid; i < n_here * (kD / 4); i += kThreads) {
            const int h = i / (kD / 4), e = (i - h * (kD / 4)) * 4;
            if (!kFull && e >= d) continue;
            float most = sh_m[0][h], all = 0.0f;
#pragma unroll
            for (int w = 1; w < kWaves; ++w) most = fmaxf(most, sh_m[w][h]);
#pragma unroll
            for (int w = 0; w < kWaves; ++w) all += weight_of(sh_m[w][h], sh_l[w][h], most) * sh_l[w][h];
            f32x4 sum = {};
#pragma unroll
            for (int w = 0; w < 4; ++w) sum += *(const f32x4 *)(sh_o + (w * n_here + h) * kD + e);
            const f32x4 zero = sum - sum;
            if (!(zero[0] + zero[1] + (zero[2] + zero[3]) == 0.0f) && all == all) {
                const f32x4 loose = loose_values<kInt8>(a, s, kvh, head0 + h, e, t0, t1);
#pragma unroll
                for (int x = 0; x < 4; ++x)
                    if (loose[x] - loose[x] != 0.0f) sum[x] = loose[x];
            }
            __builtin_amdgcn_wave_barrier();              // (O may be Q: a head's lanes are of one wave, and have read its query before one writes)
            if (whole) {
                const float inv = factor_of(most, all);
                f16x4 r;
#pragma unroll
                for (int x = 0; x < 4; ++x) r[x] = (_Float16)(sum[x] * inv);
                *(f16x4 *)(a.o + (long long)s * a.ldo + (long long)(head0 + h) * d + e) = r;
            } else {
                const int part = (blockIdx.x * 2 + (piece ? 1 : 0)) * min(a.group, kHeads<kD>) + h;
                *(f32x4 *)(plan.o + (long long)part * d + e) = sum;
                if (e == 0) plan.ml[part] = make_float2(most, most == kFloor && all > 0.0f ? kNone : all);
            }
        }
        if constexpr (!kShares) return;
        if (at >= end) {
            if (tid == 0) {
                // open: the first of the shares that have a part of this pair, which later ones finish
                const long long from = (long long)sh_before[s] * pairs + (long long)pair * n, begin = total * blockIdx.x / groups;
                const int last = (int)(((from + n) * groups - 1) / total);       // the share of the pair's last step
                const bool first_of = begin <= from && end < from + n;
                plan.open[blockIdx.x] = int4{s, pair, first_of ? last - (int)blockIdx.x + 1 : 0, begin == from ? 0 : 1};
            }
            return;
        }
        __syncthreads();                                  // (a next piece without tokens goes straight to sh_m)
        // on to the next pair, or the next sequence that has steps
        j = 0;
        if (++pair == pairs) {
            pair = 0;
            do ++s; while (sh_before[s + 1] == sh_before[s]);
            n = sh_before[s + 1] - sh_before[s];
        }
    }
}

// The pieces of a pair that several shares have, joined by weights 2^(m - max m): a workgroup to a share that leaves a pair
// open, a thread four dimensions of a head of every (512 / those)th piece.
__global__ __launch_bounds__(512) void k_attend_join(AttendArgs a, Plan plan, int heads)
{
    __shared__ float sh_top[16], sh_inv[16];
    __shared__ f32x4 part[512];
    const int4 open = plan.open[blockIdx.x];
    if (open.z == 0) return;
    const int tid = threadIdx.x, lane = tid & 63, d = a.c.head_dim, s = open.x, pieces = open.z;
    const int subs = (a.group + heads - 1) / heads, kvh = open.y / subs, sub = open.y - kvh * subs;
    const int head0 = kvh * a.group + sub * heads, n_here = min(heads, a.group - sub * heads), stride = min(a.group, heads);
    // the first share's piece is in the slot it says, the others begin with theirs
    auto place = [&](int i) { return ((blockIdx.x + i) * 2 + (i == 0 ? open.w : 0)) * stride; };
    for (int h = tid >> 6; h < n_here; h += 8) {
        float top = kFloor, all = 0.0f;
        for (int i = lane; i < pieces; i += 64) top = fmaxf(top, plan.ml[place(i) + h].x);
        for (int x = 1; x < 64; x <<= 1) top = fmaxf(top, __shfl_xor(top, x, 64));
        for (int i = lane; i < pieces; i += 64) {
            const float2 x = plan.ml[place(i) + h];
            all += weight_of(x.x, x.y, top) * x.y;
        }
        for (int x = 1; x < 64; x <<= 1) all += __shfl_xor(all, x, 64);
        if (lane == 0) sh_top[h] = top, sh_inv[h] = factor_of(top, all);
    }
    __syncthreads();
    const int lanes = d / 4, items = n_here * lanes, per = items < 512 ? 512 / items : 1;
    for (int base = 0; base < items; base += 512) {
        const int mine = items < 512 ? tid / items : 0, item = base + (items < 512 ? tid - mine * items : tid);
        const int h = item / lanes, e = (item - h * lanes) * 4;
        const bool live = mine < per && item < items;
        f32x4 sum = {};
        if (live) {
            const float top = sh_top[h];
#pragma unroll 4
            for (int i = mine; i < pieces; i += per) {
                const float2 x = plan.ml[place(i) + h];
                sum += weight_of(x.x, x.y, top) * *(const f32x4 *)(plan.o + (long long)(place(i) + h) * d + e);
            }
        }
        if (per > 1) {
            __syncthreads();
            part[tid] = sum;
            __syncthreads();
            if (live && mine == 0)
                for (int i = 1; i < per; ++i) sum += part[i * items + item];
        }
        if (live && mine == 0) {
            f16x4 r;
#pragma unroll
            for (int y = 0; y < 4; ++y) r[y] = (_Float16)(sum[y] * sh_inv[h]);
            *(f16x4 *)(a.o + (long long)s * a.ldo + (long long)(head0 + h) * d + e) = r;
        }
    }
}

int heads_of(int head_dim) { return head_dim > 128 ? kHeads<256> : kHeads<128>; }

// Workgroups that are on the chip at once, by their registers: of 4 waves with shares, and of 8 waves.
int resident(int head_dim) { return head_dim <= 64 ? 1024 : head_dim <= 128 ? 512 : 256; }
int resident8(int head_dim) { return head_dim <= 64 ? 512 : 256; }

// Shares where a workgroup of 8 waves to each sequence and head would go through many tokens one after the other, fewer
// where those workgroups leave most of the chip idle.  (us, shares against none: 8 x 8 heads of 128 to 1500 tokens
// 16.2 / 20.6, 128 x 8 to 2048 104 / 117, 64 x 8 to 8192 189 / 247, 40 x 8 to 1024 29.1 / 24.3; heads of 64: 24 x 12 to 4000
// 37.6 / 45.0, 24 x 20 to 2500 40.2 / 40.6, 64 x 12 to 2048 51.3 / 47.4, 4 x 12 to 1024 12.6 / 11.0.)
bool shares_pay(int S, int n_heads, int n_kv_heads, int head_dim, int max_length)
{
    const int group = n_heads / n_kv_heads, subs = (group + heads_of(head_dim) - 1) / heads_of(head_dim);
    const int most = head_dim <= 64 ? 2500 : 1500;
    const bool idle = (long long)S * n_kv_heads * subs * 4 <= resident8(head_dim);
    return max_length > (idle ? most / 2 : most) && S <= kMaxSeqs;
}

size_t up256(size_t v) { return (v + 255) & ~(size_t)255; }

size_t parts_of(int n_heads, int n_kv_heads, int head_dim)
{
    return (size_t)resident(head_dim) * 2 * std::min(n_heads / n_kv_heads, heads_of(head_dim));
}

template <int kD, int kWaves, bool kShares>
hipError_t launch_w(const AttendArgs &a, const Plan &plan, bool int8, hipStream_t s)
{
    const int pairs = a.c.n_kv_heads * ((a.group + kHeads<kD> - 1) / kHeads<kD>);
    const dim3 grid = kShares ? dim3(plan.groups) : dim3(pairs, a.S), block(64 * kWaves);
    const size_t offs = ((size_t)(std::min(a.max_length, kPages) >> a.c.block_shift) + 6) * 8;
    const size_t join = (size_t)4 * std::min(a.group, kHeads<kD>) * kD * 4;
    const size_t lds = std::max(offs, join) + (kShares ? (size_t)((a.S + 4) / 4) * 16 : 0);
    const bool full = a.c.head_dim == kD;
    if (int8)
        return full ? launch_kernel(k_attend<kD, true, true, kWaves, kShares>, grid, block, lds, s, a, plan)
                    : launch_kernel(k_attend<kD, true, false, kWaves, kShares>, grid, block, lds, s, a, plan);
    return full ? launch_kernel(k_attend<kD, false, true, kWaves, kShares>, grid, block, lds, s, a, plan)
                : launch_kernel(k_attend<kD, false, false, kWaves, kShares>, grid, block, lds, s, a, plan);
}

template <int kD>
hipError_t launch_d(const AttendArgs &a, const Plan &plan, bool int8, hipStream_t s)
{
    if (plan.groups) return launch_w<kD, 4, true>(a, plan, int8, s);
    // 8 waves where each has tokens (4 sequences of 12 heads to 1024 tokens: 10.8 us, 13.0 with 4)
    return a.max_length > 128 ? launch_w<kD, 8, false>(a, plan, int8, s) : launch_w<kD, 4, false>(a, plan, int8, s);
}

}  // namespace

size_t attend_workspace_need(int S, int n_heads, int n_kv_heads, int head_dim, int max_length)
{
    if (!shares_pay(S, n_heads, n_kv_heads, head_dim, max_length)) return 0;
    const size_t parts = parts_of(n_heads, n_kv_heads, head_dim);
    return up256(parts * head_dim * 4) + up256(parts * 8) + up256((size_t)resident(head_dim) * 16);
}

// Enough for every smaller S and max_length: what one of them needs does not depend on which.
size_t attend_workspace_bytes(int S, int n_heads, int n_kv_heads, int head_dim, int max_length)
{
    size_t most = 0;
    for (int x = 1; x <= S && x <= kMaxSeqs; ++x)
        if ((most = attend_workspace_need(x, n_heads, n_kv_heads, head_dim, max_length)) > 0) break;
    return most;
}

hipError_t attend_prepare()
{
    hipFuncAttributes at;
    return hipFuncGetAttributes(&at, (const void *)k_attend<64, false, true, 4, false>);
}

hipError_t launch_attend(const AttendArgs &a, bool int8, hipStream_t s)
{
    const int d = a.c.head_dim;
    Plan plan{};
    if (attend_workspace_need(a.S, a.n_heads, a.c.n_kv_heads, d, a.max_length) > 0) {
        const size_t parts = parts_of(a.n_heads, a.c.n_kv_heads, d);
        plan.groups = resident(d);
        plan.o = (float *)a.workspace;
        plan.ml = (float2 *)((char *)a.workspace + up256(parts * d * 4));
        plan.open = (int4 *)((char *)plan.ml + up256(parts * 8));
    }
    const hipError_t e = d <= 64 ? launch_d<64>(a, plan, int8, s) : d <= 128 ? launch_d<128>(a, plan, int8, s) : launch_d<256>(a, plan, int8, s);
    if (e != hipSuccess || plan.groups == 0) return e;
    return launch_kernel(k_attend_join, dim3(plan.groups), dim3(512), 0, s, a, plan, heads_of(d));
}

}  // namespace muxq
