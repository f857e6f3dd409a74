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
// one part would add an error as large as the output's rounding.  They are kept at up to 2^15 (m stands 8
// below the running maximum's exponent, and moves only when a score is 7 above it), so that small ones
// keep their bits: of the types with 16 bits fp16 has the exact codes and the bits, and this gives it the range.  8-bit codes are exact
// in fp16; the scale of a key goes to its score, the scale of a value to its weight, over a running power of two.
#include "muxq_block_kernels.h"

namespace muxq {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __fp16 fp16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kTile = 32;               // tokens of a wave's step
constexpr int kMaxChunk = kAttendMaxChunk, kMinChunk = 512;
constexpr int kWorkgroups = 1024;      // to fill the chip, four on a CU
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

// 2^(m - top) of a part with maximum m and sum l; one without weights counts nothing, unless NaN stands there.
__device__ __forceinline__ float weight_of(float m, float l, float top) { return m == kFloor ? l : exp2_(m - top); }

struct Split {
    int chunk;          // tokens of a workgroup, a multiple of 256
    int n;              // splits of the longest sequence
    float *o;           // [S][heads][n][d], unnormalised
    float2 *ml;         // [S][heads][n]: m and the sum
};

// Heads of one key-value head that a workgroup takes: the columns of the products, and what the joining in LDS holds.
template <int kD>
constexpr int kHeads = kD == 256 ? 8 : 16;

template <int kD, bool kInt8, bool kFull, int kWaves>
__global__ __launch_bounds__(64 * kWaves) void k_attend(AttendArgs a, Split sp)
{
    constexpr int NS = kD / 32, VE = kD / 16, kThreads = 64 * kWaves;
    constexpr int KW = kInt8 ? NS / 2 : NS, VW = kInt8 ? VE / 4 : VE / 2;      // 16-byte pieces of a key row, words of a value row
    extern __shared__ __align__(16) char lds[];
    __shared__ float sh_m[kWaves][16], sh_l[kWaves][16], sh_cap[kWaves];
    __shared__ int sh_bad;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 15, g = lane >> 4;
    const int subs = (a.group + kHeads<kD> - 1) / kHeads<kD>;
    const int kvh = blockIdx.x / subs, sub = blockIdx.x - kvh * subs, split = blockIdx.y, s = blockIdx.z;
    const int head0 = kvh * a.group + sub * kHeads<kD>, n_here = min(kHeads<kD>, a.group - sub * kHeads<kD>);
    const int d = a.c.head_dim, shift = a.c.block_shift, mask = (1 << shift) - 1;
    const int len = min(a.lengths[s], a.max_length);
    const int t0 = split * sp.chunk, t1 = min(len, t0 + sp.chunk);
    if (t0 >= len) {
        if (sp.n == 1)                       // an idle place
            for (int i = tid; i < n_here * d; i += kThreads) a.o[(long long)s * a.ldo + (long long)head0 * d + i] = (_Float16)0.0f;
        return;
    }

    // where the pages of the chunk stand, in elements (with codes: their numbers); -1: not in the cache
    long long *const sh_off = (long long *)lds;
    const int first = t0 >> shift, pages = ((t1 - 1) >> shift) - first + 1, room = pages + 4;
    if (tid == 0) sh_bad = 0;
    __syncthreads();
    for (int i = tid; i < room; i += kThreads) {
        long long at = -1;
        if (i < pages) {
            const int page = a.table[(long long)s * a.ld_table + first + i];
            if (page >= 0 && page < a.c.n_blocks)
                at = kInt8 ? page : page * a.c.ld_block + kvh * a.c.ld_head;
            else
                sh_bad = 1;
        }
        sh_off[i] = at;
    }

    // queries: column `col` of the right operand, the dimensions in the left one's order
    f16x8 q[NS];
    const _Float16 *qrow = a.q + (long long)s * a.ldq + (long long)(head0 + min(col, n_here - 1)) * d;
#pragma unroll
    for (int st = 0; st < NS; ++st) {
        const int at = kInt8 ? 64 * (st >> 1) + 16 * g + 8 * (st & 1) : 32 * st + 8 * g;
        q[st] = f16x8{};
        if (col < n_here && (kFull || at < d)) q[st] = *(const f16x8 *)(qrow + at);
    }
    __syncthreads();
    const bool any_bad = sh_bad != 0;

    const float c = a.scale * 1.44269504088896f;
    float m = kFloor, l = 0.0f, cap = 0.0f, cap_inv = 0.0f;
    f32x4 o[VE] = {};
    // what is on its way: keys of tokens 16 t + col, values of tokens 16 t + 4 g + i, and their scales
    uint4 k[2][KW];
    uint32_t v[8][VW];
    float4 ks[2], vs[2];

    auto is_masked = [&](int tok) { return any_bad || tok + kTile > t1; };
    auto load_k = [&](auto masked_c, int tok) {
        constexpr bool kMasked = decltype(masked_c)::value;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int kt = tok + 16 * t + col;
            long long at = sh_off[(kt >> shift) - first];
            const bool there = !kMasked || (at >= 0 && kt < t1);
            if (kInt8) at = at * a.c.ld_block + kvh * a.c.ld_head;
            const long long row = there ? at + (kt & mask) * a.c.ld_token : 0;
#pragma unroll
            for (int u = 0; u < KW; ++u) {
                const int e = kInt8 ? 64 * u + 16 * g : 32 * u + 8 * g;
                k[t][u] = uint4{0, 0, 0, 0};
                if (kFull || e < d) k[t][u] = *(const uint4 *)(a.c.k + (row + e) * (kInt8 ? 1 : 2));
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
                const bool there = !kMasked || (page >= 0 && vt + i < t1);
                const char *p = a.c.v + (there ? at + ((vt & mask) + i) * a.c.ld_token + VE * col : 0) * (kInt8 ? 1 : 2);
                uint32_t *w = v[4 * t + i];
#pragma unroll
                for (int x = 0; x < VW; ++x) w[x] = 0;
                if (kFull || VE * col < d) {
                    if constexpr (VW == 1) {
                        w[0] = *(const uint32_t *)p;
                    } else if constexpr (VW == 2) {
                        const uint2 y = *(const uint2 *)p;
                        w[0] = y.x, w[1] = y.y;
                    } else {
#pragma unroll
                        for (int x = 0; x < VW / 4; ++x) {
                            const uint4 y = ((const uint4 *)p)[x];
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

    // The keys of the next step are requested when this step's are in the matrix pipes, its values when this step's are: the
    // same registers, and something is always on its way.
    int tok = t0 + wave * kTile;
    if (tok < t1) {
        ask_k(tok);
        ask_v(tok);
    }
    for (; tok < t1; tok += kWaves * kTile) {
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
        if (next < t1) ask_k(next);

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
                if (kt >= t1 || sh_off[(kt >> shift) - first] < 0) p[j] = kFloor, w[j] = 0.0f;
            }
        }
        float top = fmaxf(fmaxf(fmaxf(p[0], p[1]), fmaxf(p[2], p[3])), fmaxf(fmaxf(p[4], p[5]), fmaxf(p[6], p[7])));
        if (__any(top > m + 7.0f)) {                    // rare after the first steps: a new maximum for the head
            top = fmaxf(top, __shfl_xor(top, 16, 64));
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            const float to = fmaxf(m, top), keep = m == kFloor ? 0.0f : exp2_(m - to);
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
        if (next < t1) ask_v(next);
    }

    // The waves' parts: m and l by head, then sum_w 2^(m_w - max m) o_w in LDS, [wave][head][d], the upper half of the waves
    // through the lower one's places.
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (lane < 16) sh_m[wave][lane] = m, sh_l[wave][lane] = l;
    __syncthreads();
    float top = sh_m[0][col];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) top = fmaxf(top, sh_m[w][col]);
    const float f = weight_of(m, l, top) * (kInt8 ? cap : 1.0f);
#pragma unroll
    for (int e = 0; e < VE; ++e) o[e] *= f;
    float *const sh_o = (float *)lds;
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
        if (sp.n == 1) {
            const float inv = most == kFloor ? 0.0f : 1.0f / all;
            f16x4 r;
#pragma unroll
            for (int x = 0; x < 4; ++x) r[x] = (_Float16)(sum[x] * inv);
            *(f16x4 *)(a.o + (long long)s * a.ldo + (long long)(head0 + h) * d + e) = r;
        } else {
            const long long part = ((long long)s * a.n_heads + head0 + h) * sp.n + split;
            *(f32x4 *)(sp.o + part * d + e) = sum;
            if (e == 0) sp.ml[part] = make_float2(most, all);
        }
    }
}

// The splits of a sequence and head joined, with weights 2^(m - max m): a thread four dimensions of every
// (512 / (d / 4))th split, its first eight requested before the weights are known.
__global__ __launch_bounds__(512) void k_attend_join(AttendArgs a, Split sp)
{
    __shared__ float red[16], weight[512];
    __shared__ f32x4 part[512];
    const int tid = threadIdx.x, h = blockIdx.x, s = blockIdx.y, d = a.c.head_dim;
    const int len = min(a.lengths[s], a.max_length), n = len <= 0 ? 0 : (len + sp.chunk - 1) / sp.chunk;
    const long long row = ((long long)s * a.n_heads + h) * sp.n;
    const float2 *const ml = sp.ml + row;
    const int lanes = d / 4, per = 512 / lanes, mine = tid / lanes, e = (tid - mine * lanes) * 4;
    const float *const o = sp.o + row * d + e;
    f32x4 early[8] = {};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (mine < per && mine + i * per < n) early[i] = *(const f32x4 *)(o + (long long)(mine + i * per) * d);
    float2 x = make_float2(kFloor, 0.0f);
    if (tid < n) x = ml[tid];
    float top = x.x;
    for (int i = tid + 512; i < n; i += 512) top = fmaxf(top, ml[i].x);
    for (int y = 1; y < 64; y <<= 1) top = fmaxf(top, __shfl_xor(top, y, 64));
    if ((tid & 63) == 0) red[tid >> 6] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 8; ++w) top = fmaxf(top, red[w]);
    weight[tid] = weight_of(x.x, x.y, top);
    float all = weight[tid] * x.y;
    for (int i = tid + 512; i < n; i += 512) all += weight_of(ml[i].x, ml[i].y, top) * ml[i].y;
    for (int y = 1; y < 64; y <<= 1) all += __shfl_xor(all, y, 64);
    if ((tid & 63) == 0) red[8 + (tid >> 6)] = all;
    __syncthreads();
    f32x4 sum = {};
    if (mine < per) {
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += weight[min(mine + i * per, 511)] * early[i];
        for (int i = mine + 8 * per; i < n; i += per) sum += weight_of(ml[i].x, ml[i].y, top) * *(const f32x4 *)(o + (long long)i * d);
    }
    part[tid] = sum;
    __syncthreads();
    if (tid < lanes) {
        all = 0.0f;
#pragma unroll
        for (int w = 0; w < 8; ++w) all += red[8 + w];
        for (int i = 1; i < per; ++i) sum += part[i * lanes + tid];
        const float inv = top == kFloor ? 0.0f : 1.0f / all;
        f16x4 r;
#pragma unroll
        for (int y = 0; y < 4; ++y) r[y] = (_Float16)(sum[y] * inv);
        *(f16x4 *)(a.o + (long long)s * a.ldo + (long long)h * d + e) = r;
    }
}

int heads_of(int head_dim) { return head_dim > 128 ? kHeads<256> : kHeads<128>; }

Split split_of(int S, int n_heads, int n_kv_heads, int head_dim, int max_length)
{
    const int group = n_heads / n_kv_heads, subs = (group + heads_of(head_dim) - 1) / heads_of(head_dim);
    const long long base = (long long)S * n_kv_heads * subs;
    const long long want = (kWorkgroups + base - 1) / base;
    const long long chunk = ((max_length + want - 1) / want + 255) / 256 * 256;
    Split sp{};
    sp.chunk = (int)(chunk < kMinChunk ? kMinChunk : chunk > kMaxChunk ? kMaxChunk : chunk);
    sp.n = (int)(((long long)max_length + sp.chunk - 1) / sp.chunk);
    return sp;
}

// 8 waves where each has a step or more and their parts are worth joining in LDS.
int waves_of(const Split &sp, int max_length) { return min(sp.chunk, max_length) > 256 ? 8 : 4; }

size_t up256(size_t v) { return (v + 255) & ~(size_t)255; }

size_t parts_bytes(size_t splits, int n_heads, int head_dim)
{
    return up256(splits * n_heads * head_dim * 4) + up256(splits * n_heads * 8);
}

template <int kD, int kWaves>
hipError_t launch_w(const AttendArgs &a, const Split &sp, bool int8, hipStream_t s)
{
    const int subs = (a.group + kHeads<kD> - 1) / kHeads<kD>;
    const dim3 grid(a.c.n_kv_heads * subs, sp.n, a.S), block(64 * kWaves);
    const size_t offs = ((size_t)(sp.chunk >> a.c.block_shift) + 5) * 8;
    const size_t join = (size_t)4 * (a.group < kHeads<kD> ? a.group : kHeads<kD>) * kD * 4;
    const size_t lds = offs > join ? offs : join;
    const bool full = a.c.head_dim == kD;
    if (int8)
        return full ? launch_kernel(k_attend<kD, true, true, kWaves>, grid, block, lds, s, a, sp)
                    : launch_kernel(k_attend<kD, true, false, kWaves>, grid, block, lds, s, a, sp);
    return full ? launch_kernel(k_attend<kD, false, true, kWaves>, grid, block, lds, s, a, sp)
                : launch_kernel(k_attend<kD, false, false, kWaves>, grid, block, lds, s, a, sp);
}

template <int kD>
hipError_t launch_d(const AttendArgs &a, const Split &sp, bool int8, hipStream_t s)
{
    return waves_of(sp, a.max_length) == 8 ? launch_w<kD, 8>(a, sp, int8, s) : launch_w<kD, 4>(a, sp, int8, s);
}

}  // namespace

// Of this call.
size_t attend_workspace_need(int S, int n_heads, int n_kv_heads, int head_dim, int max_length)
{
    const Split sp = split_of(S, n_heads, n_kv_heads, head_dim, max_length);
    return sp.n == 1 ? 0 : parts_bytes((size_t)S * sp.n, n_heads, head_dim);
}

// Of this call and every smaller one (S and max_length): there are ceil(max_length / chunk) splits, at most `want` of
// them unless the longest chunk forces more, and S want < 1024 / heads + S.
size_t attend_workspace_bytes(int S, int n_heads, int n_kv_heads, int head_dim, int max_length)
{
    if (max_length <= kMinChunk) return 0;
    const int group = n_heads / n_kv_heads, subs = (group + heads_of(head_dim) - 1) / heads_of(head_dim);
    const size_t forced = (size_t)S * ((max_length + kMaxChunk - 1) / kMaxChunk), shortest = (size_t)S * ((max_length + kMinChunk - 1) / kMinChunk);
    const size_t wanted = (size_t)(kWorkgroups / (n_kv_heads * subs)) + S;
    const size_t most = shortest < wanted ? shortest : wanted;
    return parts_bytes(forced > most ? forced : most, n_heads, head_dim);
}

hipError_t launch_attend(const AttendArgs &a, bool int8, hipStream_t s)
{
    Split sp = split_of(a.S, a.n_heads, a.c.n_kv_heads, a.c.head_dim, a.max_length);
    const size_t parts = (size_t)a.S * a.n_heads * sp.n;
    sp.o = (float *)a.workspace;
    sp.ml = (float2 *)((char *)a.workspace + up256(parts * a.c.head_dim * 4));
    const int d = a.c.head_dim;
    hipError_t e = d <= 64 ? launch_d<64>(a, sp, int8, s) : d <= 128 ? launch_d<128>(a, sp, int8, s) : launch_d<256>(a, sp, int8, s);
    if (e != hipSuccess || sp.n == 1) return e;
    return launch_kernel(k_attend_join, dim3(a.n_heads, a.S), dim3(512), 0, s, a, sp);
}

}  // namespace muxq
