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

template <int kD, bool kInt8, bool kFull>
__global__ __launch_bounds__(256) void k_attend(AttendArgs a, Split sp)
{
    constexpr int NS = kD / 32, VE = kD / 16, VW = VE / 2;
    extern __shared__ char lds[];
    __shared__ float sh_m[4][16], sh_l[4][16], sh_cap[4];
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
            for (int i = tid; i < n_here * d; i += 256) a.o[(long long)s * a.ldo + (long long)head0 * d + i] = (_Float16)0.0f;
        return;
    }

    // where the pages of the chunk stand, in elements; -1: not in the cache
    long long *const sh_off = (long long *)lds;
    const int first = t0 >> shift, pages = ((t1 - 1) >> shift) - first + 1, room = (pages + 4);
    if (tid == 0) sh_bad = 0;
    __syncthreads();
    for (int i = tid; i < room; i += 256) {
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

    // queries: column `col` of the right operand, the dimensions of the left one's order
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

    auto tile = [&](auto masked_c, const int tok) {
        constexpr bool kMasked = decltype(masked_c)::value;
        uint32_t v[8][VW];
        float ks[8], vs[8];
        f16x8 k[2][NS];
        bool k_there[2][4];                 // of the tokens whose scores the lane will hold
        long long vat[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            // keys: row `col` of the left operand is token 16 t + col
            const int kt = tok + 16 * t + col, kp = (kt >> shift) - first;
            long long at = sh_off[kp];
            if (kInt8) at = (kMasked && at < 0) ? -1 : at * a.c.ld_block + kvh * a.c.ld_head;
            const bool there = !kMasked || (at >= 0 && kt < t1);
            const long long krow = there ? at + (kt & mask) * a.c.ld_token : 0;
            if constexpr (!kInt8) {
#pragma unroll
                for (int st = 0; st < NS; ++st) {
                    k[t][st] = f16x8{};
                    if (kFull || 32 * st + 8 * g < d) k[t][st] = *(const f16x8 *)((const _Float16 *)a.c.k + krow + 32 * st + 8 * g);
                }
            } else {
#pragma unroll
                for (int u = 0; u < NS / 2; ++u) {
                    uint4 w = {0, 0, 0, 0};
                    if (kFull || 64 * u + 16 * g < d) w = *(const uint4 *)(a.c.k + krow + 64 * u + 16 * g);
                    uint32_t h[8];
                    codes_to_half(w.x, h[0], h[1]);
                    codes_to_half(w.y, h[2], h[3]);
                    codes_to_half(w.z, h[4], h[5]);
                    codes_to_half(w.w, h[6], h[7]);
                    k[t][2 * u] = half8(h[0], h[1], h[2], h[3]);
                    k[t][2 * u + 1] = half8(h[4], h[5], h[6], h[7]);
                }
            }
            // values and scores: the lane's tokens are 16 t + 4 g + 0..3, in one page
            const int vt = tok + 16 * t + 4 * g, vp = (vt >> shift) - first;
            const long long page = sh_off[vp];
            vat[t] = kInt8 ? page * a.c.ld_block + kvh * a.c.ld_head : page;
#pragma unroll
            for (int i = 0; i < 4; ++i) k_there[t][i] = !kMasked || (page >= 0 && vt + i < t1);
            if constexpr (kInt8) {
                const long long at_s = (kMasked && page < 0) ? 0 : ((page * a.c.n_kv_heads + kvh) << shift) + (vt & mask);
                const float4 ks4 = *(const float4 *)(a.c.k_scale + at_s), vs4 = *(const float4 *)(a.c.v_scale + at_s);
                const float kk[4] = {ks4.x, ks4.y, ks4.z, ks4.w}, vv[4] = {vs4.x, vs4.y, vs4.z, vs4.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) ks[4 * t + i] = kk[i] * c, vs[4 * t + i] = k_there[t][i] ? vv[i] : 0.0f;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const long long row = k_there[t][i] ? vat[t] + ((vt & mask) + i) * a.c.ld_token + VE * col : 0;
                uint32_t *w = v[4 * t + i];
#pragma unroll
                for (int x = 0; x < VW; ++x) w[x] = 0;
                if (kFull || VE * col < d) {
                    if constexpr (!kInt8) {
                        const _Float16 *p = (const _Float16 *)a.c.v + row;
                        if constexpr (VE == 4) {
                            const uint2 x = *(const uint2 *)p;
                            w[0] = x.x, w[1] = x.y;
                        } else {
#pragma unroll
                            for (int x = 0; x < VE / 8; ++x) {
                                const uint4 y = *(const uint4 *)(p + 8 * x);
                                w[4 * x] = y.x, w[4 * x + 1] = y.y, w[4 * x + 2] = y.z, w[4 * x + 3] = y.w;
                            }
                        }
                    } else {
                        const char *p = a.c.v + row;
                        if constexpr (VE == 4) {
                            codes_to_half(*(const uint32_t *)p, w[0], w[1]);
                        } else if constexpr (VE == 8) {
                            const uint2 x = *(const uint2 *)p;
                            codes_to_half(x.x, w[0], w[1]);
                            codes_to_half(x.y, w[2], w[3]);
                        } else {
                            const uint4 x = *(const uint4 *)p;
                            codes_to_half(x.x, w[0], w[1]);
                            codes_to_half(x.y, w[2], w[3]);
                            codes_to_half(x.z, w[4], w[5]);
                            codes_to_half(x.w, w[6], w[7]);
                        }
                    }
                }
                if (kMasked && !k_there[t][i]) {
#pragma unroll
                    for (int x = 0; x < VW; ++x) w[x] = 0;
                }
            }
        }

        f32x4 acc[2] = {};
#pragma unroll
        for (int st = 0; st < NS; ++st) {
            acc[0] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k[0][st], q[st], acc[0], 0, 0, 0);
            acc[1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k[1][st], q[st], acc[1], 0, 0, 0);
        }
        float p[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            p[j] = acc[j >> 2][j & 3] * (kInt8 ? ks[j] : c);
            if (kMasked && !k_there[j >> 2][j & 3]) p[j] = kFloor;
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
            float most = fmaxf(fmaxf(fmaxf(vs[0], vs[1]), fmaxf(vs[2], vs[3])), fmaxf(fmaxf(vs[4], vs[5]), fmaxf(vs[6], vs[7])));
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
            for (int j = 0; j < 8; ++j) p[j] *= vs[j] * cap_inv;
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
            const uint32_t sel = (e & 1) ? 0x07060302u : 0x05040100u;
            uint32_t t[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) t[j] = __builtin_amdgcn_perm(v[2 * j + 1][e >> 1], v[2 * j][e >> 1], sel);
            const f16x8 vt = half8(t[0], t[1], t[2], t[3]);
            o[e] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vt, ph, o[e], 0, 0, 0);
            o[e] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vt, pl, o[e], 0, 0, 0);
        }
    };
    for (int tok = t0 + wave * kTile; tok < t1; tok += 4 * kTile) {
        if (any_bad || tok + kTile > t1)
            tile(std::true_type{}, tok);
        else
            tile(std::false_type{}, tok);
    }

    // the four waves' parts: m and l by head, o as [wave][head][d]
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    __syncthreads();
    float *const sh_o = (float *)lds;
    if (lane < 16) sh_m[wave][lane] = m, sh_l[wave][lane] = l;
    if (lane == 0) sh_cap[wave] = kInt8 ? cap : 1.0f;
    if (col < n_here) {
        float *row = sh_o + (wave * n_here + col) * kD;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < VE; e += 4) *(f32x4 *)(row + VE * (4 * g + i) + e) = f32x4{o[e][i], o[e + 1][i], o[e + 2][i], o[e + 3][i]};
    }
    __syncthreads();
    for (int i = tid; i < n_here * (kD / 4); i += 256) {
        const int h = i / (kD / 4), e = (i - h * (kD / 4)) * 4;
        if (!kFull && e >= d) continue;
        const float top = fmaxf(fmaxf(sh_m[0][h], sh_m[1][h]), fmaxf(sh_m[2][h], sh_m[3][h]));
        f32x4 sum = {};
        float all = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float f = weight_of(sh_m[w][h], sh_l[w][h], top);
            all += f * sh_l[w][h];
            sum += (f * sh_cap[w]) * *(const f32x4 *)(sh_o + (w * n_here + h) * kD + e);
        }
        if (sp.n == 1) {
            typedef _Float16 h4 __attribute__((ext_vector_type(4)));
            const float inv = top == kFloor ? 0.0f : 1.0f / all;
            h4 r;
#pragma unroll
            for (int x = 0; x < 4; ++x) r[x] = (_Float16)(sum[x] * inv);
            *(h4 *)(a.o + (long long)s * a.ldo + (long long)(head0 + h) * d + e) = r;
        } else {
            const long long part = ((long long)s * a.n_heads + head0 + h) * sp.n + split;
            *(f32x4 *)(sp.o + part * d + e) = sum;
            if (e == 0) sp.ml[part] = make_float2(top, all);
        }
    }
}

// The splits of a sequence and head joined, with weights 2^(m - max m): a thread four dimensions of every
// (256 / (d / 4))th split.
__global__ __launch_bounds__(256) void k_attend_join(AttendArgs a, Split sp)
{
    __shared__ float red[8];
    __shared__ f32x4 part[256];
    const int tid = threadIdx.x, h = blockIdx.x, s = blockIdx.y, d = a.c.head_dim;
    const int len = min(a.lengths[s], a.max_length), n = len <= 0 ? 0 : (len + sp.chunk - 1) / sp.chunk;
    const long long row = ((long long)s * a.n_heads + h) * sp.n;
    const float2 *const ml = sp.ml + row;
    float top = kFloor;
    for (int i = tid; i < n; i += 256) top = fmaxf(top, ml[i].x);
    for (int x = 1; x < 64; x <<= 1) top = fmaxf(top, __shfl_xor(top, x, 64));
    if ((tid & 63) == 0) red[tid >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    float all = 0.0f;
    for (int i = tid; i < n; i += 256) all += weight_of(ml[i].x, ml[i].y, top) * ml[i].y;
    for (int x = 1; x < 64; x <<= 1) all += __shfl_xor(all, x, 64);
    if ((tid & 63) == 0) red[4 + (tid >> 6)] = all;
    const int lanes = d / 4, per = 256 / lanes, mine = tid / lanes, e = (tid - mine * lanes) * 4;
    f32x4 sum = {};
    if (mine < per)
        for (int i = mine; i < n; i += per) sum += weight_of(ml[i].x, ml[i].y, top) * *(const f32x4 *)(sp.o + (row + i) * d + e);
    part[tid] = sum;
    __syncthreads();
    all = (red[4] + red[5]) + (red[6] + red[7]);
    if (tid < lanes) {
        for (int i = 1; i < per; ++i) sum += part[i * lanes + tid];
        typedef _Float16 h4 __attribute__((ext_vector_type(4)));
        const float inv = top == kFloor ? 0.0f : 1.0f / all;
        h4 r;
#pragma unroll
        for (int x = 0; x < 4; ++x) r[x] = (_Float16)(sum[x] * inv);
        *(h4 *)(a.o + (long long)s * a.ldo + (long long)h * d + e) = r;
    }
}

int heads_of(int head_dim) { return head_dim > 128 ? kHeads<256> : kHeads<128>; }

// Tokens of a workgroup.
int chunk_of(int S, int n_heads, int n_kv_heads, int head_dim, int max_length)
{
    const int group = n_heads / n_kv_heads, subs = (group + heads_of(head_dim) - 1) / heads_of(head_dim);
    const long long base = (long long)S * n_kv_heads * subs;
    const long long want = (kWorkgroups + base - 1) / base;             // splits that give four workgroups a CU
    const long long chunk = ((max_length + want - 1) / want + 255) / 256 * 256;
    return (int)(chunk < kMinChunk ? kMinChunk : chunk > kMaxChunk ? kMaxChunk : chunk);
}

Split split_of(int S, int n_heads, int n_kv_heads, int head_dim, int max_length)
{
    Split sp{};
    sp.chunk = chunk_of(S, n_heads, n_kv_heads, head_dim, max_length);
    sp.n = (int)(((long long)max_length + sp.chunk - 1) / sp.chunk);
    return sp;
}

size_t up256(size_t v) { return (v + 255) & ~(size_t)255; }

size_t parts_bytes(size_t splits, int n_heads, int head_dim)
{
    return up256(splits * n_heads * head_dim * 4) + up256(splits * n_heads * 8);
}

template <int kD>
hipError_t launch_d(const AttendArgs &a, const Split &sp, bool int8, hipStream_t s)
{
    const int subs = (a.group + kHeads<kD> - 1) / kHeads<kD>;
    const dim3 grid(a.c.n_kv_heads * subs, sp.n, a.S);
    const size_t offs = ((size_t)(sp.chunk >> a.c.block_shift) + 5) * 8;
    const size_t join = (size_t)4 * (a.group < kHeads<kD> ? a.group : kHeads<kD>) * kD * 4;
    const size_t lds = offs > join ? offs : join;
    const bool full = a.c.head_dim == kD;
    if (int8)
        return full ? launch_kernel(k_attend<kD, true, true>, grid, dim3(256), lds, s, a, sp)
                    : launch_kernel(k_attend<kD, true, false>, grid, dim3(256), lds, s, a, sp);
    return full ? launch_kernel(k_attend<kD, false, true>, grid, dim3(256), lds, s, a, sp)
                : launch_kernel(k_attend<kD, false, false>, grid, dim3(256), lds, s, a, sp);
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
    return launch_kernel(k_attend_join, dim3(a.n_heads, a.S), dim3(256), 0, s, a, sp);
}

}  // namespace muxq
