// The paged key-value cache: new tokens in, rotated on the way (k_kv_append), and rows back out (k_kv_gather).
//
// Both only move data: a token and head is head_dim values in and as many out.  Eight lanes' worth of 8
// values are one head of 64, so a wave holds several (token, head) pairs side by side, each in a group of
// P lanes, P the power of two at or above head_dim / 8; the abs-max of a head for its codes is a reduction
// inside the group.
#include "muxq_block_kernels.h"

namespace muxq {
namespace {

typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float group_max(float v, int P)
{
    for (int m = 1; m < P; m <<= 1) v = fmaxf(v, __shfl_xor(v, m, 64));
    return v;
}

// Eight values of one head of a token: those at `e` (0, 8, ... of the head) unless they rotate in halves: then four
// at j and the four at j + rot / 2, their partners.  lo / hi: where the two runs of four stand.
__device__ __forceinline__ void runs(int unit, int rot, bool interleaved, int &lo, int &hi)
{
    const int e = unit * 8;
    if (e < rot && !interleaved) {
        lo = unit * 4;
        hi = lo + rot / 2;
    } else {
        lo = e;
        hi = e + 4;
    }
}

template <bool kInt8, bool kInterleaved>
__global__ __launch_bounds__(256) void k_kv_append(AppendArgs a, int P)
{
    const int d = a.c.head_dim, Hkv = a.c.n_kv_heads, heads = a.n_heads + 2 * Hkv;
    const long long pair = ((long long)blockIdx.x * 256 + threadIdx.x) / P;
    const int unit = threadIdx.x & (P - 1);
    const int m = (int)(pair / heads), row = (int)(pair - (long long)m * heads);
    if (m >= a.M) return;                                     // whole groups
    const bool is_q = row < a.n_heads, is_v = row >= a.n_heads + Hkv;
    const int head = is_q ? row : is_v ? row - a.n_heads - Hkv : row - a.n_heads;
    const _Float16 *src = (is_q ? a.q + (long long)m * a.ldq : is_v ? a.v + (long long)m * a.ldv : a.k + (long long)m * a.ldk) + (long long)head * d;
    const int rot = is_v ? 0 : a.rot_dim;
    int position = 0;
    bool turned = true;
    if (a.rot_dim) {
        position = a.positions[m];
        turned = (unsigned)position < (unsigned)a.n_positions;
    }
    const bool live = unit * 8 < d;
    int lo = 0, hi = 4;
    float v[8] = {};
    if (live) {
        runs(unit, rot, kInterleaved, lo, hi);
        const f16x4 x = *(const f16x4 *)(src + lo), y = *(const f16x4 *)(src + hi);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = (float)x[i], v[4 + i] = (float)y[i];
        if (unit * 8 < rot && turned) {
            const float *cs = a.cos_sin + (long long)position * rot + unit * 4;
            const float4 c4 = *(const float4 *)cs, s4 = *(const float4 *)(cs + rot / 2);
            const float c[4] = {c4.x, c4.y, c4.z, c4.w}, s[4] = {s4.x, s4.y, s4.z, s4.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float &p = kInterleaved ? v[2 * i] : v[i], &q = kInterleaved ? v[2 * i + 1] : v[4 + i];
                const float t = p * c[i] - q * s[i];
                q = q * c[i] + p * s[i];
                p = t;
            }
        }
    }
    if (is_q) {
        if (live) {
            _Float16 *dst = a.q_out + (long long)m * a.ldqo + (long long)head * d;
            f16x4 x, y;
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = (_Float16)v[i], y[i] = (_Float16)v[4 + i];
            *(f16x4 *)(dst + lo) = x;
            *(f16x4 *)(dst + hi) = y;
        }
        return;
    }
    const int slot = a.slots[m], shift = a.c.block_shift;
    const bool stored = turned && slot >= 0 && (slot >> shift) < a.c.n_blocks;
    const int page = stored ? slot >> shift : 0, t = slot & ((1 << shift) - 1);
    const long long at = page * a.c.ld_block + head * a.c.ld_head + t * a.c.ld_token;
    char *base = is_v ? a.c.v : a.c.k;
    if constexpr (!kInt8) {
        if (live && stored) {
            f16x4 x, y;
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = (_Float16)v[i], y[i] = (_Float16)v[4 + i];
            *(f16x4 *)((_Float16 *)base + at + lo) = x;
            *(f16x4 *)((_Float16 *)base + at + hi) = y;
        }
    } else {
        float top = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(v[i]));
        top = group_max(top, P);
        if (!stored) return;
        const float inv = top > 0.0f ? 127.0f / top : 0.0f;
        if (live) {
            uint32_t w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = quant_word(v[i], inv, 127.0f);
            *(uint32_t *)(base + at + lo) = pack_low_bytes(w[0], w[1], w[2], w[3]);
            *(uint32_t *)(base + at + hi) = pack_low_bytes(w[4], w[5], w[6], w[7]);
        }
        if (unit == 0) (is_v ? a.c.v_scale : a.c.k_scale)[((long long)page * Hkv + head) * (1 << shift) + t] = top / 127.0f;
    }
}

template <bool kInt8>
__global__ __launch_bounds__(256) void k_kv_gather(const int32_t *slots, int M, KvView c, _Float16 *k_out, int ldk,
                                                   _Float16 *v_out, int ldv)
{
    const int units = c.head_dim / 8, per_token = 2 * c.n_kv_heads * units;
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    const int m = (int)(i / per_token);
    if (m >= M) return;
    int rest = (int)(i - (long long)m * per_token);
    const bool is_v = rest >= per_token / 2;
    if (is_v) rest -= per_token / 2;
    const int head = rest / units, e = (rest - head * units) * 8;
    const int slot = slots[m], shift = c.block_shift;
    f16x8 x = {};
    if (slot >= 0 && (slot >> shift) < c.n_blocks) {
        const int page = slot >> shift, t = slot & ((1 << shift) - 1);
        const long long at = page * c.ld_block + head * c.ld_head + t * c.ld_token + e;
        const char *base = is_v ? c.v : c.k;
        if constexpr (!kInt8) {
            x = *(const f16x8 *)((const _Float16 *)base + at);
        } else {
            const float scale = (is_v ? c.v_scale : c.k_scale)[((long long)page * c.n_kv_heads + head) * (1 << shift) + t];
            const uint2 w = *(const uint2 *)(base + at);
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = (_Float16)((float)(int8_t)((j < 4 ? w.x : w.y) >> (8 * (j & 3))) * scale);
        }
    }
    *(f16x8 *)((is_v ? v_out + (long long)m * ldv : k_out + (long long)m * ldk) + (long long)head * c.head_dim + e) = x;
}

}  // namespace

hipError_t launch_kv_append(const AppendArgs &a, bool int8, bool interleaved, hipStream_t s)
{
    int P = 2;
    while (P * 8 < a.c.head_dim) P *= 2;
    const long long lanes = (long long)a.M * (a.n_heads + 2 * a.c.n_kv_heads) * P;
    const long long wgs = (lanes + 255) / 256;
    if (wgs > 0x7fffffffll) return hipErrorInvalidValue;
    const dim3 grid((unsigned)wgs);
    if (int8) return interleaved ? launch_kernel(k_kv_append<true, true>, grid, dim3(256), 0, s, a, P)
                                 : launch_kernel(k_kv_append<true, false>, grid, dim3(256), 0, s, a, P);
    return interleaved ? launch_kernel(k_kv_append<false, true>, grid, dim3(256), 0, s, a, P)
                       : launch_kernel(k_kv_append<false, false>, grid, dim3(256), 0, s, a, P);
}

hipError_t launch_kv_gather(const int32_t *slots, int M, const KvView &c, bool int8, _Float16 *k_out, int ldk,
                            _Float16 *v_out, int ldv, hipStream_t s)
{
    const long long wgs = ((long long)M * 2 * c.n_kv_heads * (c.head_dim / 8) + 255) / 256;
    if (wgs > 0x7fffffffll) return hipErrorInvalidValue;
    const dim3 grid((unsigned)wgs);
    return int8 ? launch_kernel(k_kv_gather<true>, grid, dim3(256), 0, s, slots, M, c, k_out, ldk, v_out, ldv)
                : launch_kernel(k_kv_gather<false>, grid, dim3(256), 0, s, slots, M, c, k_out, ldk, v_out, ldv);
}

}  // namespace muxq
