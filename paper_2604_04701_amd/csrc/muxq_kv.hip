// The paged key-value cache: new tokens in, rotated on the way (k_kv_append), and rows back out (k_kv_gather).
//
// Both only move data: a token and head is head_dim values in and as many out, and what bounds them is memory, or a launch.
// A lane takes two runs of E values of a head, E = 8 (16 bytes) where the rotation allows it: with halves as pairs
// the second run is the partners of the first, so that no value crosses lanes.  P lanes, a power of two, stand for
// a head, and with many tokens each goes through four heads of its token with the sines it has loaded once (the table is binary32: for
// 8 + 8 values of a head it is twice the head's bytes).  The abs-max of a head for its codes is a reduction over its P lanes.
// Measured: 8192 tokens of 32 + 8 + 8 heads of 128, rotated, 206 MB: 39.9 us, 5.2 TB/s; 64 of them to codes 3.6 us (kernel trace).  In a graph,
// inputs in the memory-side cache: the 8192 to fp16 32 us, to codes 32 us, read back as fp16 11.4 us from either.
#include "muxq_block_kernels.h"

namespace muxq {
namespace {

__device__ __forceinline__ float group_max(float v, int P)
{
    for (int m = 1; m < P; m <<= 1) v = fmaxf(v, __shfl_xor(v, m, 64));
    return v;
}

template <bool kInt8, bool kInterleaved, int E, int kHeadsOf>
__global__ __launch_bounds__(256) void k_kv_append(AppendArgs a, int P, int slots_of)
{
    typedef _Float16 Run __attribute__((ext_vector_type(E)));
    const int d = a.c.head_dim, Hkv = a.c.n_kv_heads, heads = a.n_heads + 2 * Hkv;
    const uint32_t at_lane = (uint32_t)(blockIdx.x * (256ull / P) + threadIdx.x / P);      // (the launch keeps it below 2^32)
    const int unit = threadIdx.x & (P - 1);
    const int m = (int)(at_lane / (uint32_t)slots_of), row0 = (int)(at_lane - (uint32_t)m * slots_of);
    if (m >= a.M) return;                                     // whole groups
    const bool live = unit * 2 * E < d;
    const int rot = a.rot_dim, slot = a.slots[m], shift = a.c.block_shift;
    int position = 0;
    bool turned = true;
    if (rot) {
        position = a.positions[m];
        turned = (unsigned)position < (unsigned)a.n_positions;
    }
    // where the lane's two runs stand in a head that rotates (in halves: partners, then what stays as it is, again in halves)
    // and in one that does not
    const int flat_lo = unit * E, flat_hi = d / 2 + unit * E;
    int lo = flat_lo, hi = flat_hi;
    if (!kInterleaved && rot) {
        const int u = unit - rot / (2 * E);
        lo = u < 0 ? unit * E : rot + u * E;
        hi = u < 0 ? rot / 2 + unit * E : rot + (d - rot) / 2 + u * E;
    }
    const bool turn_lo = turned && live && lo < rot, turn_hi = kInterleaved ? turned && live && hi < rot : turn_lo;
    // angles: E pairs (lo[i], hi[i]), or interleaved E / 2 pairs of each run
    float c[E], s[E];
#pragma unroll
    for (int i = 0; i < E; ++i) c[i] = s[i] = 0.0f;
    if (turn_lo || turn_hi) {
        const float *const cs = a.cos_sin + (long long)position * rot;
#pragma unroll
        for (int i = 0; i < E; i += 4) {
            const int j = !kInterleaved ? lo + i : E == 4 ? 0 : i < E / 2 ? lo / 2 + i : hi / 2 + i - E / 2;
            if (i < E / 2 || !kInterleaved ? turn_lo : turn_hi) {
                const float4 x = *(const float4 *)(cs + j), y = *(const float4 *)(cs + rot / 2 + j);
                c[i] = x.x, c[i + 1] = x.y, c[i + 2] = x.z, c[i + 3] = x.w;
                s[i] = y.x, s[i + 1] = y.y, s[i + 2] = y.z, s[i + 3] = y.w;
            }
        }
    }
    const bool stored = turned && slot >= 0 && (slot >> shift) < a.c.n_blocks;
    const int page = stored ? slot >> shift : 0, t = slot & ((1 << shift) - 1);

    Run x[kHeadsOf], y[kHeadsOf];
#pragma unroll
    for (int h = 0; h < kHeadsOf; ++h) {
        const int row = row0 + h * slots_of;
        x[h] = y[h] = Run{};
        if (live && row < heads) {
            const bool is_q = row < a.n_heads, is_v = row >= a.n_heads + Hkv;
            const _Float16 *const src = is_q ? a.q + (long long)m * a.ldq + (long long)row * d
                                        : is_v ? a.v + (long long)m * a.ldv + (long long)(row - a.n_heads - Hkv) * d
                                               : a.k + (long long)m * a.ldk + (long long)(row - a.n_heads) * d;
            x[h] = *(const Run *)(src + (is_v ? flat_lo : lo));
            y[h] = *(const Run *)(src + (is_v ? flat_hi : hi));
        }
    }
#pragma unroll
    for (int h = 0; h < kHeadsOf; ++h) {
        const int row = row0 + h * slots_of;
        if (row >= heads) break;                               // whole groups
        const bool is_q = row < a.n_heads, is_v = row >= a.n_heads + Hkv;
        const int head = is_q ? row : is_v ? row - a.n_heads - Hkv : row - a.n_heads;
        const int at_lo = is_v ? flat_lo : lo, at_hi = is_v ? flat_hi : hi;
        float v[2 * E];
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] = (float)x[h][i], v[E + i] = (float)y[h][i];
        auto turn = [&](float &p, float &q, int i) {
            const float u = p * c[i] - q * s[i];
            q = q * c[i] + p * s[i];
            p = u;
        };
        if (!is_v) {
            if constexpr (!kInterleaved) {
                if (turn_lo) {
#pragma unroll
                    for (int i = 0; i < E; ++i) turn(v[i], v[E + i], i);
                }
            } else {
                if (turn_lo) {
#pragma unroll
                    for (int i = 0; i < E / 2; ++i) turn(v[2 * i], v[2 * i + 1], i);
                }
                if (turn_hi) {
#pragma unroll
                    for (int i = E / 2; i < E; ++i) turn(v[2 * i], v[2 * i + 1], i);
                }
            }
        }
        if (is_q || !kInt8) {
            _Float16 *dst;
            if (is_q)
                dst = a.q_out + (long long)m * a.ldqo + (long long)head * d;
            else
                dst = (_Float16 *)(is_v ? a.c.v : a.c.k) + page * a.c.ld_block + head * a.c.ld_head + t * a.c.ld_token;
            Run u, w;
#pragma unroll
            for (int i = 0; i < E; ++i) u[i] = (_Float16)v[i], w[i] = (_Float16)v[E + i];
            if (live && (is_q || stored)) {
                *(Run *)(dst + at_lo) = u;
                *(Run *)(dst + at_hi) = w;
            }
            continue;
        }
        if constexpr (kInt8) {
            float top = 0.0f;
#pragma unroll
            for (int i = 0; i < 2 * E; ++i) top = fmaxf(top, fabsf(v[i]));
            top = group_max(top, P);
            if (!stored) continue;
            const float inv = top > 0.0f ? 127.0f / top : 0.0f;
            char *const dst = (is_v ? a.c.v : a.c.k) + page * a.c.ld_block + head * a.c.ld_head + t * a.c.ld_token;
            uint32_t w[2 * E];
#pragma unroll
            for (int i = 0; i < 2 * E; ++i) w[i] = quant_word(v[i], inv, 127.0f);
            if (live) {
#pragma unroll
                for (int i = 0; i < E; i += 4) {
                    *(uint32_t *)(dst + at_lo + i) = pack_low_bytes(w[i], w[i + 1], w[i + 2], w[i + 3]);
                    *(uint32_t *)(dst + at_hi + i) = pack_low_bytes(w[E + i], w[E + i + 1], w[E + i + 2], w[E + i + 3]);
                }
                if (unit == 0) (is_v ? a.c.v_scale : a.c.k_scale)[((long long)page * Hkv + head) * (1 << shift) + t] = top / 127.0f;
            }
        }
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

template <int E, int kHeadsOf>
static hipError_t launch_append(const AppendArgs &a, int P, bool int8, bool interleaved, hipStream_t s)
{
    const int heads = a.n_heads + 2 * a.c.n_kv_heads, slots_of = (heads + kHeadsOf - 1) / kHeadsOf;
    const unsigned long long groups = (unsigned long long)a.M * slots_of, wgs = (groups + 256 / P - 1) / (256 / P);
    if (wgs * (256 / P) > 0xffffffffull || wgs > 0x7fffffffull) return hipErrorInvalidValue;
    const dim3 grid((unsigned)wgs);
    if constexpr (E == 8)
        if (interleaved)
            return int8 ? launch_kernel(k_kv_append<true, true, E, kHeadsOf>, grid, dim3(256), 0, s, a, P, slots_of)
                        : launch_kernel(k_kv_append<false, true, E, kHeadsOf>, grid, dim3(256), 0, s, a, P, slots_of);
    return int8 ? launch_kernel(k_kv_append<true, false, E, kHeadsOf>, grid, dim3(256), 0, s, a, P, slots_of)
                : launch_kernel(k_kv_append<false, false, E, kHeadsOf>, grid, dim3(256), 0, s, a, P, slots_of);
}

hipError_t kv_prepare()
{
    hipFuncAttributes at;
    return hipFuncGetAttributes(&at, (const void *)k_kv_gather<false>);
}

hipError_t launch_kv_append(const AppendArgs &a, bool int8, bool interleaved, hipStream_t s)
{
    // runs of 8 unless halves of the rotated dimensions are not whole runs (interleaved pairs stand inside a run)
    const int E = interleaved || a.rot_dim % 16 == 0 ? 8 : 4;
    int P = 1;
    while (P * 2 * E < a.c.head_dim) P *= 2;
    // one head to a lane while that does not fill the chip (64 tokens of 48 heads with 8-bit codes: 5.4 us with the read-back,
    // 6.9 with four), then four (8192 tokens: 40.3 us, 50.3 with one)
    const bool many = (long long)a.M * (a.n_heads + 2 * a.c.n_kv_heads) * P > 1 << 18;
    if (E == 8) return many ? launch_append<8, 4>(a, P, int8, interleaved, s) : launch_append<8, 1>(a, P, int8, interleaved, s);
    return many ? launch_append<4, 4>(a, P, int8, false, s) : launch_append<4, 1>(a, P, int8, false, s);
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
