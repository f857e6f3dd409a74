// Pages and tokens moved within the paged cache: copies of pages (k_kv_copy), and the accepted nodes of drafted trees to the
// front of their sequences' new tokens (k_kv_compact).
//
// Both only move data, and memory bounds them, or a launch.  A page is rows of head_dim elements, which form longer runs where strides
// allow it; a workgroup has a part of a page's keys or values, 16 bytes a lane.  A tree's accepted nodes of one head are
// read whole before any is written, since a node may stand where another one goes.
//
// 4096 pages of 8 heads of 128 and 32 tokens: 218 us, 4.9 TB/s of the 5.2 that a copy of 1 GiB reaches, four loads of a thread on their way. One page: 6.6
// us, 3.6 of them the kernel; 64 trees, 7 nodes each: 8.7 us, 3.8 the kernel (host and launch the rest).
#include "muxq_block_kernels.h"

#include <algorithm>

namespace muxq {
namespace {

constexpr int kThreads = 256, kEach = 4;          // 16-byte pieces that a thread of a copy has on their way

// A page in 16-byte pieces: `outer` times `inner` runs of `run` pieces, strides in bytes.
struct Shape {
    uint32_t run, inner, pieces;
    long long ld_outer, ld_inner, ld_block;
};

__global__ __launch_bounds__(kThreads) void k_kv_copy(const int32_t *src, const int32_t *dst, KvView c, Shape p, uint32_t parts, uint32_t scales)
{
    const uint32_t pair = blockIdx.x / parts, part = blockIdx.x - pair * parts;
    const int from = src[pair], to = dst[pair];
    if (from < 0 || from >= c.n_blocks || to < 0 || to >= c.n_blocks || from == to) return;
    const uint32_t data = parts - scales;           // parts of keys and values; then those of scales
    if (part >= data) {
        const uint32_t per = ((uint32_t)c.n_kv_heads << c.block_shift) / 4;       // pieces of a page's scales
        for (uint32_t i = (part - data) * kThreads + threadIdx.x; i < 2 * per; i += scales * kThreads) {
            float *const x = i < per ? c.k_scale : c.v_scale;
            const uint32_t e = (i < per ? i : i - per) * 4;
            *(uint4 *)(x + (long long)to * per * 4 + e) = *(const uint4 *)(x + (long long)from * per * 4 + e);
        }
        return;
    }
    char *const base = (part & 1) ? c.v : c.k;
    const char *const in = base + from * p.ld_block;
    char *const out = base + to * p.ld_block;
    uint4 x[kEach];
    long long at[kEach];
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const uint32_t i = ((part >> 1) * kEach + j) * kThreads + threadIdx.x;
        at[j] = -1;
        if (i < p.pieces) {
            const uint32_t run = i / p.run, o = run / p.inner;
            at[j] = o * p.ld_outer + (run - o * p.inner) * p.ld_inner + (long long)(i - run * p.run) * 16;
            x[j] = *(const uint4 *)(in + at[j]);
        }
    }
#pragma unroll
    for (int j = 0; j < kEach; ++j)
        if (at[j] >= 0) *(uint4 *)(out + at[j]) = x[j];
}

template <int kBytes>
__global__ __launch_bounds__(kThreads) void k_kv_compact(CompactArgs a)
{
    extern __shared__ __align__(16) uint4 sh_rows[];         // [node][pieces of a head]
    __shared__ long long sh_from[kMaxNodes], sh_to[kMaxNodes], sh_scale_from[kMaxNodes], sh_scale_to[kMaxNodes];
    __shared__ float sh_scale[kMaxNodes];
    const int s = blockIdx.y, tid = threadIdx.x, kvh = blockIdx.x >> 1, d = a.c.head_dim, shift = a.c.block_shift;
    const int first = max(0, min(a.starts[s], a.M)), n = max(0, min(a.starts[s + 1], a.M)) - first;
    if (n < 1 || n > a.max_nodes) return;
    const int count = min(a.counts[s], n);
    const long long ctx = (long long)a.lengths[s] - n, room = (long long)a.ld_table << shift;
    if (tid < count) {
        const int x = a.path[first + tid];
        const long long from = ctx + x, to = ctx + tid;
        long long at[2] = {-1, -1}, at_scale[2] = {-1, -1};
        if (x >= 0 && x < n && x != tid && ctx >= 0 && from < room && to < room) {
            const int page[2] = {a.table[(long long)s * a.ld_table + (from >> shift)], a.table[(long long)s * a.ld_table + (to >> shift)]};
            if (page[0] >= 0 && page[0] < a.c.n_blocks && page[1] >= 0 && page[1] < a.c.n_blocks) {
                const int mask = (1 << shift) - 1, in[2] = {(int)from & mask, (int)to & mask};
                for (int i = 0; i < 2; ++i) {
                    at[i] = (page[i] * a.c.ld_block + kvh * a.c.ld_head + in[i] * a.c.ld_token) * kBytes;
                    at_scale[i] = (((long long)page[i] * a.c.n_kv_heads + kvh) << shift) + in[i];
                }
            }
        }
        sh_from[tid] = at[0];
        sh_to[tid] = at[1];
        sh_scale_from[tid] = at_scale[0];
        sh_scale_to[tid] = at_scale[1];
    }
    __syncthreads();
    char *const base = (blockIdx.x & 1) ? a.c.v : a.c.k;
    const int per = d * kBytes / 16;
    for (int i = tid; i < count * per; i += kThreads) {
        const int j = i / per;
        if (sh_from[j] >= 0) sh_rows[i] = *(const uint4 *)(base + sh_from[j] + (i - j * per) * 16);
    }
    float *const scale = (blockIdx.x & 1) ? a.c.v_scale : a.c.k_scale;
    if (kBytes == 1 && tid < count && sh_from[tid] >= 0) sh_scale[tid] = scale[sh_scale_from[tid]];
    __syncthreads();
    for (int i = tid; i < count * per; i += kThreads) {
        const int j = i / per;
        if (sh_from[j] >= 0) *(uint4 *)(base + sh_to[j] + (i - j * per) * 16) = sh_rows[i];
    }
    if (kBytes == 1 && tid < count && sh_from[tid] >= 0) scale[sh_scale_to[tid]] = sh_scale[tid];
}

}  // namespace

hipError_t pages_prepare()
{
    hipFuncAttributes at;
    return hipFuncGetAttributes(&at, (const void *)k_kv_copy);
}

hipError_t launch_kv_copy(const int32_t *src, const int32_t *dst, int n, const KvView &c, bool int8, hipStream_t s)
{
    const long long bytes = int8 ? 1 : 2, bs = 1ll << c.block_shift;
    // runs of a page, the shorter stride inside
    const bool heads_inside = c.n_kv_heads > 1 && c.ld_head < c.ld_token;
    long long inner = heads_inside ? c.n_kv_heads : bs, outer = heads_inside ? bs : c.n_kv_heads;
    const long long ld_inner = heads_inside ? c.ld_head : c.ld_token, ld_outer = heads_inside ? c.ld_token : c.ld_head;
    long long run = c.head_dim;
    if (ld_inner == run) {
        run *= inner;
        inner = 1;
        if (outer == 1 || ld_outer == run) run *= outer, outer = 1;
    }
    const long long pieces = (long long)c.n_kv_heads * bs * c.head_dim * bytes / 16;
    const long long data = 2 * ((pieces + kThreads * kEach - 1) / (kThreads * kEach));
    const long long scales = int8 ? std::min((c.n_kv_heads * bs / 2 + kThreads - 1) / kThreads, 64ll) : 0;
    const long long parts = data + scales;
    const Shape p{(uint32_t)(run * bytes / 16), (uint32_t)inner, (uint32_t)pieces, ld_outer * bytes, ld_inner * bytes, c.ld_block * bytes};
    // grids of at most 2^31 threads (a page has fewer than 2^20 parts)
    const int at_once = (int)((1ll << 23) / parts);
    for (int at = 0; at < n; at += at_once) {
        const hipError_t e = launch_kernel(k_kv_copy, dim3((unsigned)(std::min(n - at, at_once) * parts)), dim3(kThreads), 0, s, src + at, dst + at,
                                           c, p, (uint32_t)parts, (uint32_t)scales);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_kv_compact(const CompactArgs &a, bool int8, hipStream_t s)
{
    const dim3 grid(2 * a.c.n_kv_heads, a.S);
    const size_t lds = (size_t)a.max_nodes * a.c.head_dim * (int8 ? 1 : 2);
    return int8 ? launch_kernel(k_kv_compact<1>, grid, dim3(kThreads), lds, s, a) : launch_kernel(k_kv_compact<2>, grid, dim3(kThreads), lds, s, a);
}

}  // namespace muxq
