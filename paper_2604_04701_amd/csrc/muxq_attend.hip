// Attention of one new token over the paged cache.
#include "muxq_block_kernels.h"

namespace muxq {
namespace {

// One workgroup to a sequence and head: 256 tokens at a time, a thread the score of one, then the running
// maximum and sum of the softmax, then a thread one dimension of the weighted sum.
template <bool kInt8>
__global__ __launch_bounds__(256) void k_attend(AttendArgs a)
{
    __shared__ float sh_q[256], sh_p[256], sh_red[4];
    __shared__ long long sh_at[256];
    const int s = blockIdx.y, h = blockIdx.x, kvh = h / a.group, d = a.c.head_dim, tid = threadIdx.x;
    const int len = min(a.lengths[s], a.max_length), shift = a.c.block_shift;
    if (tid < d) sh_q[tid] = (float)a.q[(long long)s * a.ldq + (long long)h * d + tid];
    float top = -INFINITY, sum = 0.0f, o = 0.0f;
    for (int t0 = 0; t0 < len; t0 += 256) {
        __syncthreads();
        const int t = t0 + tid;
        long long at = -1;
        float score = -INFINITY, vs = 1.0f;
        if (t < len) {
            const int page = a.table[(long long)s * a.ld_table + (t >> shift)], in = t & ((1 << shift) - 1);
            if (page >= 0 && page < a.c.n_blocks) {
                at = page * a.c.ld_block + kvh * a.c.ld_head + in * a.c.ld_token;
                float dot = 0.0f;
                for (int i = 0; i < d; ++i)
                    dot += sh_q[i] * (kInt8 ? (float)((const int8_t *)a.c.k)[at + i] : (float)((const _Float16 *)a.c.k)[at + i]);
                if (kInt8) {
                    const long long sc = ((long long)page * a.c.n_kv_heads + kvh) * (1 << shift) + in;
                    dot *= a.c.k_scale[sc];
                    vs = a.c.v_scale[sc];
                }
                score = dot * a.scale;
            }
        }
        float m = score;
        for (int x = 1; x < 64; x <<= 1) m = fmaxf(m, __shfl_xor(m, x, 64));
        if ((tid & 63) == 0) sh_red[tid >> 6] = m;
        __syncthreads();
        m = fmaxf(fmaxf(fmaxf(sh_red[0], sh_red[1]), fmaxf(sh_red[2], sh_red[3])), top);
        const float p = at < 0 ? 0.0f : expf(score - m);
        const float keep = top == -INFINITY ? 0.0f : expf(top - m);
        float l = p;
        for (int x = 1; x < 64; x <<= 1) l += __shfl_xor(l, x, 64);
        __syncthreads();
        if ((tid & 63) == 0) sh_red[tid >> 6] = l;
        sh_p[tid] = p * vs;
        sh_at[tid] = at;
        __syncthreads();
        sum = sum * keep + ((sh_red[0] + sh_red[1]) + (sh_red[2] + sh_red[3]));
        top = m;
        o *= keep;
        if (tid < d)
            for (int j = 0; j < 256 && t0 + j < len; ++j)
                if (sh_at[j] >= 0)
                    o += sh_p[j] * (kInt8 ? (float)((const int8_t *)a.c.v)[sh_at[j] + tid] : (float)((const _Float16 *)a.c.v)[sh_at[j] + tid]);
    }
    if (tid < d) a.o[(long long)s * a.ldo + (long long)h * d + tid] = (_Float16)(top == -INFINITY ? 0.0f : o / sum);
}

}  // namespace

size_t attend_workspace_bytes(int, int, int, int, int) { return 0; }

hipError_t launch_attend(const AttendArgs &a, bool int8, hipStream_t s)
{
    const dim3 grid(a.n_heads, a.S);
    return int8 ? launch_kernel(k_attend<true>, grid, dim3(256), 0, s, a) : launch_kernel(k_attend<false>, grid, dim3(256), 0, s, a);
}

}  // namespace muxq
