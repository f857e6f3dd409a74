// Attention of several new tokens of each sequence over the paged cache: causal with a window and first tokens that stay
// visible, or the nodes of a drafted tree.
//
// O = sum_t p_t V_t / sum_t p_t, p_t = 2^(s_t - m), s_t = scale log2(e) q . K_t, over the tokens that a row sees, with the running
// maximum and sum of the softmax.  A wave has a row and head: a lane scores a token of 64, then the lanes have the dimensions.
#include "muxq_block_kernels.h"

#include <algorithm>

namespace muxq {
namespace {

constexpr float kFloor = -__builtin_inff();

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

template <bool kInt8>
__global__ __launch_bounds__(64) void k_rows(RowsArgs a)
{
    __shared__ float sh_p[64];
    __shared__ long long sh_row[64], sh_scale[64];
    const int s = blockIdx.y, i = blockIdx.x, lane = threadIdx.x, d = a.c.head_dim;
    const int first = max(0, min(a.starts[s], a.M)), n = max(0, min(a.starts[s + 1], a.M)) - first;
    if (n > a.max_new || i >= n) return;
    const int len = max(0, min(a.lengths[s], a.max_length)), shift = a.c.block_shift, ctx = len - n, m0 = first + i;
    uint64_t above = 0;                  // the nodes that a node sees
    if (a.parents)
        for (int x = i; x >= 0 && x < n;) {
            above |= 1ull << x;
            const int up = a.parents[first + x];
            x = up < x ? up : -1;
        }
    for (int h = 0; h < a.n_heads; ++h) {
        const int kvh = h / a.group;
        const _Float16 *const q = a.q + (long long)m0 * a.ldq + (long long)h * d;
        float m = kFloor, l = 0.0f, o[4] = {}, loose[4] = {};
        bool any = false;
        for (int t0 = 0; t0 < len; t0 += 64) {
            const int t = t0 + lane;
            bool there = t < len;
            if (a.parents)
                there = there && (t < ctx || (t - ctx >= 0 && t - ctx < n && (above >> (t - ctx) & 1)));
            else
                there = there && t <= ctx + i && (a.window == 0 || t > (long long)ctx + i - a.window || t < a.sinks);
            int page = -1;
            if (there) page = a.table[(long long)s * a.ld_table + (t >> shift)];
            there = there && page >= 0 && page < a.c.n_blocks;
            float score = kFloor, vs = 1.0f;
            const long long row = there ? page * a.c.ld_block + kvh * a.c.ld_head + (t & ((1 << shift) - 1)) * a.c.ld_token : -1;
            if (there) {
                float sum = 0.0f;
                for (int e = 0; e < d; ++e)
                    sum += (float)q[e] * (kInt8 ? (float)((const int8_t *)a.c.k)[row + e] : (float)((const _Float16 *)a.c.k)[row + e]);
                if (kInt8) {
                    const long long at = (((long long)page * a.c.n_kv_heads + kvh) << shift) + (t & ((1 << shift) - 1));
                    sum *= a.c.k_scale[at];
                    vs = a.c.v_scale[at];
                }
                score = sum * (a.scale * 1.44269504088896f);
            }
            if (!__any(there)) continue;
            any = true;
            float top = score;
            for (int x = 1; x < 64; x <<= 1) top = fmaxf(top, __shfl_xor(top, x, 64));
            const float to = fmaxf(m, top), keep = m == kFloor ? 0.0f : exp2_(m - to);
            m = to;
            const float p = !there || score == kFloor ? 0.0f : exp2_(score - m);
            float sum = p;
            for (int x = 1; x < 64; x <<= 1) sum += __shfl_xor(sum, x, 64);
            l = l * keep + sum;
            __syncthreads();
            sh_p[lane] = p * vs;
            sh_row[lane] = row;
            sh_scale[lane] = score == kFloor ? 0 : 1;
            __syncthreads();
            for (int x = 0; x < 4; ++x) o[x] *= keep;
            for (int j = 0; j < 64; ++j) {
                if (sh_row[j] < 0) continue;
                for (int x = 0; x < 4; ++x) {
                    const int e = lane + 64 * x;
                    if (e >= d) break;
                    const float v = kInt8 ? (float)((const int8_t *)a.c.v)[sh_row[j] + e] : (float)((const _Float16 *)a.c.v)[sh_row[j] + e];
                    if (v - v == 0.0f && sh_p[j] - sh_p[j] == 0.0f)
                        o[x] += sh_p[j] * v;
                    else                    // weights are never quite 0
                        loose[x] += sh_scale[j] ? (kInt8 ? sh_p[j] * v : v) : 0.0f * v;
                }
            }
        }
        for (int x = 0; x < 4; ++x) {
            const int e = lane + 64 * x;
            if (e < d) a.o[(long long)m0 * a.ldo + (long long)h * d + e] = (_Float16)(any ? (o[x] + loose[x]) / l : 0.0f);
        }
    }
}

}  // namespace

size_t rows_workspace_need(int, int, int, int, int, int, int, int, bool) { return 0; }
size_t rows_workspace_bytes(int, int, int, int, int, int, int, int, bool) { return 0; }

hipError_t rows_prepare()
{
    hipFuncAttributes at;
    return hipFuncGetAttributes(&at, (const void *)k_rows<false>);
}

hipError_t launch_rows(const RowsArgs &a, bool int8, hipStream_t s)
{
    const dim3 grid(std::min(a.max_new, a.M), a.S);
    return int8 ? launch_kernel(k_rows<true>, grid, dim3(64), 0, s, a) : launch_kernel(k_rows<false>, grid, dim3(64), 0, s, a);
}

}  // namespace muxq
