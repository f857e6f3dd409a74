// Low-rank adapters of many requests beside a shared projection.
#include "muxq_block_kernels.h"

namespace muxq {
namespace {

// One workgroup to a row: which request it belongs to, its r products with A, then the row of the output.
__global__ __launch_bounds__(256) void k_lora(LoraArgs g)
{
    __shared__ float h[128];
    const int m = blockIdx.x, tid = threadIdx.x;
    int lo = 0, hi = g.n_requests;                       // the last request that starts at or before m
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        (g.starts[mid] <= m ? lo : hi) = mid;
    }
    if (m < g.starts[lo] || m >= g.starts[lo + 1]) return;
    const int ad = g.adapters[lo];
    const bool has = ad >= 0 && ad < g.n_adapters;
    const _Float16 *y = g.y + (long long)m * g.ldy;
    _Float16 *out = g.out + (long long)m * g.ldo;
    if (!has) {
        for (int n = tid * 8; n < g.N; n += 2048) *(f16x8 *)(out + n) = *(const f16x8 *)(y + n);
        return;
    }
    const _Float16 *x = g.x + (long long)m * g.ldx;
    for (int j = tid >> 6; j < g.r; j += 4) {
        const _Float16 *a = g.a + ((long long)ad * g.r + j) * g.K;
        float v = 0.0f;
        for (int k = tid & 63; k < g.K; k += 64) v += (float)x[k] * (float)a[k];
        for (int i = 1; i < 64; i <<= 1) v += __shfl_xor(v, i, 64);
        if ((tid & 63) == 0) h[j] = v * g.scales[ad];
    }
    __syncthreads();
    for (int n = tid; n < g.N; n += 256) {
        const _Float16 *b = g.b + ((long long)ad * g.N + n) * g.r;
        float v = 0.0f;
        for (int j = 0; j < g.r; ++j) v += h[j] * (float)b[j];
        out[n] = (_Float16)((float)y[n] + v);
    }
}

}  // namespace

hipError_t launch_lora(const LoraArgs &g, hipStream_t s)
{
    return launch_kernel(k_lora, dim3(g.M), dim3(256), 0, s, g);
}

}  // namespace muxq
