// The norms around the residual stream, with the column maxima for the next quantised layer.
#include "muxq_block_kernels.h"

namespace muxq {
namespace {

__device__ float block_sum(float v, float *sh)
{
    for (int x = 1; x < 64; x <<= 1) v += __shfl_xor(v, x, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
    __syncthreads();
    return (sh[0] + sh[1]) + (sh[2] + sh[3]);
}

// One workgroup to a row, a thread every 256th channel; the row stays in LDS in binary32.
template <bool kRms>
__device__ void norm_row(float *row, int K, const _Float16 *w, const _Float16 *b, float eps, float *sh)
{
    float mean = 0.0f;
    if (!kRms) {
        float s = 0.0f;
        for (int k = threadIdx.x; k < K; k += 256) s += row[k];
        mean = block_sum(s, sh) / K;
    }
    float q = 0.0f;
    for (int k = threadIdx.x; k < K; k += 256) q += (row[k] - mean) * (row[k] - mean);
    const float inv = 1.0f / sqrtf(block_sum(q, sh) / K + eps);
    for (int k = threadIdx.x; k < K; k += 256) row[k] = (row[k] - mean) * inv * (float)w[k] + (b ? (float)b[k] : 0.0f);
}

template <bool kRms>
__global__ __launch_bounds__(256) void k_norm(NormArgs n)
{
    extern __shared__ float row[];
    __shared__ float sh[4];
    const int m = blockIdx.x;
    for (int k = threadIdx.x; k < n.K; k += 256) row[k] = (float)n.x[(long long)m * n.ldx + k];
    if (n.post_w) norm_row<kRms>(row, n.K, n.post_w, n.post_b, n.eps, sh);
    for (int k = threadIdx.x; k < n.K; k += 256) {
        float t = row[k];
        if (n.gate) t *= (float)n.gate[(long long)m * n.ldg + k];
        if (n.res) t = n.r_scale * (float)n.res[(long long)m * n.ldr + k] + t;
        row[k] = t;
    }
    if (n.r_out)
        for (int k = threadIdx.x; k < n.K; k += 256) n.r_out[(long long)m * n.ldro + k] = (_Float16)row[k];
    norm_row<kRms>(row, n.K, n.w, n.b, n.eps, sh);
    for (int k = threadIdx.x; k < n.K; k += 256) n.y[(long long)m * n.ldy + k] = (_Float16)row[k];
}

__global__ __launch_bounds__(256) void k_maxima(const uint16_t *y, int rows, int K, int ldy, int k_pad, uint16_t *slabs)
{
    const int k = blockIdx.x * 256 + threadIdx.x;
    if (k >= k_pad) return;
    uint16_t top = 0;
    if (k < K)
        for (int m = blockIdx.y * rows; m < (blockIdx.y + 1) * rows; ++m) top = max(top, (uint16_t)(y[(long long)m * ldy + k] & 0x7fff));
    slabs[(long long)blockIdx.y * k_pad + k] = top;
}

}  // namespace

int norm_slab_rows(int M) { return M <= 64 ? M : 1; }

size_t norm_scratch_bytes(int, int, int) { return 0; }

hipError_t launch_norm(const NormArgs &n, bool rms, hipStream_t s)
{
    const size_t lds = (size_t)n.K * 4;
    hipError_t e;
    if (lds > 60 * 1024) {
        if ((e = hipFuncSetAttribute((const void *)(rms ? k_norm<true> : k_norm<false>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds)) != hipSuccess)
            return e;
    }
    e = rms ? launch_kernel(k_norm<true>, dim3(n.M), dim3(256), lds, s, n) : launch_kernel(k_norm<false>, dim3(n.M), dim3(256), lds, s, n);
    if (e != hipSuccess || n.slabs == nullptr) return e;
    const int rows = norm_slab_rows(n.M);
    return launch_kernel(k_maxima, dim3((n.k_pad + 255) / 256, rows), dim3(256), 0, s, (const uint16_t *)n.y, n.M / rows, n.K, n.ldy, n.k_pad, n.slabs);
}

}  // namespace muxq
