// The norms around the residual stream, with the column maxima for the next quantised layer.
//
// Each element is read once and written once: X and R in, the stream and Y out, 8 bytes a channel and token.  A
// row stays in the registers of its W waves in binary32 from the first load to the last store, both means of
// both norms taken from there (the mean first, then the squares of what is left: no cancellation).  Prompts
// have a wave a row; few rows, or long ones, four waves each, 16 beyond 8192 channels, so that a lane has few
// elements and its loads go out together.
// Column maxima: every wave keeps those of the rows it writes; a workgroup's go to the scratch and a second launch folds
// them.  Up to 64 rows their magnitudes are the maxima, and there is one launch.
// Measured (kernel trace): 24 x 1280 3.4 us, 16384 x 1280 with both norms, a gate and the maxima 41 us, of which the rows take 36 (4.6 TB/s).
#include "muxq_block_kernels.h"

namespace muxq {
namespace {

constexpr int kMaxGroups = 512;             // workgroups that leave maxima

// The value of another lane of the same 16, without LDS.
template <int kCtrl>
__device__ __forceinline__ float dpp(float v)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), kCtrl, 0xf, 0xf, false));
}

template <int W>
__device__ __forceinline__ float row_sum(float v, float *sh, int &turn)
{
    v += dpp<0xB1>(v);          // lanes xor 1, xor 2, then the other half of 8, of 16
    v += dpp<0x4E>(v);
    v += dpp<0x141>(v);
    v += dpp<0x140>(v);
    v += __shfl_xor(v, 16, 64);
    v += __shfl_xor(v, 32, 64);
    if constexpr (W > 1) {                  // two buffers in turn: one barrier a sum
        float *const s = sh + (turn ^= W);
        if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int w = 0; w < W; ++w) v += s[w];
    }
    return v;
}

// W waves to a row, C runs of 8 channels to a lane; a workgroup of kWaves waves has kWaves / W rows at a time.
template <int W, int C, bool kRms>
__global__ __launch_bounds__(64 * (W == 1 ? 8 : W)) void k_norm(NormArgs n, uint16_t *maxima)
{
    constexpr int kWaves = W == 1 ? 8 : W, kRows = kWaves / W;
    __shared__ float sh[2 * W];
    extern __shared__ __align__(16) char lds[];
    const int tid = threadIdx.x, t = W == 1 ? tid & 63 : tid;
    const float by_k = 1.0f / (float)n.K;
    int turn = 0;
    bool there[C];
    int at[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        at[c] = (c * 64 * W + t) * 8;
        there[c] = at[c] < n.K;
    }
    uint4 most[C] = {};
    float v[C][8];

    // (the vectors of weights come from L1 for each row: in registers they cost more waves than they save loads)
    auto normed = [&](const _Float16 *w, const _Float16 *b) {
        f16x8 ww[C], bb[C];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            ww[c] = bb[c] = f16x8{};
            if (there[c]) {
                ww[c] = *(const f16x8 *)(w + at[c]);
                if (b) bb[c] = *(const f16x8 *)(b + at[c]);
            }
        }
        float mean = 0.0f;
        if (!kRms) {
            float s = 0.0f;
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) s += v[c][i];
            mean = row_sum<W>(s, sh, turn) * by_k;
        }
        float q = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[c][i] = there[c] ? v[c][i] - mean : 0.0f;
                q = __builtin_fmaf(v[c][i], v[c][i], q);
            }
        const float inv = 1.0f / sqrtf(row_sum<W>(q, sh, turn) * by_k + n.eps);
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[c][i] = __builtin_fmaf(v[c][i] * inv, (float)ww[c][i], (float)bb[c][i]);
    };

    const int step = gridDim.x * kRows;
    for (int m = blockIdx.x * kRows + (W == 1 ? tid >> 6 : 0); m < n.M; m += step) {
        f16x8 r[C], gate[C];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            f16x8 x = {};
            r[c] = gate[c] = f16x8{};
            if (there[c]) {
                x = *(const f16x8 *)(n.x + (long long)m * n.ldx + at[c]);
                if (n.res) r[c] = *(const f16x8 *)(n.res + (long long)m * n.ldr + at[c]);
                if (n.gate) gate[c] = *(const f16x8 *)(n.gate + (long long)m * n.ldg + at[c]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) v[c][i] = (float)x[i];
        }
        if (n.post_w) normed(n.post_w, n.post_b);
        if (n.gate) {
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) v[c][i] *= (float)gate[c][i];
        }
        if (n.res) {
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) v[c][i] = __builtin_fmaf(n.r_scale, (float)r[c][i], v[c][i]);
        }
        if (n.r_out) {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                f16x8 o;
#pragma unroll
                for (int i = 0; i < 8; ++i) o[i] = (_Float16)v[c][i];
                if (there[c]) *(f16x8 *)(n.r_out + (long long)m * n.ldro + at[c]) = o;
            }
        }
        normed(n.w, n.b);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            f16x8 o;
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = (_Float16)v[c][i];
            const uint4 bits = __builtin_bit_cast(uint4, o);
            if (there[c]) {
                *(uint4 *)(n.y + (long long)m * n.ldy + at[c]) = bits;
                most[c] = absmax_step(most[c], bits);
            }
            if (n.slabs != nullptr && maxima == nullptr && at[c] < n.k_pad)       // few rows: each a row of maxima
                *(uint4 *)(n.slabs + (long long)m * n.k_pad + at[c]) = there[c] ? absmax_step(uint4{0, 0, 0, 0}, bits) : uint4{0, 0, 0, 0};
        }
    }
    if (maxima != nullptr) {
        uint16_t *const row = maxima + (long long)blockIdx.x * n.k_pad;
        if constexpr (W == 1) {
            uint4 *const top = (uint4 *)lds;                     // [8 waves][64 C]
#pragma unroll
            for (int c = 0; c < C; ++c) top[(tid >> 6) * 64 * C + c * 64 + t] = most[c];
            __syncthreads();
            for (int i = tid; i < 64 * C && i * 8 < n.k_pad; i += 512) {
                uint4 x = top[i];
#pragma unroll
                for (int y = 1; y < 8; ++y) x = absmax_step(x, top[y * 64 * C + i]);
                *(uint4 *)(row + i * 8) = x;
            }
        } else {
#pragma unroll
            for (int c = 0; c < C; ++c)
                if (at[c] < n.k_pad) *(uint4 *)(row + at[c]) = most[c];
        }
    }
}

// Rows of maxima folded into one: 4 runs of 8 channels (64 bytes) to a workgroup, 64 threads down each.
__global__ __launch_bounds__(256) void k_norm_fold(const uint16_t *maxima, int rows, int k_pad, uint16_t *slab)
{
    __shared__ uint4 top[4][4];
    const int run = threadIdx.x & 3, c = (blockIdx.x * 4 + run) * 8;      // (k_pad is a multiple of 64)
    const uint16_t *const p = maxima + c;
    uint4 x = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < kMaxGroups / 64; ++i) {
        const int m = (threadIdx.x >> 2) + 64 * i;
        if (m < rows) x = absmax_step(x, *(const uint4 *)(p + (long long)m * k_pad));
    }
    for (int y = 4; y < 64; y <<= 1) {
        const uint4 o = {(uint32_t)__shfl_xor((int)x.x, y, 64), (uint32_t)__shfl_xor((int)x.y, y, 64), (uint32_t)__shfl_xor((int)x.z, y, 64),
                         (uint32_t)__shfl_xor((int)x.w, y, 64)};
        x = absmax_step(x, o);
    }
    if ((threadIdx.x & 63) < 4) top[threadIdx.x >> 6][run] = x;
    __syncthreads();
    if (threadIdx.x < 4) {
#pragma unroll
        for (int w = 1; w < 4; ++w) x = absmax_step(x, top[w][run]);
        *(uint4 *)(slab + c) = x;
    }
}

// Waves to a row.  us in a graph, inputs in the memory-side cache, one and four: 24 x 1280 3.5 / 2.6, 64 x 768 3.0 / 2.6, 256 x 1280
// 6.2 / 6.3, 1024 x 768 6.3 / 9.1, 16384 x 1280 33.3 / 54.5, 4096 x 1536 14.7 / 18.1, 4096 x 2048 (32 channels a lane) 20.4 / 19.2.
int waves_of(int M, int K) { return K > 8192 ? 16 : K > 1536 || M <= 64 ? 4 : 1; }

int groups_of(int M, int K)
{
    const int rows = waves_of(M, K) == 1 ? 8 : 1, need = (M + rows - 1) / rows;
    return need < kMaxGroups ? need : kMaxGroups;
}

template <int W, int C>
hipError_t launch(const NormArgs &n, bool rms, uint16_t *maxima, hipStream_t s)
{
    const dim3 grid(maxima ? groups_of(n.M, n.K) : W == 1 ? (n.M + 7) / 8 : n.M), block(64 * (W == 1 ? 8 : W));
    const size_t lds = W == 1 && maxima ? (size_t)8 * 64 * C * 16 : 0;
    return rms ? launch_kernel(k_norm<W, C, true>, grid, block, lds, s, n, maxima) : launch_kernel(k_norm<W, C, false>, grid, block, lds, s, n, maxima);
}

}  // namespace

int norm_slab_rows(int M) { return M <= 64 ? M : 1; }

size_t norm_scratch_bytes(int M, int K, int k_pad) { return M <= 64 ? 0 : (size_t)groups_of(M, K) * k_pad * 2; }

hipError_t norm_prepare()
{
    hipFuncAttributes at;
    return hipFuncGetAttributes(&at, (const void *)k_norm_fold);
}

hipError_t launch_norm(const NormArgs &n, bool rms, hipStream_t s)
{
    uint16_t *const maxima = n.slabs && n.M > 64 ? n.scratch : nullptr;
    const int W = waves_of(n.M, n.K), C = (n.k_pad + 512 * W - 1) / (512 * W);
    hipError_t e;
    if (W == 1)
        e = C == 1 ? launch<1, 1>(n, rms, maxima, s) : C == 2 ? launch<1, 2>(n, rms, maxima, s) : launch<1, 3>(n, rms, maxima, s);
    else if (W == 4)
        e = C == 1 ? launch<4, 1>(n, rms, maxima, s) : C == 2 ? launch<4, 2>(n, rms, maxima, s) : C == 3 ? launch<4, 3>(n, rms, maxima, s) : launch<4, 4>(n, rms, maxima, s);
    else
        e = C <= 2 ? launch<16, 2>(n, rms, maxima, s) : launch<16, 4>(n, rms, maxima, s);
    if (e != hipSuccess || maxima == nullptr) return e;
    return launch_kernel(k_norm_fold, dim3(n.k_pad / 32), dim3(256), 0, s, maxima, groups_of(n.M, n.K), n.k_pad, n.slabs);
}

}  // namespace muxq
