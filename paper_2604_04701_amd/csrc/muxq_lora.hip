// Low-rank adapters of many requests beside a shared projection: out = Y + s (X A^T) B^T by runs of rows.
//
// Both products are thin (r columns, then r deep), so what bounds them is X, Y and out for prompts, and A and B, or
// latency alone, for single tokens.  One launch does both: a workgroup takes a tile of 16 or 32 rows of one
// request and a strip of output channels.  Its 8 waves divide K for H = X A^T (rows of X and of A as they lie
// are the operands of the matrix pipes), add their parts in LDS, and then divide the strip's channels for H B^T,
// with rows of B as the left operand in an order that leaves a lane 16 neighbouring channels of a row of Y.
// H is what several strips of a tile compute again: it costs reads of X and A from the L2s, and saves a second
// launch and the way of H through memory.
// H is binary32; the second product takes it as two fp16 parts (22 bits) of the row over a power of two,
// whatever its size.
#include "muxq_block_kernels.h"

namespace muxq {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 8, kThreads = 64 * kWaves, kCols = 64 * kWaves;      // output channels of a workgroup's step

// First row of request q, whatever the caller's bounds hold.
__device__ __forceinline__ int start_of(const LoraArgs &g, int q) { return min(max(g.starts[q], 0), g.M); }

// kTM: tiles of 16 rows, kRT: tiles of 16 ranks (of the power of two at or above r).
template <int kTM, int kRT>
__global__ __launch_bounds__(kThreads) void k_lora(LoraArgs g, int strip)
{
    constexpr int T = 16 * kTM, R = 16 * kRT, RS = kRT == 1 ? 1 : kRT / 2, LD = R + 4, LH = 32 * RS + 8;
    __shared__ float part[kWaves / 2][T][LD];
    __shared__ __align__(16) _Float16 h_hi[T][LH], h_lo[T][LH];
    __shared__ float factor[T];
    __shared__ int found[kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 15, gr = lane >> 4;

    // Tiles are numbered so that request q has those from starts[q] / T + q on: as many as it can need.  The
    // request of tile b is the last one that starts there or before: every thread looks at one (of R > 512: at
    // one of each so many, then at those in between).
    const int b = blockIdx.x;
    int q = 0;
    for (int step = (g.n_requests + kThreads - 1) / kThreads;;) {
        int count = 0;
        const int span = step > 1 ? kThreads : min(kThreads, g.n_requests - q);
        if (tid < span) {
            const int at = q + tid * step;
            count = at < g.n_requests && start_of(g, at) / T + at <= b;
        }
        const int n = __popcll(__ballot(count));
        if (lane == 0) found[wave] = n;
        __syncthreads();
        int all = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) all += found[w];
        q = min(q + max(all - 1, 0) * step, g.n_requests - 1);
        if (step == 1) break;
        step = (step + kThreads - 1) / kThreads;
        __syncthreads();
    }
    const int first = start_of(g, q), row0 = first + (b - (first / T + q)) * T;
    const int rows = min(T, start_of(g, q + 1) - row0);
    if (rows <= 0 || row0 < first) return;
    const int n0 = blockIdx.y * strip, n1 = min(g.N, n0 + strip);
    const int ad = g.adapters[q];
    const _Float16 *const y = g.y + (long long)row0 * g.ldy;
    _Float16 *const out = g.out + (long long)row0 * g.ldo;
    if (ad < 0 || ad >= g.n_adapters) {
        if (g.y != g.out)
            for (int m = wave; m < rows; m += kWaves)
                for (int n = n0 + lane * 8; n < n1; n += 512) *(f16x8 *)(out + (long long)m * g.ldo + n) = *(const f16x8 *)(y + (long long)m * g.ldy + n);
        return;
    }

    // H: lanes of a 16-lane row read 64 bytes of 16 rows; rows past the tile's last repeat it, ranks past r the last one
    const _Float16 *xr[kTM], *ar[kRT];
#pragma unroll
    for (int t = 0; t < kTM; ++t) xr[t] = g.x + (long long)(row0 + min(16 * t + col, rows - 1)) * g.ldx;
#pragma unroll
    for (int t = 0; t < kRT; ++t) ar[t] = g.a + ((long long)ad * g.r + min(16 * t + col, g.r - 1)) * g.K;
    f32x4 acc[kTM][kRT] = {};
    auto step = [&](auto whole, int k0) {
        f16x8 xv[4][kTM], av[4][kRT];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int k = k0 + 32 * s + 8 * gr;
            const bool there = decltype(whole)::value || k < g.K;
            const int at = there ? k : 0;
#pragma unroll
            for (int t = 0; t < kTM; ++t) xv[s][t] = there ? *(const f16x8 *)(xr[t] + at) : f16x8{};
#pragma unroll
            for (int t = 0; t < kRT; ++t) av[s][t] = there ? *(const f16x8 *)(ar[t] + at) : f16x8{};
        }
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int t = 0; t < kTM; ++t)
#pragma unroll
                for (int u = 0; u < kRT; ++u) acc[t][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(xv[s][t], av[s][u], acc[t][u], 0, 0, 0);
    };
    for (int k0 = wave * 128; k0 < g.K; k0 += 128 * kWaves)
        if (k0 + 128 <= g.K)
            step(std::true_type{}, k0);
        else
            step(std::false_type{}, k0);
    // parts of the upper waves to the lower ones, then all of them to the rows' owners
    auto put = [&](int at) {
#pragma unroll
        for (int t = 0; t < kTM; ++t)
#pragma unroll
            for (int u = 0; u < kRT; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) part[at][16 * t + 4 * gr + i][16 * u + col] = acc[t][u][i];
    };
    if (wave >= kWaves / 2) put(wave - kWaves / 2);
    __syncthreads();
    if (wave < kWaves / 2) {
#pragma unroll
        for (int t = 0; t < kTM; ++t)
#pragma unroll
            for (int u = 0; u < kRT; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[t][u][i] += part[wave][16 * t + 4 * gr + i][16 * u + col];
        put(wave);                                // its own place, read by itself alone
    }
    __syncthreads();
    const float scale = g.scales[ad];
    for (int m = wave; m < T; m += kWaves) {
        constexpr int per = R > 64 ? R / 64 : 1;
        float v[per], top = 0.0f;
#pragma unroll
        for (int i = 0; i < per; ++i) {
            const int j = lane + 64 * i;
            v[i] = 0.0f;
            if (j < g.r) v[i] = (part[0][m][j] + part[1][m][j]) + (part[2][m][j] + part[3][m][j]);
            top = fmaxf(top, fabsf(v[i]));
        }
        for (int x = 1; x < 64; x <<= 1) top = fmaxf(top, __shfl_xor(top, x, 64));
        const uint32_t ex = min(max(__float_as_uint(top) >> 23, 15u), 250u);
        const float up = __uint_as_float((268u - ex) << 23);            // the row's largest to 2^14 .. 2^15
        if (lane == 0) factor[m] = scale * __uint_as_float((ex - 14u) << 23);
#pragma unroll
        for (int i = 0; i < per; ++i) {
            const int j = lane + 64 * i;
            if (j < 32 * RS) {
                const float w = v[i] * up;
                const _Float16 hi = (_Float16)w;
                h_hi[m][j] = hi;
                h_lo[m][j] = (_Float16)(w - (float)hi);
            }
        }
    }
    __syncthreads();

    f16x8 hh[kTM][RS], hl[kTM][RS];
    float f[kTM];
#pragma unroll
    for (int t = 0; t < kTM; ++t) {
        f[t] = factor[16 * t + col];
#pragma unroll
        for (int s = 0; s < RS; ++s) {
            hh[t][s] = *(const f16x8 *)&h_hi[16 * t + col][32 * s + 8 * gr];
            hl[t][s] = *(const f16x8 *)&h_lo[16 * t + col][32 * s + 8 * gr];
        }
    }
    const _Float16 *const br = g.b + (long long)ad * g.N * g.r;
    for (int nb = n0 + wave * 64; nb < n1; nb += kCols) {
        // 64 channels: row m of operand t is channel nb + 16 (m / 4) + 4 t + m % 4, so that a lane ends up with 16 in a row
        // (loads past the tile's rows, the strip's channels or the ranks go to what is there; none of it is stored or counts)
        f16x8 yv[kTM][2];
        const int n = nb + 16 * gr;
#pragma unroll
        for (int t = 0; t < kTM; ++t)
#pragma unroll
            for (int x = 0; x < 2; ++x) yv[t][x] = *(const f16x8 *)(y + (long long)min(16 * t + col, rows - 1) * g.ldy + min(n + 8 * x, n1 - 8));
        f16x8 bv[4][RS];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int nn = min(nb + 16 * (col >> 2) + 4 * u + (col & 3), n1 - 1);
#pragma unroll
            for (int s = 0; s < RS; ++s) {
                const int k = 32 * s + 8 * gr;
                bv[u][s] = *(const f16x8 *)(br + (long long)nn * g.r + (k < g.r ? k : 0));
                if (k >= g.r) bv[u][s] = f16x8{};
            }
        }
        f32x4 o[kTM][4] = {};
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int s = 0; s < RS; ++s)
#pragma unroll
                for (int t = 0; t < kTM; ++t) {
                    o[t][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(bv[u][s], hh[t][s], o[t][u], 0, 0, 0);
                    o[t][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(bv[u][s], hl[t][s], o[t][u], 0, 0, 0);
                }
#pragma unroll
        for (int t = 0; t < kTM; ++t)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                if (16 * t + col >= rows || n + 8 * x >= n1) continue;
                f16x8 r;
#pragma unroll
                for (int i = 0; i < 8; ++i) r[i] = (_Float16)((float)yv[t][x][i] + f[t] * o[t][2 * x + (i >> 2)][i & 3]);
                *(f16x8 *)(out + (long long)(16 * t + col) * g.ldo + n + 8 * x) = r;
            }
    }
}

template <int kTM, int kRT>
hipError_t launch(const LoraArgs &g, hipStream_t s)
{
    // strips: about 512 workgroups, each a step of all its waves at least
    const int tiles = g.M / (16 * kTM) + g.n_requests, steps = (g.N + kCols - 1) / kCols;
    int strips = (512 + tiles - 1) / tiles;
    strips = strips < steps ? strips : steps;
    const int strip = (steps + strips - 1) / strips * kCols;
    return launch_kernel(k_lora<kTM, kRT>, dim3(tiles, (g.N + strip - 1) / strip), dim3(kThreads), 0, s, g, strip);
}

}  // namespace

hipError_t launch_lora(const LoraArgs &g, hipStream_t s)
{
    const bool two = (long long)g.M >= 32ll * g.n_requests;      // prompts: 32 rows share what is read of A and B
    if (g.r <= 16) return two ? launch<2, 1>(g, s) : launch<1, 1>(g, s);
    if (g.r <= 32) return two ? launch<2, 2>(g, s) : launch<1, 2>(g, s);
    if (g.r <= 64) return two ? launch<2, 4>(g, s) : launch<1, 4>(g, s);
    return launch<1, 8>(g, s);
}

}  // namespace muxq
