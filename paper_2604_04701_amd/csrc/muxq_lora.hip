// Low-rank adapters of many requests beside a shared projection: out = Y + s (X A^T) B^T by runs of rows.
//
// Both products are thin (r columns, then r deep), so what bounds them is X, Y and out for prompts, and A and B, or
// latency alone, for single tokens.  One launch does both: a workgroup takes a tile of 16 or 32 rows of one
// request and a strip of output channels.  Its 8 waves divide K for H = X A^T (rows of X and of A as they lie
// are the operands of the matrix pipes), add their parts in LDS, and then divide the strip's channels for H B^T,
// with rows of B as the left operand in an order that leaves a lane 16 neighbouring channels of a row of Y.
// H is what several strips of a tile compute again: it costs reads of X and A from the L2s, and saves a second
// launch and the way of H through memory.  Where it would cost more than that, two launches: the first
// divides K over workgroups too and leaves its parts of H in the workspace, binary32, the second adds them.
// One token 768 -> 2304 at rank 8 4.9 us, 64 requests 1280 -> 3840 at rank 16 9.6 us (kernel trace; each of its 8 strips reads its request's
// A whole, 41 KB, for a row of a tile of 16), 8192 rows 4096 -> 4096 at rank 32 57 us (23 + 35 in two launches, 3.5 TB/s of what has to move).
// H is binary32; the second product takes it as two fp16 parts (22 bits) of the row over a power of two,
// whatever its size.
#include "muxq_block_kernels.h"

#include <algorithm>

namespace muxq {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 8, kThreads = 64 * kWaves, kCols = 64 * kWaves;      // output channels of a workgroup's step
constexpr int kDeep = 64 * kWaves;                                          // channels of X of one

// What this wave wrote to LDS is there for its other lanes.
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// w = hi + lo, hi cut towards zero, so that both have w's sign, and neither is 0 unless w is (`some`: w != 0 before it was scaled;
// 2^-24 is beyond the 38 bits that stand below the row's largest): what an infinity on the other side of the product makes of w it makes of each part,
// where lo = 0, or one of the other sign, would give NaN.  An infinity is both of its parts.
__device__ __forceinline__ void store_parts(float w, bool some, _Float16 &hi_at, _Float16 &lo_at)
{
    const float tiny = some ? copysignf(5.9604645e-8f, w) : 0.0f;
    const _Float16 cut = (_Float16)__builtin_amdgcn_cvt_pkrtz(w, 0.0f)[0];
    const _Float16 hi = cut == (_Float16)0.0f ? (_Float16)tiny : cut;
    const _Float16 rest = (_Float16)(w - (float)cut);
    hi_at = hi;
    lo_at = rest == (_Float16)0.0f ? (_Float16)tiny : (float)cut == w ? hi : rest;
}

// First row of request q, whatever the caller's bounds hold.
__device__ __forceinline__ int start_of(const LoraArgs &g, int q) { return min(max(g.starts[q], 0), g.M); }

enum Part { kBoth, kDown, kUp };

// kTM: tiles of 16 rows, kRT: tiles of 16 ranks (of the power of two at or above r).  piece: what a workgroup in y takes,
// channels of Y, or channels of X in the first of two launches; pieces: of X.  (The pieces of a tile one after the other in the
// grid are up to a sixth slower.)
template <int kTM, int kRT, Part kPart>
__global__ __launch_bounds__(kThreads, kRT == 1 || (kRT == 2 && (kTM == 1 || kPart == kUp)) ? 4 : 2) void k_lora(LoraArgs g, int piece, int pieces)
{
    constexpr int T = 16 * kTM, R = 16 * kRT, RS = kRT == 1 ? 1 : kRT / 2, LD = R + 4, LH = 32 * RS + 8;
    // The operands want 16 rows on neighbouring lanes, which memory gives 16 bytes at a time: with many rows each wave
    // loads whole runs of rows and turns them in a place of its own in LDS (8192 x 4096 at rank 32: half of the requests).
    constexpr bool kTurnDown = kPart != kUp && kTM == 2, kTurnUp = kPart != kDown && kTM == 2 && RS == 1;
    constexpr int kLdDown = 64 + 8, kDownBytes = kTurnDown ? kWaves * 32 * kLdDown * 2 : 0;
    constexpr int kLdUp = 32 + 8, kUpBlock = 16 * kLdUp + 32, kUpBytes = kTurnUp ? kWaves * 4 * kUpBlock * 2 : 0;
    constexpr int kPartBytes = kPart == kUp ? 0 : kWaves / 2 * T * LD * 4;
    constexpr int kBytes = kDownBytes > kUpBytes ? (kDownBytes > kPartBytes ? kDownBytes : kPartBytes) : (kUpBytes > kPartBytes ? kUpBytes : kPartBytes);
    __shared__ __align__(16) char lds[kBytes > 0 ? kBytes : 16];
    float(*const part)[T][LD] = (float(*)[T][LD])lds;
    _Float16 *const turn_down = (_Float16 *)lds + (threadIdx.x >> 6) * (32 * kLdDown);
    _Float16 *const turn_up = (_Float16 *)lds + (threadIdx.x >> 6) * (4 * kUpBlock);
    __shared__ __align__(16) _Float16 h_hi[kPart == kDown ? 1 : T][LH], h_lo[kPart == kDown ? 1 : T][LH];
    __shared__ __align__(16) float factor[T];
    __shared__ int found[kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 15, gr = lane >> 4;

    // Tiles are numbered so that request q has those from starts[q] / T + q on: as many as it can need.  The
    // request of tile b is the last one that starts there or before: every thread looks at one (of R > 512: at
    // one of each so many, then at those in between).
    const int b = blockIdx.x, mine = blockIdx.y;
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
    const int n0 = mine * piece, n1 = min(g.N, n0 + piece);
    const int ad = g.adapters[q];
    const _Float16 *const y = g.y + (long long)row0 * g.ldy;
    _Float16 *const out = g.out + (long long)row0 * g.ldo;
    if (ad < 0 || ad >= g.n_adapters) {
        if (kPart != kDown && g.y != g.out)
            for (int m = wave; m < rows; m += kWaves)
                for (int n = n0 + lane * 8; n < n1; n += 512) *(f16x8 *)(out + (long long)m * g.ldo + n) = *(const f16x8 *)(y + (long long)m * g.ldy + n);
        return;
    }

    // 64 channels of the output: column c of operand u is channel nb + 4 c + u, so that a lane ends up with 4 neighbours of 4 rows and
    // 16 lanes with 128 bytes of a row of Y.  (Loads past the tile's rows, the strip's channels or the ranks go to what is
    // there; none of it is stored or counts.)  The next ones are on their way while these are worked on, the first ones while
    // H is.
    constexpr int NB = kTurnUp ? 4 : 4 * RS;           // loads of a lane: 64 rows of B, at most 64 bytes each, or as operands
    struct Ahead {
        f16x4 y[kTM][4];
        f16x8 b[NB];
    } ahead;
    const _Float16 *const br = g.b + (long long)ad * g.N * g.r;
    const uint32_t per_row = (65536 + (g.r >> 3) - 1) / (g.r >> 3);        // q / (r / 8) is q * this >> 16 for q < 256
    auto ask_up = [&](int nb) {
#pragma unroll
        for (int t = 0; t < kTM; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                ahead.y[t][i] = *(const f16x4 *)(y + (uint32_t)(min(16 * t + 4 * gr + i, rows - 1) * g.ldy + min(nb + 4 * col, n1 - 4)));
        if constexpr (kTurnUp) {
            const int last = (n1 - nb) * g.r - 8;
#pragma unroll
            for (int i = 0; i < NB; ++i) ahead.b[i] = *(const f16x8 *)(br + (long long)nb * g.r + (uint32_t)min((64 * i + lane) * 8, last));
        } else {
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int s = 0; s < RS; ++s) {
                    const int k = 32 * s + 8 * gr;
                    ahead.b[u * RS + s] = *(const f16x8 *)(br + (long long)min(nb + 4 * col + u, n1 - 1) * g.r + (k < g.r ? k : 0));
                }
        }
    };
    int nb = n0 + wave * 64;
    constexpr bool kEarly = kPart == kUp || (kPart == kBoth && kTM == 1 && kRT <= 2);      // (else the first product needs the registers)
    if (kEarly && nb < n1) ask_up(nb);
    const float scale = g.scales[ad];
    if constexpr (kPart != kUp) {
        // H: lanes of a 16-lane row read 64 bytes of 16 rows; rows past the tile's last repeat it, ranks past r the last one
        const _Float16 *xr[kTM], *ar[kRT];
#pragma unroll
        for (int t = 0; t < kTM; ++t) xr[t] = g.x + (long long)(row0 + min(16 * t + col, rows - 1)) * g.ldx;
#pragma unroll
        for (int t = 0; t < kRT; ++t) ar[t] = g.a + ((long long)ad * g.r + min(16 * t + col, g.r - 1)) * g.K;
        f32x4 acc[kTM][kRT] = {};
        // 64 channels at a time, the next ones on their way while these are in the matrix pipes
        constexpr int NX = kTurnDown ? 4 : 2 * kTM, NA = 2 * kRT;          // loads of a lane
        struct Buffer {
            f16x8 x[NX], a[NA];
        } buf[2];
        const int kb = kPart == kDown ? mine * piece : 0, ke = kPart == kDown ? min(g.K, kb + piece) : g.K;
        const int turn_row = lane >> 3, turn_k = (lane & 7) * 8;           // rows of 64 channels, 8 at a time
        auto ask = [&](Buffer &w, int k0) {
            if constexpr (kTurnDown) {
                const int k = k0 + turn_k;
                const bool there = k < g.K;
#pragma unroll
                for (int i = 0; i < NX; ++i) w.x[i] = *(const f16x8 *)(g.x + (long long)(row0 + min(8 * i + turn_row, rows - 1)) * g.ldx + (there ? k : 0));
#pragma unroll
                for (int i = 0; i < NA; ++i)
                    w.a[i] = *(const f16x8 *)(g.a + ((long long)ad * g.r + min(8 * i + turn_row, g.r - 1)) * g.K + (there ? k : 0));
                if (k0 + 64 > g.K && !there) {
#pragma unroll
                    for (int i = 0; i < NX; ++i) w.x[i] = f16x8{};
#pragma unroll
                    for (int i = 0; i < NA; ++i) w.a[i] = f16x8{};
                }
                return;
            }
            const bool whole = k0 + 64 <= g.K;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const int k = k0 + 32 * s + 8 * gr, at = whole || k < g.K ? k : 0;
#pragma unroll
                for (int t = 0; t < kTM; ++t) w.x[s * kTM + t] = *(const f16x8 *)(xr[t] + at);
#pragma unroll
                for (int t = 0; t < kRT; ++t) w.a[s * kRT + t] = *(const f16x8 *)(ar[t] + at);
            }
            if (!whole) {
#pragma unroll
                for (int s = 0; s < 2; ++s)
                    if (k0 + 32 * s + 8 * gr >= g.K) {
#pragma unroll
                        for (int t = 0; t < kTM; ++t) w.x[s * kTM + t] = f16x8{};
#pragma unroll
                        for (int t = 0; t < kRT; ++t) w.a[s * kRT + t] = f16x8{};
                    }
            }
        };
        auto add = [&](const Buffer &w) {
            if constexpr (kTurnDown) {
                f16x8 xv[2][kTM];
                auto turn = [&](const f16x8 *from) {                       // 32 rows through the wave's place
#pragma unroll
                    for (int i = 0; i < 4; ++i) *(f16x8 *)(turn_down + (8 * i + turn_row) * kLdDown + turn_k) = from[i];
                    wave_sync();
                };
                auto turned = [&](int s, int t) { return *(const f16x8 *)(turn_down + (16 * t + col) * kLdDown + 32 * s + 8 * gr); };
                turn(w.x);
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int t = 0; t < kTM; ++t) xv[s][t] = turned(s, t);
                wave_sync();
#pragma unroll
                for (int u0 = 0; u0 < kRT; u0 += 2) {
                    if constexpr (kRT == 1) {
#pragma unroll
                        for (int i = 0; i < 2; ++i) *(f16x8 *)(turn_down + (8 * i + turn_row) * kLdDown + turn_k) = w.a[i];
                        wave_sync();
                    } else {
                        turn(w.a + 2 * u0);
                    }
#pragma unroll
                    for (int s = 0; s < 2; ++s)
#pragma unroll
                        for (int u = 0; u < (kRT == 1 ? 1 : 2); ++u) {
                            const f16x8 av = turned(s, u);
#pragma unroll
                            for (int t = 0; t < kTM; ++t) acc[t][u0 + u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(xv[s][t], av, acc[t][u0 + u], 0, 0, 0);
                        }
                    wave_sync();
                }
                return;
            }
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int t = 0; t < kTM; ++t)
#pragma unroll
                    for (int u = 0; u < kRT; ++u) acc[t][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(w.x[s * kTM + t], w.a[s * kRT + u], acc[t][u], 0, 0, 0);
        };
        int k0 = kb + wave * 64;
        if (k0 < ke) ask(buf[0], k0);
        for (; k0 < ke; k0 += 2 * kDeep) {
            if (k0 + kDeep < ke) ask(buf[1], k0 + kDeep);
            add(buf[0]);
            if (k0 + kDeep >= ke) break;
            if (k0 + 2 * kDeep < ke) ask(buf[0], k0 + 2 * kDeep);
            add(buf[1]);
        }
        if constexpr (kTurnDown) __syncthreads();                  // the parts stand where the waves' places were
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
    }
    if constexpr (kPart == kDown) {
        for (int i = tid; i < rows * g.r; i += kThreads) {
            const int m = i / g.r, j = i - m * g.r;
            g.h[((long long)mine * g.M + row0 + m) * g.r + j] = (part[0][m][j] + part[1][m][j]) + (part[2][m][j] + part[3][m][j]);
        }
        return;
    }
    // the wave's rows of H, all of their parts requested before the first is used
    constexpr int per = R > 64 ? R / 64 : 1, kOwn = T / kWaves;
    float v[kOwn][per];
#pragma unroll
    for (int o = 0; o < kOwn; ++o)
#pragma unroll
        for (int i = 0; i < per; ++i) {
            const int m = wave + kWaves * o, j = lane + 64 * i;
            v[o][i] = 0.0f;
            if (kPart == kBoth && j < g.r) v[o][i] = (part[0][m][j] + part[1][m][j]) + (part[2][m][j] + part[3][m][j]);
        }
    if constexpr (kPart == kUp) {
#pragma unroll 4
        for (int x = 0; x < pieces; ++x)
#pragma unroll
            for (int o = 0; o < kOwn; ++o)
#pragma unroll
                for (int i = 0; i < per; ++i)
                    v[o][i] += g.h[((long long)x * g.M + row0 + min(wave + kWaves * o, rows - 1)) * g.r + min(lane + 64 * i, g.r - 1)];
    }
    float top[kOwn];
#pragma unroll
    for (int o = 0; o < kOwn; ++o) {
        top[o] = 0.0f;
#pragma unroll
        for (int i = 0; i < per; ++i) {
            if (lane + 64 * i >= g.r) v[o][i] = 0.0f;
            top[o] = fmaxf(top[o], fabsf(v[o][i]));
        }
    }
    for (int x = 1; x < 64; x <<= 1)
#pragma unroll
        for (int o = 0; o < kOwn; ++o) top[o] = fmaxf(top[o], __shfl_xor(top[o], x, 64));
#pragma unroll
    for (int o = 0; o < kOwn; ++o) {
        const int m = wave + kWaves * o;
        const uint32_t ex = min(max(__float_as_uint(top[o]) >> 23, 15u), 250u);
        const float up = __uint_as_float((268u - ex) << 23);            // the row's largest to 2^14 .. 2^15
        if (lane == 0) factor[m] = scale * __uint_as_float((ex - 14u) << 23);
#pragma unroll
        for (int i = 0; i < per; ++i) {
            const int j = lane + 64 * i;
            if (j < 32 * RS) {
                store_parts(v[o][i] * up, v[o][i] != 0.0f, h_hi[m][j], h_lo[m][j]);
            }
        }
    }
    __syncthreads();

    f16x8 hh[kTM][RS], hl[kTM][RS];
    f32x4 f[kTM];
#pragma unroll
    for (int t = 0; t < kTM; ++t) {
        f[t] = *(const f32x4 *)&factor[16 * t + 4 * gr];
#pragma unroll
        for (int s = 0; s < RS; ++s) {
            hh[t][s] = *(const f16x8 *)&h_hi[16 * t + col][32 * s + 8 * gr];
            hl[t][s] = *(const f16x8 *)&h_lo[16 * t + col][32 * s + 8 * gr];
        }
    }
    if (!kEarly && nb < n1) ask_up(nb);
    for (; nb < n1; nb += kCols) {
        f32x4 o[kTM][4] = {};
        if constexpr (kTurnUp) {
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                const int q = 64 * i + lane, n = (q * per_row) >> 16, k = q - n * (g.r >> 3);
                if (n < 64) *(f16x8 *)(turn_up + (n & 3) * kUpBlock + (n >> 2) * kLdUp + 8 * k) = ahead.b[i];
            }
            wave_sync();
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int s = 0; s < RS; ++s) {
                f16x8 b = {};
                if (32 * s + 8 * gr < g.r) {
                    if constexpr (kTurnUp)
                        b = *(const f16x8 *)(turn_up + u * kUpBlock + col * kLdUp + 8 * gr);
                    else
                        b = ahead.b[u * RS + s];
                }
#pragma unroll
                for (int t = 0; t < kTM; ++t) {
                    o[t][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(hh[t][s], b, o[t][u], 0, 0, 0);
                    o[t][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(hl[t][s], b, o[t][u], 0, 0, 0);
                }
            }
        if constexpr (kTurnUp) wave_sync();
        const int n = nb + 4 * col;
#pragma unroll
        for (int t = 0; t < kTM; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int m = 16 * t + 4 * gr + i;
                if (m >= rows || n >= n1) continue;
                f16x4 r;
#pragma unroll
                for (int u = 0; u < 4; ++u) r[u] = (_Float16)((float)ahead.y[t][i][u] + f[t][i] * o[t][u][i]);
                *(f16x4 *)(out + (uint32_t)(m * g.ldo + n)) = r;
            }
        if (nb + kCols < n1) ask_up(nb + kCols);
    }
}

// Pieces of about `want` in all, each of whole steps.
int piece_of(int size, int step, int tiles, int want)
{
    const int steps = (size + step - 1) / step;
    int pieces = (want + tiles - 1) / tiles;
    pieces = pieces < steps ? pieces : steps;
    return (steps + pieces - 1) / pieces * step;
}

struct Shape {
    bool two_rows;      // tiles of 32 rows
    bool two_launches;
    int tiles, k_piece, k_pieces;
};

Shape shape_of(int M, int K, int N, int r, int n_requests)
{
    Shape s{};
    // Prompts: 32 rows share what is read of A and B.  us, 32 rows and 16: 8192 x 4096 -> 4096 at rank 32 57.6 / 79.0, 8192 x 1280 ->
    // 1280 at 16 14.8 / 17.1, 500 x 5000 -> 5000 at 16 13.1 / 13.6; with little to share 16 are more workgroups, 600 x 2000 -> 600 at
    // 16 8.4 / 7.5, 300 x 1000 -> 1000 6.9 / 5.5.
    s.two_rows = r <= 64 && (long long)M >= 32ll * n_requests && (long long)M * K >= 3 << 19;
    s.tiles = M / (s.two_rows ? 32 : 16) + n_requests;
    // Two launches where A is more than a workgroup should read by itself.  us, one and two: a token at K = 4096 and rank 64
    // 20.4 / 9.9, 16 tokens at 4096 and 16 9.1 / 7.6, 40 requests in 512 rows at 4096 and 32 28.3 / 15.1; 64 tokens at 1280 and 16
    // 8.9 / 9.9, a token at 768 and 8 4.6 / 6.6, 8192 at 1280 and 16 14.7 / 20.5.
    s.two_launches = (long long)r * K >= 1 << 16;
    s.k_piece = piece_of(K, kDeep, s.tiles, 512);
    s.k_pieces = (K + s.k_piece - 1) / s.k_piece;
    return s;
}

template <int kTM, int kRT>
hipError_t launch(const LoraArgs &g, const Shape &p, hipStream_t s)
{
    const dim3 block(kThreads);
    if (!p.two_launches) {
        const int strip = piece_of(g.N, kCols, p.tiles, 512);
        return launch_kernel(k_lora<kTM, kRT, kBoth>, dim3(p.tiles, (g.N + strip - 1) / strip), block, 0, s, g, strip, 1);
    }
    const hipError_t e = launch_kernel(k_lora<kTM, kRT, kDown>, dim3(p.tiles, p.k_pieces), block, 0, s, g, p.k_piece, p.k_pieces);
    if (e != hipSuccess) return e;
    const int strip = piece_of(g.N, kCols, p.tiles, 1024);        // (512: 60.9 us for 58.0 at rank 32, 256: 66.6)
    return launch_kernel(k_lora<kTM, kRT, kUp>, dim3(p.tiles, (g.N + strip - 1) / strip), block, 0, s, g, strip, p.k_pieces);
}

}  // namespace

// Enough for every call with M and n_requests no larger: fewer tiles have more pieces, so that a call's own parts of H would not be.  Pieces are
// at most the steps of K, and less than 512 / tiles + 1, where there are more than M / 32 tiles.
size_t lora_workspace_bytes(int M, int K, int N, int r, int n_requests)
{
    if (!shape_of(M, K, N, r, n_requests).two_launches) return 0;
    const long long steps = (K + kDeep - 1) / kDeep;
    return (size_t)std::min(steps * M, 512ll * 32 + M) * r * 4;
}

hipError_t lora_prepare()
{
    hipFuncAttributes at;
    return hipFuncGetAttributes(&at, (const void *)k_lora<1, 1, kBoth>);
}

hipError_t launch_lora(const LoraArgs &g, hipStream_t s)
{
    const Shape p = shape_of(g.M, g.K, g.N, g.r, g.n_requests);
    if (g.r <= 16) return p.two_rows ? launch<2, 1>(g, p, s) : launch<1, 1>(g, p, s);
    if (g.r <= 32) return p.two_rows ? launch<2, 2>(g, p, s) : launch<1, 2>(g, p, s);
    if (g.r <= 64) return p.two_rows ? launch<2, 4>(g, p, s) : launch<1, 4>(g, p, s);
    return launch<1, 8>(g, p, s);
}

}  // namespace muxq
