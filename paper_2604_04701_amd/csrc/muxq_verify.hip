// Drafted trees against the target's probabilities: which nodes stand, and the token after them.
//
// A node's children, ascending, are tried against r, at first the target's probabilities p after the node: child c with token x
// stands if u_c q(x) Z < r(x), where q is what it was drawn from; otherwise r becomes max(r / Z - q, 0) and Z its sum, which keeps the
// result distributed as p.  A workgroup has a tree: the comparisons need two numbers of a row each, which all nodes request
// together at the start; a rejection needs a sum over the vocabulary, which is what the time goes into.  r is never stored: a pass
// forms it anew from p, q and the sums of the earlier rejections, in binary64 (the difference of two binary32 numbers is
// exact there but for 2^-53, and a sum's order moves a token only where u is within 2^-45 of a border).
// Sums stand for blocks of 1024 tokens in LDS, so that the search for the next token goes through the blocks' sums and one block.
//
// 64 sampled trees of 32 nodes, 50257 tokens: 45 us, two to six passes a tree of 7 to 9 us, each 400 KB through one CU and 100000 conversions to
// binary64; 64 of the 256 CUs work.  More CUs a tree would have to wait for each other within a launch, or take a launch for each
// rejection.  A chain of four, greedy: 13 us, 6.5 of them the rows' largest, five workgroups, and 2.4 the walk.
// Taken back: half of the threads, more blocks on their way (50 us, greedy ones 28 against 23); sixteen numbers of a lane at once (they spilled: 111 us).
#include "muxq_block_kernels.h"

namespace muxq {
namespace {

// Numbers of a target whose rows are looked at all at once where greedy: 8 chains of 16 nodes, 50257 tokens each, 12.8 us, 45.4 row after row along the
// path; 5 trees of 32 14.5 and 20.0; 8 of them 19.0 and 19.9; 32 of 8 nodes (12 million numbers) 16.9 and 13.4.
constexpr long long kAtOnce = 8 << 20;
constexpr int kThreads = 1024, kWaves = kThreads / 64, kBlock = 1024;

typedef float Four __attribute__((ext_vector_type(4), aligned(4)));        // rows of an odd vocabulary begin anywhere

// v plus the value of another lane: lanes of a row of 16 to the right, or the last lane of a row to the rows in kRows.
template <int kWhere, int kRows>
__device__ __forceinline__ double plus(double v)
{
    typedef int Two __attribute__((ext_vector_type(2)));
    const Two x = __builtin_bit_cast(Two, v);
    return v + __builtin_bit_cast(double, Two{__builtin_amdgcn_update_dpp(0, x[0], kWhere, kRows, 0xf, false),
                                              __builtin_amdgcn_update_dpp(0, x[1], kWhere, kRows, 0xf, false)});
}

// The sums up to each lane, without LDS.
__device__ __forceinline__ double wave_scan(double v)
{
    v = plus<0x111, 0xf>(v);
    v = plus<0x112, 0xf>(v);
    v = plus<0x114, 0xf>(v);
    v = plus<0x118, 0xf>(v);
    v = plus<0x142, 0xa>(v);
    return plus<0x143, 0xc>(v);
}

__device__ __forceinline__ double lane_of(double v, int lane)
{
    typedef int Two __attribute__((ext_vector_type(2)));
    const Two x = __builtin_bit_cast(Two, v);
    return __builtin_bit_cast(double, Two{__builtin_amdgcn_readlane(x[0], lane), __builtin_amdgcn_readlane(x[1], lane)});
}

__device__ __forceinline__ double wave_sum(double v) { return lane_of(wave_scan(v), 63); }

// Where a node's children are tried: p, q (NULL: 1 for the child's token) and the rejections so far.
struct Rest {
    const float *p, *q;
    int rejected;               // rejections
    const double *inv;          // 1 / Z of all but the last
    const int *gone;            // without q: their tokens
};

// r of one token, from p and q there.
__device__ __forceinline__ double less(const Rest &r, double x, double q, int t)
{
    if (r.q) {
        if (r.rejected) x = fmax(x - q, 0.0);
        for (int j = 1; j < r.rejected; ++j) x = fmax(x * r.inv[j] - q, 0.0);
    } else {
        // (what the earlier sums divide it by does not change its share: one number for all tokens)
        for (int j = 0; j < r.rejected; ++j)
            if (r.gone[j] == t) x = 0.0;
    }
    return x;
}

// Four numbers of a row from t on, or its last four where t is near its end or beyond: of those the ones before t are another lane's.
// (Rows of an odd vocabulary begin between 16-byte pieces; blocks that begin at such a piece instead were no faster.)
__device__ __forceinline__ int first_of(int t, int V) { return V >= 4 ? min(t, V - 4) : 0; }
__device__ __forceinline__ Four four(const float *p, int t, int V)
{
    if (V >= 4) return *(const Four *)(p + first_of(t, V));
    return Four{p[0], p[min(1, V - 1)], p[min(2, V - 1)], p[V - 1]};
}

// A lane's tokens of a block: four runs of four, 256 tokens apart.
struct Tokens {
    Four p[4], q[4];
};

__device__ __forceinline__ void ask(const Rest &r, int block, int V, Tokens &x)
{
    const int t0 = block * kBlock + (threadIdx.x & 63) * 4;
#pragma unroll
    for (int i = 0; i < 4; ++i) x.p[i] = four(r.p, t0 + i * 256, V);
    if (r.q && r.rejected)
#pragma unroll
        for (int i = 0; i < 4; ++i) x.q[i] = four(r.q, t0 + i * 256, V);
}

// r of the i-th of these runs, 0 for what is another lane's or none's.
__device__ __forceinline__ void values(const Rest &r, int block, int i, int V, const Tokens &y, double x[4])
{
    const int t = block * kBlock + i * 256 + (threadIdx.x & 63) * 4, from = first_of(t, V);
#pragma unroll
    for (int z = 0; z < 4; ++z) x[z] = y.p[i][z];
    if (r.q && r.rejected) {
#pragma unroll
        for (int z = 0; z < 4; ++z) x[z] = fmax(x[z] - (double)y.q[i][z], 0.0);
        for (int j = 1; j < r.rejected; ++j) {
            const double inv = r.inv[j];
#pragma unroll
            for (int z = 0; z < 4; ++z) x[z] = fmax(x[z] * inv - (double)y.q[i][z], 0.0);
        }
    } else {
        for (int j = 0; j < r.rejected; ++j) {
            const int gone = r.gone[j];
#pragma unroll
            for (int z = 0; z < 4; ++z) x[z] = from + z == gone ? 0.0 : x[z];
        }
    }
    if ((block + 1) * kBlock > V)
#pragma unroll
        for (int z = 0; z < 4; ++z) x[z] = from + z < t || from + z >= V ? 0.0 : x[z];
}

// The largest of a row, the lowest index of equal ones, for all threads of a workgroup.
__device__ int largest(const float *p, int V, float *sh_most, int *sh_best)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    constexpr int kEach = 8;                            // loads on their way
    float most = -__builtin_inff();
    int best = 0x7fffffff;
    auto look = [&](float x, int t) {
        if (x > most) most = x, best = t;
    };
    // (numbers looked at twice change nothing)
    for (int t0 = 0; t0 < V; t0 += 4 * kThreads * kEach) {
        Four x[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            if (t0 + i * 4 * kThreads < V) x[i] = four(p, t0 + (i * kThreads + tid) * 4, V);
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            if (t0 + i * 4 * kThreads < V) {
                const int at = first_of(t0 + (i * kThreads + tid) * 4, V);
#pragma unroll
                for (int y = 0; y < 4; ++y) look(x[i][y], at + y);
            }
    }
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) {
        const float other = __shfl_xor(most, x, 64);
        const int at = __shfl_xor(best, x, 64);
        if (other > most || (other == most && at < best)) most = other, best = at;
    }
    __syncthreads();                        // the last row's readers
    if (lane == 0) sh_most[wave] = most, sh_best[wave] = best;
    __syncthreads();
    most = sh_most[0], best = sh_best[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w)
        if (sh_most[w] > most || (sh_most[w] == most && sh_best[w] < best)) most = sh_most[w], best = sh_best[w];
    return best == 0x7fffffff ? 0 : best;       // nothing above -infinity
}

// The largest of each row, left in path, which is not yet needed for anything else.
__global__ __launch_bounds__(kThreads) void k_largest(VerifyArgs a)
{
    __shared__ float sh_most[kWaves];
    __shared__ int sh_best[kWaves];
    if ((int)blockIdx.x < a.starts[0] || (int)blockIdx.x >= a.starts[a.S]) return;       // a row of no sequence
    const int best = largest(a.target + blockIdx.x * a.ldt, a.V, sh_most, sh_best);
    if (threadIdx.x == 0) a.path[blockIdx.x] = best;
}

__global__ __launch_bounds__(kThreads) void k_verify(VerifyArgs a, bool known)
{
    extern __shared__ __align__(16) double sh_block[];         // [blocks of the vocabulary]
    __shared__ double sh_inv[kMaxNodes + 1], sh_total;
    __shared__ float sh_p[kMaxNodes], sh_q[kMaxNodes], sh_u[kMaxNodes];
    __shared__ int sh_token[kMaxNodes], sh_parent[kMaxNodes], sh_gone[kMaxNodes], sh_best[kWaves];
    __shared__ float sh_most[kWaves];
    const int s = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, V = a.V, blocks = (V + kBlock - 1) / kBlock;
    const int first = max(0, min(a.starts[s], a.M)), n = max(0, min(a.starts[s + 1], a.M)) - first;
    if (n < 1 || n > a.max_nodes) {
        for (int i = tid; i < n; i += kThreads) a.path[first + i] = -1;
        if (tid == 0) a.counts[s] = 0, a.next[s] = -1;
        return;
    }
    if (tid < n) {
        const int token = a.tokens[first + tid], up = a.parents[first + tid];
        sh_token[tid] = token;
        sh_parent[tid] = up;
        float p = 0.0f, q = 1.0f;
        if (known) sh_gone[tid] = a.path[first + tid];        // the largest of the node's row
        if (a.uniforms) {
            sh_u[tid] = a.uniforms[first + tid];
            if (up >= 0 && up < tid && token >= 0 && token < V) {
                p = a.target[(first + up) * a.ldt + token];
                if (a.draft) q = a.draft[(first + up) * a.ldd + token];
            }
        }
        sh_p[tid] = p;
        sh_q[tid] = q;
    }
    __syncthreads();

    int v = 0, count = 1;
    if (tid == 0) a.path[first] = 0;
    auto accept = [&](int c) {
        v = c;
        if (tid == 0) a.path[first + count] = c;
        ++count;
    };
    auto finish = [&](int token) {
        if (tid >= count && tid < n) a.path[first + tid] = -1;
        if (tid == 0) a.counts[s] = count, a.next[s] = token;
    };

    if (!a.uniforms) {
        for (;;) {
            const int best = known ? sh_gone[v] : largest(a.target + (first + v) * a.ldt, V, sh_most, sh_best);
            int taken = -1;
            for (int c = v + 1; c < n; ++c)
                if (sh_parent[c] == v && sh_token[c] == best) {
                    taken = c;
                    break;
                }
            if (taken < 0) return finish(best);
            accept(taken);
        }
    }

    Rest r{};
    r.inv = sh_inv;
    r.gone = sh_gone;
    double Z = 1.0;
    auto at_node = [&]() {
        r.p = a.target + (first + v) * a.ldt;
        r.q = a.draft ? a.draft + (first + v) * a.ldd : nullptr;
        r.rejected = 0;
        Z = 1.0;
    };
    // the sum of r, and of its blocks
    auto pass = [&]() {
        Tokens y[2];
        int b = wave;
        if (b < blocks) ask(r, b, V, y[0]);
        for (; b < blocks; b += kWaves) {
            if (b + kWaves < blocks) ask(r, b + kWaves, V, y[1]);
            double sum = 0.0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                double x[4];
                values(r, b, i, V, y[0], x);
                sum += (x[0] + x[1]) + (x[2] + x[3]);
            }
            sum = wave_sum(sum);
            if (lane == 0) sh_block[b] = sum;
            y[0] = y[1];
        }
        __syncthreads();
        if (wave == 0) {
            double sum = 0.0;
            for (int b = lane; b < blocks; b += 64) sum += sh_block[b];
            sum = wave_sum(sum);
            if (lane == 0) sh_total = sum;
        }
        __syncthreads();
        return sh_total;
    };
    at_node();
    bool summed = false;                // sh_block holds the sums of r as it is
    double sum = 0.0;
    for (int c = 1; c < n; ++c) {
        if (sh_parent[c] != v || sh_token[c] < 0 || sh_token[c] >= V) continue;
        double x = sh_p[c], q = sh_q[c];
        if (r.q) {
            x = less(r, x, q, 0);
        } else {
            for (int j = 0; j < r.rejected; ++j)
                if (sh_gone[j] == sh_token[c]) x = 0.0;
        }
        if ((double)sh_u[c] * q * Z < x) {
            accept(c);
            at_node();
            summed = false;
            continue;
        }
        __syncthreads();                // readers of the list
        if (tid == 0) {
            sh_inv[r.rejected] = 1.0 / Z;
            sh_gone[r.rejected] = sh_token[c];
        }
        ++r.rejected;
        __syncthreads();
        sum = pass();
        summed = true;
        if (!(sum > 0.0)) {             // nothing is left
            r.rejected = 0;
            summed = false;
            break;
        }
        Z = sum;
    }
    if (!summed) sum = pass();
    if (!(sum > 0.0)) return finish(-1);
    if (wave == 0) {
        // the block in which the running sum passes u * sum, or the last one with a sum
        const double to = (double)sh_u[0] * sum;
        double before = 0.0;
        int found = -1, last = 0;
        double at_last = 0.0, at_found = 0.0;
        for (int b0 = 0; b0 < blocks && found < 0; b0 += 64) {
            const int b = b0 + lane;
            const double mine = b < blocks ? sh_block[b] : 0.0;
            const double up = wave_scan(mine);
            const unsigned long long past = __ballot(before + up > to && mine > 0.0), some = __ballot(mine > 0.0);
            if (past) {
                const int l = __ffsll((long long)past) - 1;
                found = b0 + l;
                at_found = before + lane_of(up - mine, l);
            } else if (some) {
                const int l = 63 - __clzll((long long)some);
                last = b0 + l;
                at_last = before + lane_of(up - mine, l);
            }
            before += lane_of(up, 63);
        }
        if (found < 0) found = last, at_found = at_last;
        int token = -1, positive = -1;
        Tokens y;
        ask(r, found, V, y);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = first_of(found * kBlock + i * 256 + lane * 4, V);
            double x[4];
            values(r, found, i, V, y, x);
            const double mine = (x[0] + x[1]) + (x[2] + x[3]);
            const double up = wave_scan(mine);
            double run = at_found + (up - mine);
            int here = -1, some = -1;
#pragma unroll
            for (int z = 0; z < 4; ++z) {
                run += x[z];
                if (x[z] > 0.0) {
                    some = t + z;
                    if (here < 0 && run > to) here = t + z;
                }
            }
            const unsigned long long past = __ballot(here >= 0), any = __ballot(some >= 0);
            if (past && token < 0) token = __shfl(here, __ffsll((long long)past) - 1, 64);
            if (any) positive = __shfl(some, 63 - __clzll((long long)any), 64);
            at_found += lane_of(up, 63);
        }
        if (token < 0) token = positive;        // rounding, or u = 1
        if (lane == 0) a.next[s] = token;
    }
    if (tid >= count && tid < n) a.path[first + tid] = -1;
    if (tid == 0) a.counts[s] = count;
}

}  // namespace

hipError_t verify_prepare()
{
    hipFuncAttributes at;
    return hipFuncGetAttributes(&at, (const void *)k_verify);
}

hipError_t launch_verify(const VerifyArgs &a, hipStream_t s)
{
    const size_t lds = (size_t)((a.V + kBlock - 1) / kBlock) * sizeof(double);
    // Greedy: all rows at once and the walk after them, or the rows of a walk one after the other.
    // (A launch has fewer than 2^32 threads.)
    const bool known = !a.uniforms && (long long)a.M * a.V <= kAtOnce && (long long)a.M * kThreads < 1ll << 32;
    if (known) {
        const hipError_t e = launch_kernel(k_largest, dim3(a.M), dim3(kThreads), 0, s, a);
        if (e != hipSuccess) return e;
    }
    return launch_kernel(k_verify, dim3(a.S), dim3(kThreads), lds, s, a, known);
}

}  // namespace muxq
