// Drafted trees against the target's probabilities: which nodes stand, and the token after them.
//
// A node's children, ascending, are tried against r, at first the target's probabilities p after the node: child c with token x
// stands if u_c q(x) Z < r(x), where q is what it was drawn from; otherwise r becomes max(r / Z - q, 0) and Z its sum, which keeps the
// result distributed as p.  A workgroup has a tree: the comparisons need two numbers of a row each, which all nodes request
// together at the start; a rejection needs a sum over the vocabulary, which is what the time goes into.  r is never stored: a pass
// forms it anew from p, q and the sums of the earlier rejections, in binary64 (the difference of two binary32 numbers is
// exact there but for 2^-53, and a sum's order moves a token only where u is within 2^-45 of a border).
// Sums stand for blocks of 1024 tokens in LDS, so that the search for the next token goes through the blocks' sums and one block.
#include "muxq_block_kernels.h"

namespace muxq {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64, kBlock = 1024, kMaxBlocks = (1 << 22) / kBlock;

typedef float Four __attribute__((ext_vector_type(4), aligned(4)));        // rows of an odd vocabulary begin anywhere

__device__ __forceinline__ double wave_sum(double v)
{
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) v += __shfl_xor(v, x, 64);
    return v;
}

// Where a node's children are tried: p, q (NULL: 1 for the child's token) and the rejections so far.
struct Rest {
    const float *p, *q;
    int rejected;               // rejections
    const double *inv;          // 1 / Z of all but the last
    const int *gone;            // without q: their tokens
};

__device__ __forceinline__ double less(const Rest &r, double x, double q, int t)
{
    if (r.rejected == 0) return x;
    if (r.q) {
        x = fmax(x - q, 0.0);
        for (int j = 1; j < r.rejected; ++j) x = fmax(x * r.inv[j] - q, 0.0);
    } else {
        for (int j = 0; j < r.rejected; ++j)
            if (r.gone[j] == t) x = 0.0;
        // what the earlier sums divide it by does not change its share: one number for all tokens
    }
    return x;
}

// Four tokens from t on.
__device__ __forceinline__ void four(const Rest &r, int t, int V, double out[4])
{
    Four p = {}, q = {};
    if (t + 4 <= V) {
        p = *(const Four *)(r.p + t);
        if (r.q && r.rejected) q = *(const Four *)(r.q + t);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (t + i < V) {
                p[i] = r.p[t + i];
                if (r.q && r.rejected) q[i] = r.q[t + i];
            }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = less(r, p[i], q[i], t + i);
}

__global__ __launch_bounds__(kThreads) void k_verify(VerifyArgs a)
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
            // the largest of target[v], the lowest of equal ones
            const float *const p = a.target + (first + v) * a.ldt;
            float most = -__builtin_inff();
            int best = 0x7fffffff;
            auto look = [&](float x, int t) {
                if (x > most) most = x, best = t;
            };
            for (int t = tid * 4; t < V; t += 4 * kThreads) {
                if (t + 4 <= V) {
                    const Four x = *(const Four *)(p + t);
#pragma unroll
                    for (int i = 0; i < 4; ++i) look(x[i], t + i);
                } else {
                    for (int i = t; i < V; ++i) look(p[i], i);
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
            if (best == 0x7fffffff) best = 0;       // nothing above -infinity
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
        for (int b = wave; b < blocks; b += kWaves) {
            double sum = 0.0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int t = b * kBlock + i * 256 + lane * 4;
                double x[4] = {};
                if (t < V) four(r, t, V, x);
                sum += (x[0] + x[1]) + (x[2] + x[3]);
            }
            sum = wave_sum(sum);
            if (lane == 0) sh_block[b] = sum;
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
            double up = mine;
#pragma unroll
            for (int x = 1; x < 64; x <<= 1) {
                const double y = __shfl_up(up, x, 64);
                if (lane >= x) up += y;
            }
            const unsigned long long past = __ballot(before + up > to && mine > 0.0), some = __ballot(mine > 0.0);
            if (past) {
                const int l = __ffsll((long long)past) - 1;
                found = b0 + l;
                at_found = before + __shfl(up - mine, l, 64);
            } else if (some) {
                const int l = 63 - __clzll((long long)some);
                last = b0 + l;
                at_last = before + __shfl(up - mine, l, 64);
            }
            before += __shfl(up, 63, 64);
        }
        if (found < 0) found = last, at_found = at_last;
        int token = -1, positive = -1;
        for (int i = 0; i < 4 && token < 0; ++i) {
            const int t = found * kBlock + i * 256 + lane * 4;
            double x[4] = {};
            if (t < V) four(r, t, V, x);
            const double mine = (x[0] + x[1]) + (x[2] + x[3]);
            double up = mine;
#pragma unroll
            for (int y = 1; y < 64; y <<= 1) {
                const double z = __shfl_up(up, y, 64);
                if (lane >= y) up += z;
            }
            double run = at_found + (up - mine);
            int here = -1, some = -1;
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                run += x[y];
                if (x[y] > 0.0) {
                    some = t + y;
                    if (here < 0 && run > to) here = t + y;
                }
            }
            const unsigned long long past = __ballot(here >= 0), any = __ballot(some >= 0);
            if (past) token = __shfl(here, __ffsll((long long)past) - 1, 64);
            if (any) positive = __shfl(some, 63 - __clzll((long long)any), 64);
            at_found += __shfl(up, 63, 64);
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
    return launch_kernel(k_verify, dim3(a.S), dim3(kThreads), lds, s, a);
}

}  // namespace muxq
