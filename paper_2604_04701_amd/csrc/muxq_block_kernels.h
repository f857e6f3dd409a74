// Launch interface between the checks of the entry points in muxq_block.h (muxq_block_api.hip) and
// their kernels.  Every function enqueues on `s` and returns the status of the launch.
#pragma once
#include "../../include/muxq_block.h"
#include "muxq_kernels.h"

namespace muxq {

// The cache as the kernels see it.
struct KvView {
    char *k, *v;
    float *k_scale, *v_scale;
    int n_blocks, block_shift, n_kv_heads, head_dim;   // block_size = 1 << block_shift
    long long ld_block, ld_head, ld_token;             // elements
};

struct AppendArgs {
    const _Float16 *k, *v, *q;
    _Float16 *q_out;
    const int32_t *slots, *positions;
    const float *cos_sin;
    int M, ldk, ldv, ldq, ldqo, n_heads, n_positions, rot_dim;
    KvView c;
};
hipError_t launch_kv_append(const AppendArgs &a, bool int8, bool interleaved, hipStream_t s);
hipError_t launch_kv_gather(const int32_t *slots, int M, const KvView &c, bool int8, _Float16 *k_out, int ldk,
                            _Float16 *v_out, int ldv, hipStream_t s);

struct AttendArgs {
    const _Float16 *q;
    _Float16 *o;
    const int32_t *table, *lengths;
    int S, n_heads, group, ldq, ldo, ld_table, max_length;
    float scale;
    void *workspace;
    KvView c;
    // one row of a sequence at most, with a window (launch_attend_rows only)
    const int32_t *starts;
    int M, window, sinks;
};
bool attend_rows_fits(int S, int n_heads, int n_kv_heads, int head_dim, int max_length, int window, int sinks);
hipError_t launch_attend_rows(const AttendArgs &a, bool int8, hipStream_t s);
size_t attend_workspace_need(int S, int n_heads, int n_kv_heads, int head_dim, int max_length);
size_t attend_workspace_bytes(int S, int n_heads, int n_kv_heads, int head_dim, int max_length);
hipError_t launch_attend(const AttendArgs &a, bool int8, hipStream_t s);

struct LoraArgs {
    const _Float16 *x, *a, *b, *y;
    _Float16 *out;
    const float *scales;
    const int32_t *starts, *adapters;
    int M, K, N, r, n_adapters, n_requests, ldx, ldy, ldo;
    float *h;       // [pieces of K][M][r]
};
size_t lora_workspace_bytes(int M, int K, int N, int r, int n_requests);
hipError_t launch_lora(const LoraArgs &a, hipStream_t s);

struct NormArgs {
    const _Float16 *x, *res, *post_w, *post_b, *gate, *w, *b;
    _Float16 *r_out, *y;
    int M, K, ldx, ldr, ldg, ldro, ldy, k_pad;
    float r_scale, eps;
    uint16_t *slabs, *scratch;
};
int norm_slab_rows(int M);                        // rows of maxima a call leaves
size_t norm_scratch_bytes(int M, int K, int k_pad);
hipError_t launch_norm(const NormArgs &a, bool rms, hipStream_t s);

constexpr int kMaxNodes = 64;           // nodes of a drafted tree: the bits of a word

// Attention of several new tokens a sequence; parents: of a tree's nodes, NULL: causal, with a window.
struct RowsArgs {
    const _Float16 *q;
    _Float16 *o;
    const int32_t *table, *starts, *lengths, *parents;
    int M, S, n_heads, group, ldq, ldo, ld_table, max_new, max_length, window, sinks;
    float scale;
    void *workspace;
    KvView c;
};
size_t rows_workspace_need(int S, int n_heads, int n_kv_heads, int head_dim, int max_new, int max_length, int window, int sinks, bool tree);
size_t rows_workspace_bytes(int S, int n_heads, int n_kv_heads, int head_dim, int max_new, int max_length, int window, int sinks, bool tree);
hipError_t launch_rows(const RowsArgs &a, bool int8, hipStream_t s);

struct VerifyArgs {
    const float *target, *draft, *uniforms;
    const int32_t *tokens, *parents, *starts;
    int32_t *path, *counts, *next;
    long long ldt, ldd;
    int M, V, S, max_nodes;
};
hipError_t launch_verify(const VerifyArgs &a, hipStream_t s);

hipError_t launch_kv_copy(const int32_t *src, const int32_t *dst, int n, const KvView &c, bool int8, hipStream_t s);
struct CompactArgs {
    const int32_t *path, *counts, *starts, *lengths, *table;
    int ld_table, M, S, max_nodes;
    KvView c;
};
hipError_t launch_kv_compact(const CompactArgs &a, bool int8, hipStream_t s);

// Load a file's kernels on the current device, so that a first call may be captured.
hipError_t attend_prepare();
hipError_t kv_prepare();
hipError_t lora_prepare();
hipError_t norm_prepare();
hipError_t rows_prepare();
hipError_t verify_prepare();
hipError_t pages_prepare();

}  // namespace muxq
