// Entry points of muxq_block.h: argument checks and the choice of kernels.
#include "muxq_block_kernels.h"

#include <math.h>

namespace {

inline bool aligned(const void *p, size_t a) { return ((uintptr_t)p % a) == 0; }
inline int kpad(int K) { return (K + muxq::kKStep - 1) / muxq::kKStep * muxq::kKStep; }

// A row stride: at least the row, whole 16-byte pieces.
inline bool bad_ld(long long ld, long long width) { return ld < width || ld % 8 != 0; }

// Whether two fp16 matrices of `rows` rows share an element.  Rows of one buffer side by side (same stride)
// are told apart by where they start in a row; with different strides one inside the other's span counts as shared.
bool share(const void *p, long long ldp, long long width_p, const void *q, long long ldq, long long width_q, long long rows)
{
    const long long a = (long long)(uintptr_t)p / 2, b = (long long)(uintptr_t)q / 2;
    if (a + (rows - 1) * ldp + width_p <= b || b + (rows - 1) * ldq + width_q <= a) return false;
    if (ldp != ldq || rows == 1) return true;
    const long long off = ((b - a) % ldp + ldp) % ldp;           // q's columns start here in p's rows
    return off < width_p || off + width_q > ldp;
}

int check_cache(const muxq_kv_cache *c, muxq::KvView *view)
{
    if (!c || !c->k || !c->v) return MUXQ_ERR_NULL;
    if (c->type != MUXQ_KV_FP16 && c->type != MUXQ_KV_INT8) return MUXQ_ERR_PARAM;
    if (c->reserved != 0) return MUXQ_ERR_PARAM;
    if (c->type == MUXQ_KV_INT8 && (!c->k_scale || !c->v_scale)) return MUXQ_ERR_NULL;
    const int bs = c->block_size;
    if (bs < 8 || bs > 256 || (bs & (bs - 1)) != 0) return MUXQ_ERR_SHAPE;
    if (c->head_dim < 16 || c->head_dim > 256 || c->head_dim % 16 != 0) return MUXQ_ERR_SHAPE;
    if (c->n_kv_heads < 1 || c->n_kv_heads > 65535 || c->n_blocks < 1 || (long long)c->n_blocks * bs > 0x7fffffffll) return MUXQ_ERR_SHAPE;
    if (c->ld_token < c->head_dim || c->ld_head < c->head_dim || c->ld_token % 16 != 0 || c->ld_head % 16 != 0 ||
        c->ld_block % 16 != 0 || c->ld_token > (1ll << 32) || c->ld_head > (1ll << 32) || c->ld_block > (1ll << 60) / c->n_blocks)
        return MUXQ_ERR_SHAPE;
    if (c->ld_block < (bs - 1) * c->ld_token + (c->n_kv_heads - 1) * c->ld_head + c->head_dim) return MUXQ_ERR_SHAPE;
    // within a page rows of two heads or two tokens do not meet
    if (c->n_kv_heads > 1 && c->ld_head < (bs - 1) * c->ld_token + c->head_dim &&
        c->ld_token < (c->n_kv_heads - 1) * c->ld_head + c->head_dim)
        return MUXQ_ERR_SHAPE;
    if (!aligned(c->k, 16) || !aligned(c->v, 16)) return MUXQ_ERR_ALIGN;
    if (c->type == MUXQ_KV_INT8 && (!aligned(c->k_scale, 16) || !aligned(c->v_scale, 16))) return MUXQ_ERR_ALIGN;
    view->k = (char *)c->k;
    view->v = (char *)c->v;
    view->k_scale = c->k_scale;
    view->v_scale = c->v_scale;
    view->n_blocks = c->n_blocks;
    view->block_shift = __builtin_ctz((unsigned)bs);
    view->n_kv_heads = c->n_kv_heads;
    view->head_dim = c->head_dim;
    view->ld_block = c->ld_block;
    view->ld_head = c->ld_head;
    view->ld_token = c->ld_token;
    return MUXQ_OK;
}

constexpr int kMaxRows = 1 << 24, kMaxCols = 1 << 21;

// Sizes of an attention call without its cache.
int check_attend(int S, int n_heads, int n_kv_heads, int head_dim, int max_length)
{
    if (S < 1 || S > 65535 || n_heads < 1 || n_kv_heads < 1 || n_heads % n_kv_heads != 0 || max_length < 1 ||
        max_length > (1 << 26) ||
        head_dim < 16 || head_dim > 256 || head_dim % 16 != 0 || n_heads > kMaxCols / head_dim)
        return MUXQ_ERR_SHAPE;
    return MUXQ_OK;
}

#define MUXQ_TRY(expr)                          \
    do {                                        \
        if ((expr) != hipSuccess) return MUXQ_ERR_HIP; \
    } while (0)

}  // namespace

extern "C" {

int muxq_kv_append(const void *K, const void *V, int M, int ldk, int ldv, const void *Q, int n_heads, int ldq,
                   void *Q_out, int ldqo, const int32_t *slots, const int32_t *positions, const float *cos_sin,
                   int n_positions, int rot_dim, int interleaved, const muxq_kv_cache *cache, void *stream)
{
    if (!K || !V || !slots || (Q && !Q_out)) return MUXQ_ERR_NULL;
    muxq::AppendArgs a{};
    int st = check_cache(cache, &a.c);
    if (st) return st;
    if (rot_dim != 0 && (!positions || !cos_sin)) return MUXQ_ERR_NULL;
    const int d = a.c.head_dim, width = a.c.n_kv_heads * d;
    if (M < 1 || M > kMaxRows || a.c.n_kv_heads > kMaxCols / d || bad_ld(ldk, width) || bad_ld(ldv, width)) return MUXQ_ERR_SHAPE;
    if (rot_dim < 0 || rot_dim > d || rot_dim % 8 != 0 || (rot_dim != 0 && n_positions < 1)) return MUXQ_ERR_SHAPE;
    if (Q && (n_heads < 1 || n_heads > kMaxCols / d || bad_ld(ldq, (long long)n_heads * d) || bad_ld(ldqo, (long long)n_heads * d)))
        return MUXQ_ERR_SHAPE;
    if (!aligned(K, 16) || !aligned(V, 16) || (Q && (!aligned(Q, 16) || !aligned(Q_out, 16))) || !aligned(slots, 4) ||
        (rot_dim && (!aligned(positions, 4) || !aligned(cos_sin, 16))))
        return MUXQ_ERR_ALIGN;
    // queries may be turned in place; otherwise what is written is nobody's input
    if (Q && ((Q != Q_out || ldq != ldqo) && share(Q, ldq, (long long)n_heads * d, Q_out, ldqo, (long long)n_heads * d, M))) return MUXQ_ERR_PARAM;
    if (Q && (share(K, ldk, width, Q_out, ldqo, (long long)n_heads * d, M) || share(V, ldv, width, Q_out, ldqo, (long long)n_heads * d, M)))
        return MUXQ_ERR_PARAM;
    a.k = (const _Float16 *)K;
    a.v = (const _Float16 *)V;
    a.q = (const _Float16 *)Q;
    a.q_out = (_Float16 *)Q_out;
    a.slots = slots;
    a.positions = positions;
    a.cos_sin = cos_sin;
    a.M = M; a.ldk = ldk; a.ldv = ldv; a.ldq = ldq; a.ldqo = ldqo;
    a.n_heads = Q ? n_heads : 0;
    a.n_positions = n_positions;
    a.rot_dim = rot_dim;
    MUXQ_TRY(muxq::launch_kv_append(a, cache->type == MUXQ_KV_INT8, interleaved != 0, (hipStream_t)stream));
    return MUXQ_OK;
}

int muxq_kv_gather(const int32_t *slots, int M, const muxq_kv_cache *cache, void *K_out, int ldk, void *V_out,
                   int ldv, void *stream)
{
    if (!slots || !K_out || !V_out) return MUXQ_ERR_NULL;
    muxq::KvView c;
    int st = check_cache(cache, &c);
    if (st) return st;
    const int width = c.n_kv_heads * c.head_dim;
    if (M < 1 || M > kMaxRows || c.n_kv_heads > kMaxCols / c.head_dim || bad_ld(ldk, width) || bad_ld(ldv, width)) return MUXQ_ERR_SHAPE;
    if (!aligned(slots, 4) || !aligned(K_out, 16) || !aligned(V_out, 16)) return MUXQ_ERR_ALIGN;
    if (share(K_out, ldk, width, V_out, ldv, width, M)) return MUXQ_ERR_PARAM;
    MUXQ_TRY(muxq::launch_kv_gather(slots, M, c, cache->type == MUXQ_KV_INT8, (_Float16 *)K_out, ldk, (_Float16 *)V_out,
                                    ldv, (hipStream_t)stream));
    return MUXQ_OK;
}

size_t muxq_paged_attention_workspace_bytes(int S, int n_heads, int n_kv_heads, int head_dim, int max_length)
{
    if (check_attend(S, n_heads, n_kv_heads, head_dim, max_length)) return 0;
    return muxq::attend_workspace_bytes(S, n_heads, n_kv_heads, head_dim, max_length);
}

int muxq_paged_attention(const void *Q, int S, int n_heads, int ldq, const muxq_kv_cache *cache,
                         const int32_t *block_table, int ld_table, const int32_t *lengths, int max_length,
                         float scale, void *O, int ldo, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!Q || !O || !block_table || !lengths) return MUXQ_ERR_NULL;
    muxq::AttendArgs a{};
    int st = check_cache(cache, &a.c);
    if (st) return st;
    const int d = a.c.head_dim;
    if ((st = check_attend(S, n_heads, a.c.n_kv_heads, d, max_length))) return st;
    if (bad_ld(ldq, (long long)n_heads * d) || bad_ld(ldo, (long long)n_heads * d)) return MUXQ_ERR_SHAPE;
    if (ld_table < 1 || (long long)max_length > ((long long)ld_table << a.c.block_shift)) return MUXQ_ERR_SHAPE;
    if (!(fabsf(scale) <= 3.4e38f)) return MUXQ_ERR_PARAM;
    if (!aligned(Q, 16) || !aligned(O, 16) || !aligned(block_table, 4) || !aligned(lengths, 4)) return MUXQ_ERR_ALIGN;
    if ((Q != O || ldq != ldo) && share(Q, ldq, (long long)n_heads * d, O, ldo, (long long)n_heads * d, S)) return MUXQ_ERR_PARAM;
    const size_t need = muxq::attend_workspace_need(S, n_heads, a.c.n_kv_heads, d, max_length);
    if (need > 0) {
        if (!workspace) return MUXQ_ERR_NULL;
        if (!aligned(workspace, 256)) return MUXQ_ERR_ALIGN;
        if (workspace_bytes < need) return MUXQ_ERR_WORKSPACE;
    }
    a.q = (const _Float16 *)Q;
    a.o = (_Float16 *)O;
    a.table = block_table;
    a.lengths = lengths;
    a.S = S; a.n_heads = n_heads; a.group = n_heads / a.c.n_kv_heads;
    a.ldq = ldq; a.ldo = ldo; a.ld_table = ld_table;
    a.max_length = max_length;
    a.scale = scale;
    a.workspace = workspace;
    MUXQ_TRY(muxq::launch_attend(a, cache->type == MUXQ_KV_INT8, (hipStream_t)stream));
    return MUXQ_OK;
}

constexpr int kMaxLd = 1 << 25;              // 32 rows within 32-bit offsets

static bool lora_shape_ok(int M, int K, int N, int r, int n_requests)
{
    return M >= 1 && M <= kMaxRows && K >= 8 && K % 8 == 0 && K <= kMaxCols && N >= 8 && N % 8 == 0 && N <= kMaxCols &&
           r >= 8 && r % 8 == 0 && r <= 128 && n_requests >= 1 && n_requests <= (1 << 20);
}

size_t muxq_lora_workspace_bytes(int M, int K, int N, int r, int n_requests)
{
    return lora_shape_ok(M, K, N, r, n_requests) ? muxq::lora_workspace_bytes(M, K, N, r, n_requests) : 0;
}

int muxq_lora(const void *X, int M, int K, int ldx, const void *A, const void *B, const float *scales,
              int n_adapters, int r, const int32_t *starts, const int32_t *adapters, int n_requests,
              const void *Y, int ldy, int N, void *out, int ldo, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!X || !A || !B || !scales || !starts || !adapters || !Y || !out) return MUXQ_ERR_NULL;
    if (!lora_shape_ok(M, K, N, r, n_requests) || n_adapters < 1 || bad_ld(ldx, K) || bad_ld(ldy, N) || bad_ld(ldo, N) ||
        ldx > kMaxLd || ldy > kMaxLd || ldo > kMaxLd)
        return MUXQ_ERR_SHAPE;
    if (!aligned(X, 16) || !aligned(A, 16) || !aligned(B, 16) || !aligned(Y, 16) || !aligned(out, 16) || !aligned(scales, 4) ||
        !aligned(starts, 4) || !aligned(adapters, 4))
        return MUXQ_ERR_ALIGN;
    if (share(X, ldx, K, out, ldo, N, M) || ((Y != out || ldy != ldo) && share(Y, ldy, N, out, ldo, N, M))) return MUXQ_ERR_PARAM;
    const size_t need = muxq::lora_workspace_bytes(M, K, N, r, n_requests);
    if (need > 0) {
        if (!workspace) return MUXQ_ERR_NULL;
        if (!aligned(workspace, 16)) return MUXQ_ERR_ALIGN;
        if (workspace_bytes < need) return MUXQ_ERR_WORKSPACE;
    }
    muxq::LoraArgs g{};
    g.x = (const _Float16 *)X;
    g.a = (const _Float16 *)A;
    g.b = (const _Float16 *)B;
    g.y = (const _Float16 *)Y;
    g.out = (_Float16 *)out;
    g.scales = scales;
    g.starts = starts;
    g.adapters = adapters;
    g.M = M; g.K = K; g.N = N; g.r = r;
    g.n_adapters = n_adapters; g.n_requests = n_requests;
    g.ldx = ldx; g.ldy = ldy; g.ldo = ldo;
    g.h = (float *)workspace;
    MUXQ_TRY(muxq::launch_lora(g, (hipStream_t)stream));
    return MUXQ_OK;
}

static bool norm_shape_ok(int M, int K) { return M >= 1 && M <= kMaxRows && K >= 8 && K % 8 == 0 && K <= 32768; }

int muxq_norm_slabs(int M, int K) { return norm_shape_ok(M, K) ? muxq::norm_slab_rows(M) : 0; }

size_t muxq_norm_scratch_bytes(int M, int K) { return norm_shape_ok(M, K) ? muxq::norm_scratch_bytes(M, K, kpad(K)) : 0; }

int muxq_norm(const void *X, int M, int K, int ldx, const void *R, int ldr, float r_scale, const void *post_w,
              const void *post_b, const void *gate, int ldg, const void *w, const void *b, int kind, float eps,
              void *R_out, int ldro, void *Y, int ldy, void *slabs, void *scratch, size_t scratch_bytes, void *stream)
{
    if (!X || !w || !Y || (post_b && !post_w)) return MUXQ_ERR_NULL;
    if (!norm_shape_ok(M, K) || bad_ld(ldx, K) || bad_ld(ldy, K) || (R && bad_ld(ldr, K)) || (R_out && bad_ld(ldro, K)) ||
        (gate && ldg != 0 && bad_ld(ldg, K)))
        return MUXQ_ERR_SHAPE;
    if ((kind != MUXQ_NORM_LAYER && kind != MUXQ_NORM_RMS) || !(eps >= 0.0f) || eps > 3.4e38f || !(fabsf(r_scale) <= 3.4e38f)) return MUXQ_ERR_PARAM;
    for (const void *p : {X, R, post_w, post_b, gate, w, b, (const void *)R_out, (const void *)Y, (const void *)slabs})
        if (p && !aligned(p, 16)) return MUXQ_ERR_ALIGN;
    if (R_out && share(R_out, ldro, K, Y, ldy, K, M)) return MUXQ_ERR_PARAM;
    // in place, or apart (a row is read whole before it is written, other rows are not waited for)
    struct { void *p; int ld; } outs[2] = {{Y, ldy}, {R_out, ldro}};
    for (const auto &o : outs) {
        if (!o.p) continue;
        if ((X != o.p || ldx != o.ld) && share(X, ldx, K, o.p, o.ld, K, M)) return MUXQ_ERR_PARAM;
        if (R && (R != o.p || ldr != o.ld) && share(R, ldr, K, o.p, o.ld, K, M)) return MUXQ_ERR_PARAM;
        if (gate && ldg != 0 && share(gate, ldg, K, o.p, o.ld, K, M)) return MUXQ_ERR_PARAM;
    }
    muxq::NormArgs n{};
    n.k_pad = kpad(K);
    if (slabs) {
        const size_t need = muxq::norm_scratch_bytes(M, K, n.k_pad);
        if (need > 0) {
            if (!scratch) return MUXQ_ERR_NULL;
            if (!aligned(scratch, 16)) return MUXQ_ERR_ALIGN;
            if (scratch_bytes < need) return MUXQ_ERR_WORKSPACE;
        }
    }
    n.x = (const _Float16 *)X;
    n.res = (const _Float16 *)R;
    n.post_w = (const _Float16 *)post_w;
    n.post_b = (const _Float16 *)post_b;
    n.gate = (const _Float16 *)gate;
    n.w = (const _Float16 *)w;
    n.b = (const _Float16 *)b;
    n.r_out = (_Float16 *)R_out;
    n.y = (_Float16 *)Y;
    n.M = M; n.K = K; n.ldx = ldx; n.ldr = ldr; n.ldg = ldg; n.ldro = ldro; n.ldy = ldy;
    n.r_scale = r_scale;
    n.eps = eps;
    n.slabs = (uint16_t *)slabs;
    n.scratch = (uint16_t *)scratch;
    MUXQ_TRY(muxq::launch_norm(n, kind == MUXQ_NORM_RMS, (hipStream_t)stream));
    return MUXQ_OK;
}

}  // extern "C"
