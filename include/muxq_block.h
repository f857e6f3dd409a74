/*
 * muxq_block.h -- C ABI of what stands between the quantised projections of muxq.h when a block
 * of a decoder serves requests: the paged key-value cache and the attention of one new token that
 * reads it, low-rank adapters beside a projection that many requests share, and the norms around
 * the residual stream, which hand the channel maxima to the next quantised layer.
 *
 * Conventions are those of muxq.h: DEVICE pointers owned by the caller; nothing is allocated, freed
 * or synchronised; every call only enqueues kernels on `stream` and may be captured into a graph (the first
 * call on a device after muxq_init(), which loads the kernels);
 * the return value is a muxq_status, and on any status other than MUXQ_OK (MUXQ_ERR_HIP apart)
 * nothing has been enqueued.  Activations are fp16, rows contiguous, with row strides in elements
 * that are multiples of 8, from 16-byte aligned pointers.  Sums, maxima and softmax
 * statistics are binary32.  Results do not depend on the order in which workgroups run.
 * Index arrays (slots, positions, block tables, lengths, request starts, adapter numbers) are read
 * on the device; values out of range are never used as an address, and what they give instead
 * stands at each entry point.
 */
#ifndef MUXQ_BLOCK_H
#define MUXQ_BLOCK_H

#include "muxq.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- paged key-value cache -----------------------------------------------------------------
 * Keys and values of all sequences live in pages of block_size tokens.  Element (page p, head h,
 * token t of the page, dimension i) of `k` sits at p * ld_block + h * ld_head + t * ld_token + i
 * (strides in elements, 64-bit, the same for `v`): heads before tokens or tokens before heads, or
 * pages that hold keys and values side by side, as the caller likes.  A page's keys (and values) of
 * one head are read together, so heads before tokens reads longer runs of memory.
 * type: MUXQ_KV_FP16, or MUXQ_KV_INT8: symmetric abs-max codes in [-127, 127] (Eq. 1) with one
 * scale per token and head, k_scale / v_scale float [n_blocks][n_kv_heads][block_size] (contiguous).
 * Rules: block_size a power of two, 8 to 256; head_dim a multiple of 16, 16 to 256; n_kv_heads >= 1;
 * n_blocks >= 1, n_blocks * block_size < 2^31; strides positive multiples of 16, ld_token and ld_head
 * >= head_dim, and ld_block at least what one page spans. */
typedef enum { MUXQ_KV_FP16 = 0, MUXQ_KV_INT8 = 1 } muxq_kv_type;
typedef struct {
    void *k, *v;
    float *k_scale, *v_scale;   /* NULL with MUXQ_KV_FP16 */
    int32_t type;
    int32_t n_blocks, block_size, n_kv_heads, head_dim;
    int32_t reserved;           /* 0 */
    int64_t ld_block, ld_head, ld_token;
} muxq_kv_cache;

/* Keys and values of M new tokens to their slots of the cache, rotated by position on the way.
 * K, V: M rows of n_kv_heads * head_dim fp16 (row strides ldk, ldv); Q: M rows of n_heads * head_dim
 * (NULL: no queries).  Typically three column ranges of one projection's output.
 * slots: int32 [M], slot = page * block_size + token of the page.  A token whose slot lies outside
 * [0, n_blocks * block_size) is not stored (-1 for the padding of a batch); two tokens with the same slot
 * leave parts of both there.
 * Rotation: cos_sin float [n_positions][rot_dim], a row holds rot_dim / 2 cosines, then as many sines;
 * rot_dim a multiple of 8, 0 (no rotation, cos_sin and positions may be NULL) to head_dim.  Pair j of
 * a head is (x[j], x[j + rot_dim / 2]), with interleaved != 0 (x[2j], x[2j + 1]):
 *   (a, b) -> (a cos_j - b sin_j, b cos_j + a sin_j)   in binary32, products and sum rounded one by one;
 * the other dimensions and V stay as they are.  A token whose position lies outside [0, n_positions)
 * is not rotated and not stored.
 * Q_out: M rows of n_heads * head_dim, row stride ldqo: the rotated queries, rounded once to fp16;
 * may be Q itself (same stride).
 * Stored: fp16 values rounded once; or codes clamp(rne(x * (127 / max|x|))) of the rotated binary32
 * values with scale max|x| / 127 over the head (0 and codes 0 where all are 0; a head that holds
 * NaN or infinity gives unspecified codes). */
int muxq_kv_append(const void *K_fp16, const void *V_fp16, int M, int ldk, int ldv, const void *Q_fp16,
                   int n_heads, int ldq, void *Q_out_fp16, int ldqo, const int32_t *slots,
                   const int32_t *positions, const float *cos_sin, int n_positions, int rot_dim,
                   int interleaved, const muxq_kv_cache *cache, void *stream);

/* The other way: rows of the cache as fp16 (codes times scale in binary32, rounded once), e.g. the
 * cached prefix of a prompt for a caller's own attention over it (there is none for prompts here).  K_out, V_out: M rows of
 * n_kv_heads * head_dim, row strides ldk, ldv.  Rows of slots outside the cache are zeros. */
int muxq_kv_gather(const int32_t *slots, int M, const muxq_kv_cache *cache, void *K_out_fp16, int ldk,
                   void *V_out_fp16, int ldv, void *stream);

/* Attention of one new token of each of S sequences over the cache:
 *   O[s][h] = sum_t softmax_t(scale * Q[s][h] . K[t][h / g]) V[t][h / g],  t < lengths[s],
 * g = n_heads / n_kv_heads queries to each key-value head (n_heads % n_kv_heads == 0).  Q, O: S rows
 * of n_heads * head_dim fp16, row strides ldq, ldo; O may be Q itself (same stride).  Token t of sequence s is token t % block_size of
 * page block_table[s * ld_table + t / block_size]; table entries are int32.  lengths: int32 [S].
 * A length below 1 (an idle place of the batch) gives a row of zeros, one above max_length counts as
 * max_length.  Tokens of a page outside [0, n_blocks) are left out as if masked.  What the cache holds
 * beyond a sequence's length, NaN included, has no influence.  max_length: the host's bound on
 * lengths[], 1 <= max_length <= ld_table * block_size, at most 2^26 (S <= 65535); the work is divided
 * by it, so a bound near
 * the longest sequence is best.
 * Arithmetic: products of fp16 (codes are exact in fp16) with binary32 sums; the scale of a code's key multiplies its score; the
 * softmax weights enter the second product as two 16-bit parts: 22 bits, and a token's weight is cut to whole
 * multiples of 2^-32 of the largest (with codes weight times scale, to multiples of 2^-31 of the largest weight times the largest scale).
 * Values (and scales of values) that are infinite or NaN, and a sequence whose scores are all -infinity (0 / 0), come out as the formula has
 * them.
 * workspace: muxq_paged_attention_workspace_bytes(...) bytes, 256-byte aligned, content undefined on
 * entry; enough for every call with S and max_length no larger; NULL where that is 0.  Calls that share one
 * must not overlap in time. */
size_t muxq_paged_attention_workspace_bytes(int S, int n_heads, int n_kv_heads, int head_dim, int max_length);
int muxq_paged_attention(const void *Q_fp16, int S, int n_heads, int ldq, const muxq_kv_cache *cache,
                         const int32_t *block_table, int ld_table, const int32_t *lengths, int max_length,
                         float scale, void *O_fp16, int ldo, void *workspace, size_t workspace_bytes,
                         void *stream);

/* Low-rank adapters of many requests beside a projection that they share:
 *   out[m] = Y[m] + scales[i] * (X[m] A_i^T) B_i^T,   i the adapter of m's request,
 * in binary32, rounded once to fp16; X A_i^T enters the second product as two 16-bit parts of its row (22 bits of
 * the row's largest); infinities and NaN come out as the formula has them.  X: M x K (the projection's input), Y: M x N (its output), out:
 * M x N, may be Y itself (same stride) but share no memory with X.  A: fp16 [n_adapters][r][K], B: fp16
 * [n_adapters][N][r], scales: float [n_adapters]; smaller ranks are padded with zeros.
 * Requests are runs of rows: request q has the rows starts[q] <= m < starts[q + 1] (int32 [n_requests + 1],
 * ascending, starts[0] = 0, starts[n_requests] = M) and the adapter adapters[q] (int32; outside
 * [0, n_adapters), e.g. -1: none, its rows are copied from Y).  Rows in no request are not written; bounds
 * are clamped to [0, M].
 * workspace: muxq_lora_workspace_bytes(...) bytes, 16-byte aligned, content undefined on entry; enough for every call with
 * M, K, r and n_requests no larger; NULL where that is 0.  Calls that share one must not overlap in time.
 * Rules: K, N, r multiples of 8, r <= 128, K, N <= 2^21, M <= 2^24, row strides <= 2^25, n_adapters >= 1,
 * 1 <= n_requests <= 2^20. */
size_t muxq_lora_workspace_bytes(int M, int K, int N, int r, int n_requests);   /* 0 on bad shapes, and where none is needed */
int muxq_lora(const void *X_fp16, int M, int K, int ldx, const void *A_fp16, const void *B_fp16,
              const float *scales, int n_adapters, int r, const int32_t *starts, const int32_t *adapters,
              int n_requests, const void *Y_fp16, int ldy, int N, void *out_fp16, int ldo, void *workspace,
              size_t workspace_bytes, void *stream);

/* The step between two blocks: the norm behind a block, its gate, the residual stream, and the norm in
 * front of the next block, row by row:
 *   t = post-norm(X[m]) if post_w is given, else X[m]
 *   r = r_scale * R[m] + gate * t        (R NULL: no stream yet, r = gate * t; gate NULL: 1)
 *   R_out[m] = fp16(r),  Y[m] = fp16(norm(r))
 * norm(v) = (v - mean(v)) / sqrt(var(v) + eps) * w + b with MUXQ_NORM_LAYER (var the mean square
 * deviation), v / sqrt(mean(v^2) + eps) * w + b with MUXQ_NORM_RMS; b may be NULL.  Everything in between is
 * binary32: Y is formed from r before its rounding.  w, b, post_w, post_b: fp16 [K].  gate: fp16, row m at
 * gate + m * ldg; ldg = 0 gives all rows the same [K].  R_out may be NULL.  In place: R_out may be R or X,
 * Y may be X or R (same stride), R_out and Y share no memory.
 * Hand-over to the next muxq_linear_opts / muxq_linear_static call on Y (same M and K, absmax_ready = 1):
 * slabs (may be NULL) is the absmax_partial region of its workspace; it receives
 * muxq_norm_slabs(M, K) rows of k_pad fp16 column maxima (absmax_slabs = that count): up to 64 tokens
 * the magnitudes of each, else one row of the maxima over all tokens.  scratch:
 * muxq_norm_scratch_bytes(M, K) bytes, 16-byte aligned, content undefined; NULL where that is 0 or slabs
 * is NULL.  Rules: K % 8 == 0, K <= 32768, M <= 2^24, eps >= 0, finite r_scale. */
typedef enum { MUXQ_NORM_LAYER = 0, MUXQ_NORM_RMS = 1 } muxq_norm_kind;
int muxq_norm_slabs(int M, int K);                 /* 0 on bad shapes */
size_t muxq_norm_scratch_bytes(int M, int K);      /* 0 on bad shapes, and where none is needed */
int muxq_norm(const void *X_fp16, int M, int K, int ldx, const void *R_fp16, int ldr, float r_scale,
              const void *post_w, const void *post_b, const void *gate, int ldg, const void *w, const void *b,
              int kind, float eps, void *R_out_fp16, int ldro, void *Y_fp16, int ldy, void *slabs,
              void *scratch, size_t scratch_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* MUXQ_BLOCK_H */
