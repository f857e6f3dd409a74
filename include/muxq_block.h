/*
 * muxq_block.h -- C ABI of what stands between the quantised projections of muxq.h when a block
 * of a decoder serves requests: the paged key-value cache and the attention of one new token that
 * reads it, low-rank adapters beside a projection that many requests share, and the norms around
 * the residual stream, which hand the channel maxima to the next quantised layer; and what a sequence with several new
 * tokens needs: attention of prompts, within a sliding window if asked, attention of the nodes of a drafted tree, the
 * verification of drafted tokens, and pages and tokens moved within the cache.
 *
 * Conventions are those of muxq.h: DEVICE pointers owned by the caller; nothing is allocated, freed
 * or synchronised; every call only enqueues kernels on `stream` and may be captured into a graph (the first
 * call on a device after muxq_init(), which loads the kernels);
 * the return value is a muxq_status, and on any status other than MUXQ_OK (MUXQ_ERR_HIP apart)
 * nothing has been enqueued.  (MUXQ_ERR_HIP is also what a call gives that would take a launch of 2^32 threads or more, some
 * 2^34 elements.)  Activations are fp16, rows contiguous, with row strides in elements
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

/* The other way: rows of the cache as fp16 (codes times scale in binary32, rounded once), e.g. a
 * cached prefix for a caller's own use of it.  K_out, V_out: M rows of
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

/* ---- several new tokens of a sequence --------------------------------------------------------
 * The rows of sequence s are starts[s] <= m < starts[s + 1] (int32 [S + 1], ascending, clamped to [0, M]); n of them are its
 * n new tokens, which stand in the cache already, as the last n of its lengths[s] tokens: row starts[s] + i is token
 * lengths[s] - n + i.  A length above max_length counts as max_length.  A sequence with more rows than max_new (max_nodes)
 * counts as one without rows.  Rows in no sequence are not written.  S <= 65535, M <= 2^24, and the
 * smaller of M and max_new times n_heads at most 2^30 for the attention.
 *
 * Attention of these tokens over the cache:
 *   O[m][h] = sum_t softmax_t(scale * Q[m][h] . K[t][h / g]) V[t][h / g]   over the tokens t that m sees,
 * g = n_heads / n_kv_heads (n_heads % n_kv_heads == 0).  Q, O: M rows of n_heads * head_dim fp16, row strides ldq, ldo, which share
 * no memory.  Cache, table and pages as for muxq_paged_attention; tokens of a page outside [0, n_blocks) are left out.
 * muxq_window_attention: token p = lengths[s] - n + i sees t <= p; with window > 0 of these t > p - window and t < sinks.
 *   (window 0: all; sinks counts only with a window.)  One row a sequence is the form for decoding.
 * muxq_tree_attention: the rows are the nodes of a tree (or forest), parents (int32 [M]) the parent of each as its number within the
 *   sequence, smaller than its own; anything else (-1) marks a root.  Node i sees all tokens before the
 *   tree (t < lengths[s] - n), itself and the nodes above it.  max_nodes <= 64.
 *   (There is no window: for a model with a sliding one this is its attention only while lengths[s] <= window.)
 * A row that sees nothing (a length below 1, pages outside the cache) is zeros.  What stands in places that a row
 * does not see, NaN and infinity included, has no influence on it; infinite and NaN values in places that it sees
 * come out as the formula has them, with weights that are never quite 0, and scores that are all -infinity give NaN (0 / 0).
 * Arithmetic: products of fp16 with binary32 sums; scales of codes multiply scores and weights; statistics of the softmax are
 * binary32; the weights enter the second product rounded to fp16: each is off by at most 2^-11 of itself, or 2^-31 of the row's
 * largest where that is more (with codes 2^-30 of the largest weight times the largest scale that the row sees).  Calls with max_new = 1 may take the
 * kernel of muxq_paged_attention, by their sizes, whose weights have 22 bits.
 * max_length: the host's bound on lengths[], 1 <= max_length <= ld_table * block_size, at most 2^26; max_new and max_nodes: the
 * host's bound on the rows of a sequence.  The work is divided by them, as if each sequence had that many rows: a long chunk of a prompt and
 * many single tokens are faster as two calls (2048 tokens beside 256 single ones of 500 to 8000: 1.9 ms, in two calls 0.83).
 * workspace: ..._workspace_bytes(...) bytes, 256-byte aligned, content undefined on entry; enough for every call with S, max_new
 * (max_nodes), max_length, window and sinks no larger (a window of 0 is the largest); NULL where that is 0.  Calls that share one must
 * not overlap in time. */
size_t muxq_window_attention_workspace_bytes(int S, int n_heads, int n_kv_heads, int head_dim, int max_new, int max_length,
                                             int window, int sinks);
int muxq_window_attention(const void *Q_fp16, int M, int n_heads, int ldq, const muxq_kv_cache *cache,
                          const int32_t *block_table, int ld_table, const int32_t *starts, const int32_t *lengths, int S,
                          int max_new, int max_length, int window, int sinks, float scale, void *O_fp16, int ldo,
                          void *workspace, size_t workspace_bytes, void *stream);
size_t muxq_tree_attention_workspace_bytes(int S, int n_heads, int n_kv_heads, int head_dim, int max_nodes, int max_length);
int muxq_tree_attention(const void *Q_fp16, int M, int n_heads, int ldq, const muxq_kv_cache *cache,
                        const int32_t *block_table, int ld_table, const int32_t *starts, const int32_t *lengths,
                        const int32_t *parents, int S, int max_nodes, int max_length, float scale, void *O_fp16, int ldo,
                        void *workspace, size_t workspace_bytes, void *stream);

/* Drafted tokens against the target's probabilities.  Each sequence has a tree of n <= max_nodes <= 64 nodes (starts, parents as
 * above; a chain is a tree), whose node 0 is its last token and stands already; tokens[m] (int32 [M]) is the token of node m.  target: float
 * [M][V] (row stride ldt), row m what the target says after node m; draft: float [M][V] (ldd), row m what the children of
 * node m were drawn from, each by itself and with replacement (for others, drawn without replacement for instance, what comes out is not distributed
 * as the target), NULL: they were chosen without drawing (a probability of 1).  uniforms: float [M] in [0, 1).
 * From v = 0, r = target[v], Z = 1 the children c of v, ascending, are tried:
 *   accepted if uniforms[c] * draft[v][x_c] * Z < r[x_c]: then v = c, and on with its children;
 *   otherwise r = max(r / Z - draft[v], 0), Z = sum r, and on with the next one.  If Z is 0, no other child is accepted and r = target[v].
 * Where no child is left the next token is the smallest t with r_0 + ... + r_t > uniforms[node 0] * (sum of r) (the last one with
 * r_t > 0 if there is none, -1 if the sum is not positive).  All in binary64, so that the order of sums does not matter.
 * uniforms NULL (draft is not read): the child whose token is the largest of target[v], the lowest index of equal ones (NaN counts as -infinity),
 * is accepted, the first of several; where there is none that token is the next.
 * A drafted token outside [0, V) is not accepted and leaves r as it is.  Probabilities need not sum to 1; infinite, NaN or
 * negative ones give unspecified tokens within [-1, V).
 * path: int32 [M], the accepted nodes of sequence s, as numbers within it, at starts[s] + j (0 first), -1 behind them; counts: int32 [S], how
 * many; next_token: int32 [S]; the three share no memory with each other or with what is read.  A sequence without rows gives a count of 0 and a token of -1.  1 <= V <= 2^22, strides
 * below 2^31. */
int muxq_verify_tree(const float *target, int ldt, const float *draft, int ldd, int M, int V, const int32_t *tokens,
                     const int32_t *parents, const float *uniforms, const int32_t *starts, int S, int max_nodes,
                     int32_t *path, int32_t *counts, int32_t *next_token, void *stream);

/* Pages dst[i] of the cache become copies of pages src[i] (int32 [n], n <= 2^24): keys, values and scales.  A pair with a page outside
 * [0, n_blocks) is left out.  A page that two pairs write, or that one pair writes and another reads, has unspecified content. */
int muxq_kv_copy(const int32_t *src, const int32_t *dst, int n, const muxq_kv_cache *cache, void *stream);

/* The accepted nodes of each tree become the first of its new tokens in the cache: token lengths[s] - n + j becomes what token
 * lengths[s] - n + path[starts[s] + j] was, for j < counts[s] (at most n <= max_nodes <= 64), keys, values and scales, as if
 * all were read before any is written.  The sequence is then lengths[s] - n + counts[s] tokens long.  Arguments as
 * muxq_verify_tree and the attention take and give them.  Numbers outside [0, n), tokens outside the table (ld_table * block_size
 * tokens) and pages outside the cache are left out.  No two sequences may share the pages of their new tokens. */
int muxq_kv_compact(const int32_t *path, const int32_t *counts, const int32_t *starts, const int32_t *lengths,
                    const int32_t *block_table, int ld_table, int M, int S, int max_nodes, const muxq_kv_cache *cache,
                    void *stream);

#ifdef __cplusplus
}
#endif
#endif /* MUXQ_BLOCK_H */
