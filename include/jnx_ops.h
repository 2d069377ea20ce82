/*
 * Stage-level entry points of libjnx.so: each step of jnx_backbone_forward
 * on its own, for stage-wise parity tests and per-kernel measurement.  The
 * conventions of jnx.h apply (borrowed pointers, asynchronous on `stream`,
 * host-checked arguments, bf16 as uint16_t bit patterns, row-major).
 */
#ifndef JNX_OPS_H
#define JNX_OPS_H

#include "jnx.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Epilogues of jnx_op_gemm. */
#define JNX_EPI_BF16 0  /* out bf16 [M, ldo] = C */
#define JNX_EPI_F32 1   /* out fp32 [M, ldo] = C */
#define JNX_EPI_RESID 2 /* out fp32 [M, ldo] += C (residual stream update) */
#define JNX_EPI_GLU 3   /* W holds 128-row blocks alternating gate / up rows;
                           out bf16 [M, ldo] columns j < N/2 = act(C_gate) * C_up */
#define JNX_EPI_ROPE 4  /* out bf16 [M, ldo] = C with rotate-half RoPE at
                           position pos[row] on columns < rope_cols */
#define JNX_EPI_GLU_SAVE 6 /* W as for JNX_EPI_GLU; out bf16 [M, ldo], N columns in W's
                              packed order: u act'(g) in each gate column, act(g) in each
                              up column (the GLU backward's multipliers) */

/* The canonical packing step (§4.3: the VLAFeature is where the tenants'
 * samples are concatenated): x[t, :] = fp32 of vision[gather_src[t]] or of
 * text_table[text_ids[-gather_src[t] - 1]].  x is [n_tokens, d] fp32.  A
 * source index outside its buffer or a text id outside [0, vocab) writes a
 * zero row and JNX_ERR_DEVICE_BOUNDS to *status (device int, may be NULL). */
jnx_status jnx_op_pack(const jnx_group* g, const uint16_t* vision, int64_t n_vision_rows,
                       const int32_t* text_ids, int64_t n_text, const uint16_t* text_table,
                       int32_t vocab, int32_t d, float* x, int32_t* status, void* stream);

/* out[M, d] bf16 = x / sqrt(mean(x^2) + eps) * gamma, fp32 statistics;
 * d in {256, 512, 1024, 2048, 4096}. */
jnx_status jnx_op_rmsnorm(const float* x, const uint16_t* gamma, float eps, int32_t M, int32_t d,
                          uint16_t* out, void* stream);

/* Workspace bytes of jnx_op_gemm with JNX_EPI_ROPE for positions < max_pos. */
size_t jnx_op_gemm_workspace_bytes(int32_t max_pos, int32_t head_dim);

/* C[M, N] = A[M, K] W[N, K]^T on the tcgen05 tensor cores, fp32 accumulate,
 * then the epilogue.  N % 256 == 0, K % 64 == 0, A/W rows 16-byte aligned.
 * out has rows of ldo elements (bf16, or fp32 for JNX_EPI_F32 / RESID),
 * ldo >= the output width (N, or N / 2 for JNX_EPI_GLU), 16-byte aligned
 * rows and base, else JNX_ERR_INVALID_ARG.
 * pos/max_pos/rope_cols/head_dim/rope_theta are read for JNX_EPI_ROPE only
 * (workspace then holds the status word and the RoPE table; rope_cols a
 * multiple of head_dim within [0, N]; a position outside [0, max_pos) leaves
 * its row unrotated and records JNX_ERR_DEVICE_BOUNDS in the status word,
 * read by jnx_check_status(workspace)); act
 * (JNX_GLU_*) for JNX_EPI_GLU only.  workspace may be NULL otherwise. */
jnx_status jnx_op_gemm(const uint16_t* A, const uint16_t* W, int32_t M, int32_t N, int32_t K,
                       int32_t epilogue, void* out, int32_t ldo, const int32_t* pos,
                       int32_t max_pos, int32_t rope_cols, int32_t head_dim, float rope_theta,
                       int32_t act, void* workspace, size_t ws_bytes, void* stream);

/* Attention confined to each sample: for every sample s, head h,
 * out[t] = softmax(q_t K_s^T / sqrt(hd)) V_s over the sample's own tokens.
 * qkv [n_tokens, (H + 2 Hkv) hd] bf16 (q heads, then k heads, then v heads),
 * out [n_tokens, H hd] bf16; head_dim in {64, 128, 256}.  A wait that ran
 * out of time writes JNX_ERR_TIMEOUT to *status (device int, may be NULL). */
jnx_status jnx_op_attention(const uint16_t* qkv, int32_t n_tokens, int32_t n_heads,
                            int32_t n_kv_heads, int32_t head_dim, const int32_t* cu_seqlens,
                            int32_t n_samples, int32_t max_seqlen, uint16_t* out,
                            int32_t* status, void* stream);

/* Final RMSNorm and per-sample mean: pooled[s] = gamma * mean over the
 * sample's rows of x_t / sqrt(mean(x_t^2) + eps) (fp32), hidden[t] = bf16
 * of the normed row.  Either output may be NULL. */
jnx_status jnx_op_final_pool(const float* x, const uint16_t* gamma, float eps,
                             const int32_t* cu_seqlens, int32_t n_samples, int32_t d,
                             float* pooled, uint16_t* hidden, void* stream);

/* ---- stages of the adapter backward (jnx_backbone_backward_lora) ---- */

/* jnx_op_attention that also writes lse [n_tokens, H] fp32: each query
 * row's log2-sum-exp of its scaled scores, log2(sum_j 2^(s_j log2(e) /
 * sqrt(hd))), from which the backward recomputes the probabilities. */
jnx_status jnx_op_attention_lse(const uint16_t* qkv, int32_t n_tokens, int32_t n_heads,
                                int32_t n_kv_heads, int32_t head_dim, const int32_t* cu_seqlens,
                                int32_t n_samples, int32_t max_seqlen, uint16_t* out, float* lse,
                                int32_t* status, void* stream);

/* The attention backward's prologue: dO [n_tokens, H hd] bf16 = bf16(datt)
 * (fp32) and D [n_tokens, H] = per head, the sum over its hd columns of
 * dO * att (att = the forward's output, bf16). */
jnx_status jnx_op_attention_backward_prep(const float* datt, const uint16_t* att, int32_t n_tokens,
                                          int32_t n_heads, int32_t head_dim, uint16_t* dO,
                                          float* D, void* stream);

/* Workspace bytes of jnx_op_attention_backward. */
size_t jnx_op_attention_backward_workspace_bytes(int32_t n_tokens, int32_t max_seqlen,
                                                 int32_t head_dim);

/* Gradients of jnx_op_attention with respect to its input qkv, given dO,
 * the forward's lse and D (jnx_op_attention_backward_prep): for query head
 * h on K/V head g, P = softmax(q k^T / sqrt(hd)) inside each sample,
 * dv_g += P^T dO_h, dS = P * (dO_h v_g^T - D), dq_h = dS k_g / sqrt(hd),
 * dk_g += dS^T q_h / sqrt(hd).  qkv holds q and k after RoPE; dqkv
 * [n_tokens, (H + 2 Hkv) hd] bf16 receives the gradients of the pre-RoPE
 * projections (dq, dk rotated back by the rotate-half RoPE of theta at
 * pos[t]; dv as is).  h_cu_seqlens is the host copy of cu_seqlens (the work
 * list is built from it).  A wait that ran out of time writes
 * JNX_ERR_TIMEOUT to *status. */
jnx_status jnx_op_attention_backward(const uint16_t* qkv, const uint16_t* dO, const float* lse,
                                     const float* D, int32_t n_tokens, int32_t n_heads,
                                     int32_t n_kv_heads, int32_t head_dim,
                                     const int32_t* cu_seqlens, const int32_t* h_cu_seqlens,
                                     int32_t n_samples, int32_t max_seqlen, const int32_t* pos,
                                     float rope_theta, uint16_t* dqkv, void* workspace,
                                     size_t ws_bytes, int32_t* status, void* stream);

/* RMSNorm backward: with s = rsqrt(mean(x^2) + eps) per row,
 * dx = dres + s gamma dn - x s^3 mean(gamma dn x) (fp32; dres may be NULL
 * or dx itself) and dx_bf = bf16(dx) when not NULL.  d % 128 == 0. */
jnx_status jnx_op_rms_backward(const float* x, const uint16_t* gamma, float eps, const float* dn,
                               const float* dres, int32_t M, int32_t d, float* dx,
                               uint16_t* dx_bf, void* stream);

/* The feed-forward backward's first GEMM with the GLU backward fused:
 * dm[M, F] = A[M, K] W[F, K]^T is the gradient at act(g) * u; gu [M, 2F]
 * bf16 holds on entry what JNX_EPI_GLU_SAVE wrote (u act'(g) in the gate
 * columns, act(g) in the up columns of the packed order, 128-column blocks
 * alternating gate and up) and on return dg = dm u act'(g) in the gate
 * columns, du = dm act(g) in the up columns.  F % 256 == 0, K % 64 == 0.
 * act is not read (the multipliers already hold the activation). */
jnx_status jnx_op_gemm_glu_backward(const uint16_t* A, const uint16_t* W, int32_t M, int32_t F,
                                    int32_t K, uint16_t* gu, int32_t act, void* stream);

/* The feed-forward backward's GLU step with the gate/up GEMM recomputed
 * (what jnx_backbone_backward_lora runs per block): dm[M, F] = dy[M, d]
 * w_down_t[F, d]^T is the gradient at act(g) * u; it is stored bf16 in the
 * up columns of gu [M, 2F] (packed order: 128-column blocks alternating
 * gate and up), then the gate/up GEMM g|u = n2[M, d] w_gu[2F, d]^T (w_gu in
 * the packed order of jnx_pack_gate_up) leaves dg = dm u act'(g) in the gate
 * columns and du = dm act(g) in the up columns, bf16.  gu needs no content
 * on entry.  F % 256 == 0 (the GEMM's 256-column tiles), d % 64 == 0, gu
 * 16-byte aligned, act a JNX_GLU_* value (JNX_ERR_INVALID_ARG otherwise). */
jnx_status jnx_op_ffn_glu_backward(const uint16_t* dy, const uint16_t* w_down_t,
                                   const uint16_t* n2, const uint16_t* w_gu, int32_t M, int32_t F,
                                   int32_t d, int32_t act, uint16_t* gu, void* stream);

/* The fused QKV projection + RoPE of jnx_op_gemm (JNX_EPI_ROPE) for callers
 * that cannot allocate device memory — e.g. a plugin in a serving process
 * whose pool owns every device allocation, or a batching worker that must
 * not call cudaMalloc between requests because it can stall the device.
 * The paper has no counterpart: this is a deployment variant of the library.
 * The caller passes inputs and outputs only; the status word and the RoPE
 * table live in a fixed file-scope device array inside the library (every
 * GPU that loads the library holds it until exit; nothing is allocated).
 * Limits: max_pos * head_dim / 2 <= JNX_NOALLOC_MAX_ROPE_ENTRIES, otherwise
 * JNX_ERR_UNSUPPORTED before any launch.  Host-detected errors (null
 * pointers, head_dim not 64/128/256, rope_cols not a multiple of head_dim
 * within [0, N], ldo < N, out or its rows not 16-byte aligned) return
 * JNX_ERR_INVALID_ARG before any launch with nothing written.  A position
 * outside [0, max_pos) is a device-detected error: its row is written
 * unrotated and JNX_ERR_DEVICE_BOUNDS is recorded in the array's status
 * word (read it with jnx_op_gemm_rope_noalloc_status).
 * The first call on a device looks up the array's address (make it before
 * any stream capture).  All calls on a device share the array: each clears
 * the status word and rewrites the table it reads, and calls that overlap on
 * the GPU race.  Arguments and results otherwise as jnx_op_gemm. */
#define JNX_NOALLOC_MAX_ROPE_ENTRIES (1 << 19)
jnx_status jnx_op_gemm_rope_noalloc(const uint16_t* A, const uint16_t* W, int32_t M, int32_t N,
                                    int32_t K, uint16_t* out, int32_t ldo, const int32_t* pos,
                                    int32_t max_pos, int32_t rope_cols, int32_t head_dim,
                                    float rope_theta, void* stream);

/* Reads and clears the status word of jnx_op_gemm_rope_noalloc's fixed
 * array on the current device, after the work queued on `stream` (it
 * synchronises the stream; allocates nothing).  Returns JNX_OK, or the
 * first error a kernel recorded since the last read or call (a call clears
 * it on entry): JNX_ERR_DEVICE_BOUNDS, JNX_ERR_TIMEOUT. */
jnx_status jnx_op_gemm_rope_noalloc_status(void* stream);

/* Diagnostics: two device routines of the hot path run on their own, so
 * tests can pin them.  Neither is part of the grouped path.
 *
 * y[i] = 2^x[i] by the polynomial exponential that the varlen attention's
 * softmax evaluates for one key pair in four (range reduction j = rint(x),
 * f = x - j, 2^f by the degree-3 minimax polynomial on [-0.5, 0.5], x
 * clamped at -126).  x, y: n device floats.  It stands for the softmax
 * probabilities 2^(s - m) of §5.2's shared backbone attention. */
jnx_status jnx_diag_ex2_poly(const float* x, float* y, int32_t n, void* stream);

/* One thread waits, through the library's bounded mbarrier wait, on a
 * barrier that completes (arrive != 0) or that nothing ever arrives on
 * (arrive == 0), giving up after limit_cycles SM clocks (0 < limit <= 2^31,
 * else JNX_ERR_INVALID_ARG before the launch).  A wait that gave up writes
 * JNX_ERR_TIMEOUT to *status (a device int) and the kernel returns; every
 * spin in the library's kernels behaves this way.  The paper has no
 * counterpart (failure detection of the kernels themselves). */
jnx_status jnx_diag_bounded_wait(int64_t limit_cycles, int32_t arrive, int32_t* status,
                                 void* stream);

/* ---- operators of text tenants ----
 * A tenant whose module reads and writes text (or actions as tokens) behind the
 * shared prefix: norms and rotations of queries and keys, causal attention of
 * packed prompts, attention of single tokens against a cache, and next-token
 * losses over the vocabulary.  `status` (device int, may be NULL) receives what a
 * kernel detects: JNX_ERR_DEVICE_BOUNDS, JNX_ERR_TIMEOUT; the caller clears it.
 * No call uploads from host memory, so each can be captured into a CUDA graph.
 * Workspaces are 16-byte aligned and serve one call at a time. */

/* Rows of attention heads, bf16: element c of head h of row t is
 * ptr[t * row_stride + h * head_stride + c].  ptr is 16-byte aligned and the
 * strides are multiples of 8 elements (JNX_ERR_INVALID_ARG otherwise). */
typedef struct {
    uint16_t* ptr;
    int64_t row_stride, head_stride;
} jnx_head_rows;

/* Norms of each query and key head with the position rotation.  head_dim in
 * {64, 128, 256}.  gamma_q / gamma_k [head_dim] bf16: a head row x becomes
 * x / sqrt(mean(x^2) + eps) * gamma first; NULL: no norm.  Then rotate-half RoPE
 * over up to four position axes: frequency i of head_dim / 2,
 * theta^(-2 i / head_dim), turns the pair (i, i + head_dim / 2) by the position on
 * the axis in whose section i lies (sections[0] frequencies belong to axis 0, the
 * next sections[1] to axis 1, ...); frequencies beyond the sections do not turn.
 * Positions count in full over the whole int32 range: an angle is off by 2^-50 of itself. */
typedef struct {
    int32_t n_heads, n_kv_heads, head_dim;
    int32_t n_axes, sections[4];
    float theta, eps;
    const uint16_t *gamma_q, *gamma_k;
} jnx_qk_rope;

/* A cache of keys and values, bf16: element c of head h of token t of slot s is
 * k[s * slot_stride + t * row_stride + h * head_stride + c], v alike; n_slots slots
 * of `room` tokens.  Alignment as jnx_head_rows. */
typedef struct {
    uint16_t *k, *v;
    int32_t n_slots, room;
    int64_t slot_stride, row_stride, head_stride;
} jnx_kv_cache;

/* q = rotated normed query heads, k = key heads of qkv [n_tokens, ldqkv] bf16 (q
 * heads, then k heads, then v heads, which are not read), at positions
 * pos [n_axes, n_tokens].  q and k may be qkv's own rows. */
jnx_status jnx_op_qk_norm_rope(const jnx_qk_rope* p, const uint16_t* qkv, int64_t ldqkv,
                               const int32_t* pos, int32_t n_tokens, const jnx_head_rows* q,
                               const jnx_head_rows* k, void* stream);

/* The same for new tokens of live sequences: token t's key and value heads go to
 * row at[t] of slot slot[t].  A row outside the cache is not written and reported. */
jnx_status jnx_op_qk_norm_rope_append(const jnx_qk_rope* p, const uint16_t* qkv, int64_t ldqkv,
                                      const int32_t* pos, int32_t n_tokens,
                                      const jnx_head_rows* q, const jnx_kv_cache* cache,
                                      const int32_t* slot, const int32_t* at, int32_t* status,
                                      void* stream);

/* Gradients: dqkv's query and key columns [n_tokens, ldqkv] from dq and dk (its value
 * columns are not written), and the norms' gains' gradients dgamma_q / dgamma_k
 * [head_dim] fp32 (overwritten; NULL where there is no norm).  dq and dk may be
 * dqkv's own rows.  Sums run in an order set by the sizes. */
size_t jnx_op_qk_norm_rope_backward_workspace_bytes(const jnx_qk_rope* p, int32_t n_tokens);
jnx_status jnx_op_qk_norm_rope_backward(const jnx_qk_rope* p, const uint16_t* qkv, int64_t ldqkv,
                                        const int32_t* pos, int32_t n_tokens,
                                        const jnx_head_rows* dq, const jnx_head_rows* dk,
                                        uint16_t* dqkv, float* dgamma_q, float* dgamma_k,
                                        void* workspace, size_t ws_bytes, void* stream);

/* Packed prompts.  Sequence s has query rows [cu_q[s], cu_q[s + 1]) and key rows
 * [cu_kv[s], cu_kv[s + 1]); its queries are the last of its positions, so row i of
 * Lq sees keys j < min(Lk, max(Lk - Lq + i + 1, prefix[s])).  A row that sees none
 * has output 0, log-sum-exp -inf and gradient 0.  The arrays are on the device, the
 * h_ ones the same on the host; prefix may be NULL (0).  items: the work list of
 * jnx_prompt_items for the same heads, on the device.  A list of other lengths or heads is
 * refused by its counts (JNX_ERR_INVALID_ARG); an entry that names no row or key of the
 * prompt, or a sequence beyond the rows and keys of the host's arrays, is left out and
 * reported. */
typedef struct {
    int32_t n_seqs;
    const int32_t *cu_q, *cu_kv, *prefix;
    const int32_t *h_cu_q, *h_cu_kv, *h_prefix;
    const int32_t* items;
    /* items of each pass, and parts that the gradients sum a key's rows in, at most: as
     * jnx_prompt_items sets them */
    int32_t n_forward, n_keys, n_queries, n_parts;
} jnx_prompt;

/* The work list of a prompt for a head layout: writes up to cap pairs of int32 to out
 * (NULL: none), sets p's n_forward, n_keys, n_queries, n_parts and returns the number of pairs,
 * the longest work first in each pass.  Negative: a jnx_status. */
int32_t jnx_prompt_items(jnx_prompt* p, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                         int32_t* out, int32_t cap);

/* out = softmax(q k^T / sqrt(head_dim)) v over what each row sees; query head h reads
 * key/value head h / (n_heads / n_kv_heads).  n_heads / n_kv_heads <= 64, head_dim in
 * {64, 128, 256}.  lse [rows, n_heads] fp32 (NULL: not written): log2 of the row's sum
 * of 2^(s log2(e) / sqrt(head_dim)).  rest is not used: NULL.  q, k, v are finite; other
 * sequences' rows may hold anything. */
jnx_status jnx_op_prompt_attention(const jnx_prompt* p, int32_t n_heads, int32_t n_kv_heads,
                                   int32_t head_dim, const jnx_head_rows* q,
                                   const jnx_head_rows* k, const jnx_head_rows* v,
                                   const jnx_head_rows* out, const jnx_head_rows* rest,
                                   float* lse, int32_t* status, void* stream);

/* Gradients of q, k and v from out's gradient dout, with the forward's out and lse (rest is
 * not used: NULL).  A row that sees one key has no gradient at its scores: exactly zero.  The
 * same bits whatever else is packed beside a sequence. */
size_t jnx_op_prompt_attention_backward_workspace_bytes(const jnx_prompt* p, int32_t n_heads,
                                                        int32_t n_kv_heads, int32_t head_dim);
jnx_status jnx_op_prompt_attention_backward(const jnx_prompt* p, int32_t n_heads,
                                            int32_t n_kv_heads, int32_t head_dim,
                                            const jnx_head_rows* q, const jnx_head_rows* k,
                                            const jnx_head_rows* v, const jnx_head_rows* out,
                                            const jnx_head_rows* rest, const float* lse,
                                            const jnx_head_rows* dout,
                                            const jnx_head_rows* dq, const jnx_head_rows* dk,
                                            const jnx_head_rows* dv, void* workspace,
                                            size_t ws_bytes, int32_t* status, void* stream);

/* One token of each of `batch` live sequences against its cache: sequence b's query
 * heads (row b of q) over the first n_cached[b] tokens of slot slot[b] (0: output 0).
 * A slot or length outside the cache is read as length 0 and reported.  The bits of a
 * sequence do not depend on the others. */
size_t jnx_op_decode_attention_workspace_bytes(int32_t batch, int32_t n_heads, int32_t head_dim);
jnx_status jnx_op_decode_attention(const jnx_kv_cache* cache, int32_t batch, int32_t n_heads,
                                   int32_t n_kv_heads, int32_t head_dim, const jnx_head_rows* q,
                                   const int32_t* slot, const int32_t* n_cached,
                                   const jnx_head_rows* out, void* workspace, size_t ws_bytes,
                                   int32_t* status, void* stream);

/* Next-token losses: loss[i] = log(sum_v exp(x_iv)) - x_i,targets[i] with logits
 * x = h w^T of h [n_rows, d] (row stride ldh) and w [vocab, d] (ldw), bf16; 0 where
 * targets[i] < 0.  A target >= vocab is reported and read as negative.  The logits are
 * never stored.  d and the strides are multiples of 8. */
size_t jnx_op_vocab_loss_workspace_bytes(int32_t n_rows, int32_t vocab, int32_t d);
jnx_status jnx_op_vocab_loss(const uint16_t* h, int64_t ldh, const uint16_t* w, int64_t ldw,
                             const int32_t* targets, int32_t n_rows, int32_t vocab, int32_t d,
                             float* loss, void* workspace, size_t ws_bytes, int32_t* status,
                             void* stream);

/* The losses and the gradients of sum_i row_weight[i] loss[i]: dh [n_rows, d] (lddh) and
 * dw [vocab, d] (lddw; NULL: a frozen vocabulary), bf16, summed in fp32.  Rows are taken
 * in pieces of piece_rows (0: at most 8,192): the workspace holds one piece's
 * probabilities in bf16; one for so many rows serves fewer as well. */
size_t jnx_op_vocab_loss_train_workspace_bytes(int32_t n_rows, int32_t vocab, int32_t d,
                                               int32_t piece_rows);
jnx_status jnx_op_vocab_loss_train(const uint16_t* h, int64_t ldh, const uint16_t* w, int64_t ldw,
                                   const int32_t* targets, const float* row_weight,
                                   int32_t n_rows, int32_t vocab, int32_t d, int32_t piece_rows,
                                   float* loss, uint16_t* dh, int64_t lddh, uint16_t* dw,
                                   int64_t lddw, void* workspace, size_t ws_bytes,
                                   int32_t* status, void* stream);

/* The same against a teacher's top logits.  Row i has up to `top` entries (1 to 128): words
 * ids[i * top + k] with the teacher's logits teacher[i * top + k]; a negative id or a logit
 * that is -inf over the temperature in fp32 is no entry, an id >= vocab is reported and read
 * as none, an id given twice has both entries' probability.  With T = softmax(teacher /
 * temperature) over the row's entries and P = softmax(h w^T / temperature) over the
 * vocabulary, loss[i] = sum_k T_k (log T_k - log P_k); 0 for a row without entries, whose h
 * is not read into any sum.  Logits over the temperature are finite or -inf; temperature > 0.
 * Otherwise as the next-token losses. */
size_t jnx_op_vocab_distill_workspace_bytes(int32_t n_rows, int32_t vocab, int32_t d, int32_t top);
jnx_status jnx_op_vocab_distill(const uint16_t* h, int64_t ldh, const uint16_t* w, int64_t ldw,
                                const int32_t* ids, const float* teacher, int32_t top,
                                float temperature, int32_t n_rows, int32_t vocab, int32_t d,
                                float* loss, void* workspace, size_t ws_bytes, int32_t* status,
                                void* stream);
size_t jnx_op_vocab_distill_train_workspace_bytes(int32_t n_rows, int32_t vocab, int32_t d,
                                                  int32_t top, int32_t piece_rows);
jnx_status jnx_op_vocab_distill_train(const uint16_t* h, int64_t ldh, const uint16_t* w,
                                      int64_t ldw, const int32_t* ids, const float* teacher,
                                      int32_t top, float temperature, const float* row_weight,
                                      int32_t n_rows, int32_t vocab, int32_t d,
                                      int32_t piece_rows, float* loss, uint16_t* dh, int64_t lddh,
                                      uint16_t* dw, int64_t lddw, void* workspace,
                                      size_t ws_bytes, int32_t* status, void* stream);

/* ---- answering with drafted tokens ----
 * Several tokens a step: a live sequence's last known token and the tokens drafted behind
 * it are the nodes of a tree, its root first and every node behind its parent.  Their keys
 * and values are appended behind the sequence's cached ones, the tree is attended in one
 * call, verified against the target's probabilities, and the accepted rows are kept.
 * Node i of sequence s is row cu_nodes[s] + i of the nodes' tensors; a sequence has up to
 * 64 nodes, or none.  The conventions of the text tenants' operators apply. */

/* Where live sequences' tokens lie in a cache whose slots are pages: token t of sequence s
 * in row t % room of page table[s * ld + t / room].  max_pages: entries of a sequence.  Only
 * entries whose pages hold tokens of a call are read. */
typedef struct {
    const int32_t* table;
    int64_t ld;
    int32_t n_seqs, max_pages;
} jnx_pages;

/* jnx_op_qk_norm_rope_append to pages: token i's key and value heads go to token at[i] of
 * sequence seq[i].  A token whose sequence, entry or page is not there is not written and
 * reported.  No two tokens of a call have the same place. */
jnx_status jnx_op_qk_norm_rope_append_paged(const jnx_qk_rope* p, const uint16_t* qkv,
                                            int64_t ldqkv, const int32_t* pos, int32_t n_tokens,
                                            const jnx_head_rows* q, const jnx_kv_cache* cache,
                                            const jnx_pages* pages, const int32_t* seq,
                                            const int32_t* at, int32_t* status, void* stream);

/* out = softmax(q k^T / sqrt(head_dim)) v for every node of every sequence (n_rows rows of q
 * and out hold them): node i of sequence s sees the n_cached[s] cached tokens and those nodes
 * j of its sequence, at tokens n_cached[s] + j, whose bit j of sees[row] is set (its ancestors
 * and itself, or any others).  A row that sees nothing has output 0, rows of no sequence stay
 * as they were.  cu_nodes [n_seqs + 1], n_cached [n_seqs] and sees [n_rows] are on the device.
 * A sequence whose rows are not among n_rows, more than 64, or start ahead of an earlier one's
 * end is left out and reported; one whose tokens are more than its entries hold has output 0
 * and is reported; a page that is not there is read as zeros and reported.  A cache whose
 * sequences have several pages has room a multiple of 16 (JNX_ERR_UNSUPPORTED otherwise).  q and
 * the keys and values of cached tokens and nodes are finite, whoever sees them; all other rows of
 * the pages may hold anything.  The bits of a sequence do not depend on the others.  The
 * workspace serves sequences of up to max_tokens tokens, nodes among them: max_pages * room of
 * the call. */
size_t jnx_op_tree_attention_workspace_bytes(int32_t n_seqs, int32_t n_rows, int32_t n_heads,
                                             int32_t head_dim, int64_t max_tokens);
jnx_status jnx_op_tree_attention(const jnx_kv_cache* cache, const jnx_pages* pages,
                                 int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                                 int32_t n_rows, const jnx_head_rows* q, const int32_t* cu_nodes,
                                 const int32_t* n_cached, const uint64_t* sees,
                                 const jnx_head_rows* out, void* workspace, size_t ws_bytes,
                                 int32_t* status, void* stream);

/* Verification of drafted trees by speculative sampling, so that the tokens are distributed
 * as the target's own.  Row cu_nodes[s] + i of p [n_rows, vocab] fp32 (row stride ldp) holds
 * the target's probabilities behind node i, of q (ldq) those that node i's children were
 * drawn from, one by one and independently; q NULL: the children are certain guesses, each
 * with probability one where it stands.  tokens and parent [n_rows]: a node's token and its
 * parent's number in the sequence (the root's are not read); u [n_rows] in [0, 1).
 * From the root on: the children of the node are tried in order.  With r = p and R = 1 at
 * first, child c of token x is accepted if u[c] q(x) R < r(x), and the walk goes on at c; else
 * r <- max(r - R q, 0) and R <- sum r.  Where no child is accepted, next[s] is the first word
 * whose sum of r up to it is above u[root] sum r (r = p if nothing is left of it).
 * path [n_seqs, max_nodes]: the root and the accepted nodes' numbers, then -1; n_kept[s] of
 * them.  A sequence of no nodes has n_kept 0 and next -1.  Left out and reported: sequences
 * whose rows are not among n_rows or more than max_nodes (as of no nodes), nodes whose parent
 * is not ahead of them or whose token is no word (never accepted), sums that are not finite
 * and positive, as of a row of p or q with a NaN (next -1).  p and q are not negative;
 * max_nodes in 1 to 64.  Sums are kept to 2^-44 of themselves or closer. */
jnx_status jnx_op_verify_drafts(const float* p, int64_t ldp, const float* q, int64_t ldq,
                                const int32_t* tokens, const int32_t* parent, const float* u,
                                const int32_t* cu_nodes, int32_t n_seqs, int32_t n_rows,
                                int32_t vocab, int32_t max_nodes, int32_t* path, int32_t* n_kept,
                                int32_t* next, int32_t* status, void* stream);

/* The accepted rows' keys and values to their places: token n_cached[s] + path[s * ld_path + k]
 * goes to token n_cached[s] + k, for k < n_kept[s], in each of n_layers caches that are
 * layer_stride elements apart.  A path increases and starts anywhere at or behind 0; n_kept up
 * to max_kept <= 64 (path's columns).  A sequence with another path or whose places are not
 * there is left as it was and reported.  No page serves two sequences of the call where rows
 * are moved. */
jnx_status jnx_op_keep_drafts(const jnx_kv_cache* cache, int32_t n_layers, int64_t layer_stride,
                              const jnx_pages* pages, int32_t n_kv_heads, int32_t head_dim,
                              const int32_t* n_cached, const int32_t* path, int64_t ld_path,
                              const int32_t* n_kept, int32_t max_kept, int32_t* status,
                              void* stream);

#ifdef __cplusplus
}
#endif

#endif /* JNX_OPS_H */
