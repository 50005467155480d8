/*
 * ssd_ops.h -- finer-grained entry points of the same library (libssd.so),
 * for parity checks against the CPU oracle, kernel timing and test fixtures.
 * Conventions as in ssd.h (status codes, caller-owned memory, the context's
 * stream unless a stream is given).
 */
#ifndef SSD_OPS_H
#define SSD_OPS_H

#include "ssd.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Statistics of one early-exit distribution P^(l) = softmax(z) (§3.1.1):
 * conf_k = C_k = -(1/k) sum of the log-probabilities of the k most probable
 * tokens; entropy = H^l; pmax = max probability (the per-step term of
 * C_trace); argmax = greedy token (lowest id on ties); margin = top-1 minus
 * top-2 logit. */
typedef struct {
  int32_t argmax;
  int32_t top_idx[8];
  float top_logit[8];
  float zmax, lse, entropy, conf_k, pmax, margin;
} ssd_exit_stats;

/* Teacher-forced partial forward (§3.1.1: P_t^(l) from the hidden state at
 * layer l): ids[0..M) (host) at positions pos0..pos0+M-1 run through layers
 * 1..l_exit, writing their KV (positions below pos0 must already hold KV for
 * all l_exit layers), then the shared final RMSNorm and LM head over all M
 * rows.  logits (host, optional) receives [M][vocab] fp32; stats (host,
 * optional) receives M records computed with top-k = topk (1..8).  1 <= M <= 17.
 * Does not change the pending token or the trace.  Synchronises. */
ssd_status ssd_forward_exit(ssd_ctx* ctx, const int32_t* ids, int32_t M, int32_t pos0,
                            int32_t l_exit, int32_t topk, float* logits, ssd_exit_stats* stats);

/* The Q-network of the current LEDE policy on n states (host [n][3] fp32:
 * C_k, H, C_trace) -> q (host [n][2]: Q(continue), Q(exit)).  SSD_ERR_STATE
 * when the policy's network takes the pooled state (qnet_in = d_model + 1).
 * Synchronises. */
ssd_status ssd_qnet_eval(ssd_ctx* ctx, const float* states, int32_t n, float* q);

/* KV-cache rows as fp32: layer (0-based), kind 0 = K (after RoPE) or 1 = V,
 * KV head, positions [p0, p0 + n) -> out (host) [n][head_dim]. */
ssd_status ssd_read_kv(ssd_ctx* ctx, int32_t layer, int32_t kind, int32_t head, int32_t p0,
                       int32_t n, float* out);

/* Sequence state: pending token, its position (= KV length) and the C_trace
 * window (host out[cap], oldest first; *n_trace entries). */
ssd_status ssd_read_state(ssd_ctx* ctx, int32_t* x, int32_t* pos, float* trace, int32_t cap,
                          int32_t* n_trace);

/* The weight-streaming matrix-vector kernel on the weights of layer `layer`:
 * which = 0 wqkv, 1 wo, 2 w_gate_up, 3 w_down, 4 lm_head (layer ignored).
 * y[m][r] = sum_c W[r][c] x[m][c] for m < M (1 <= M <= 17), x_dev [M][cols] and
 * y_dev [M][rows] fp32 device buffers.  fp32: one launch; bf16: a short launch
 * splits x into two bf16 parts in front of it.  Enqueued on `stream` (NULL =
 * the context's stream); no synchronisation. */
ssd_status ssd_op_gemv(ssd_ctx* ctx, int32_t which, int32_t layer, int32_t M, const float* x_dev,
                       float* y_dev, void* stream);

/* One hot-path kernel of layer `layer`, on M rows at positions
 * pos0..pos0+M-1 of the context's own buffers: kernel = 0 QKV (+RMSNorm, RoPE,
 * KV append), 1 attention (bf16: the splits and, in a second launch, their
 * merge; fp32: one launch), 2 O projection (+residual), 3 gate/up (+RMSNorm,
 * SwiGLU), 4 down projection (+residual), 5 exit head (final RMSNorm and LM
 * head, then the statistics in a launch of their own; layer ignored), 6 (bf16)
 * the chained launch the layer passes use: O projection, gate/up and down of
 * `layer` and the QKV of layer + 1 (when there is one) as the phases of one
 * persistent kernel.  The kernels are the ones the passes launch.  Each reads
 * what the kernel before it in a layer wrote; 0, 3 and 5 read the residual rows
 * under their own norm weights, whatever wrote them last (bf16: a short launch
 * in front multiplies the rows, which in a pass the kernel that writes them
 * does).  It overwrites the activations and the KV rows at those positions: for
 * timing and profiling, not inside a generation.
 * Needs pos0 + M <= max_seq.  Enqueued on `stream` (NULL = the context's). */
ssd_status ssd_op_layer(ssd_ctx* ctx, int32_t kernel, int32_t layer, int32_t M, int32_t pos0,
                        void* stream);

/* Allocation-free form of ssd_op_gemv (the paper has no counterpart: this is
 * an interface for callers that cannot allocate device memory, e.g. code that
 * runs while a CUDA graph is being captured, where cudaMalloc is not a
 * capturable operation, or a host framework that owns the device's memory
 * pool and allows no other allocations).  Computes y[m][r] = sum_c W[r][c]
 * x[m][c] for m < M exactly as ssd_op_gemv, without a context: W (device,
 * rows x cols, dtype, 16-byte aligned rows), x_dev [M][cols] and y_dev
 * [M][rows] fp32 (device) are the caller's; the kernel's scratch is a fixed
 * static device array inside libssd.so (about 1.1 MB, held on every device
 * that uses it until the process exits).
 * Limits: 1 <= M <= 17 and rows <= 131072 (SSD_ERR_CAPACITY beyond), cols *
 * element size a multiple of 16 (SSD_ERR_INVALID_ARG otherwise).
 * Device-side failure: the kernel's pipeline waits are bounded; one that gives
 * up sets an error word (SSD error bits, 16 = a wait timed out) in the static
 * array and leaves y_dev undefined.  With err_dev (device, one int32, may be
 * NULL) the call enqueues, after the kernel, a copy of that word into
 * *err_dev: 0 once the stream has reached it means y_dev holds the product.
 * The returned status covers only the host-side checks and the launch.
 * The first call on a device looks up the array's device address and sets
 * kernel attributes; make that first call before any stream capture.  Every
 * call clears the scratch's tickets and error word on `stream` and shares the
 * one array, so calls that overlap on the GPU (other streams, other threads)
 * race.  Enqueued on `stream`; no synchronisation; allocates nothing. */
ssd_status ssd_gemv_noalloc(const void* W, int32_t dtype, int32_t rows, int32_t cols,
                            const float* x_dev, int32_t M, float* y_dev, int32_t* err_dev,
                            void* stream);

/* ------------------------------------------------------------------------
 * A KV cache held in 8 bits, and what a verification pass over it needs: rows
 * into the cache, attention over it, and the log-probabilities of tokens (the
 * paper has no counterpart; its cache is in the model's type).  These calls
 * take no context.  They enqueue on `stream` (NULL: the legacy default stream),
 * whose device must be the current one, do not synchronise, allocate nothing and
 * keep nothing between calls, so they can be captured into graphs; the first
 * call of a kind on a device sets kernel attributes and has to come before a
 * capture.  Calls on different streams can run at the same time where they
 * share no output and no workspace; so can captured ones.  The returned
 * status covers the host-side checks and the launches, ssd_last_error(NULL) has
 * its message; what only the device can see sets bits (SSD_DEV_ERR_*) in
 * *err_dev (device int32; NULL: nothing tells of it), which the caller clears. */
#define SSD_KV8_BLOCK 64       /* positions that share a scale */
#define SSD_KV8_MAX_SEQS 4096
#define SSD_DEV_ERR_TOKEN 1    /* a token id outside [0, vocab) */
#define SSD_DEV_ERR_CAPACITY 2 /* positions outside the cache */
#define SSD_DEV_ERR_CONTROL 4  /* a number of rows outside 0..M */
#define SSD_DEV_ERR_TIMEOUT 16 /* ssd_kv8_attention: a wait inside a kernel gave up after some
                                * seconds; none of that call's outputs mean anything */

/* Cache of one layer for n_seq sequences (all memory the caller's, device).
 * k, v: e4m3 codes [n_seq][n_kv_heads][max_seq][head_dim], 16-byte aligned; k_scale,
 * v_scale: fp32 [n_seq][n_kv_heads][max_seq / 64].  A value is code * scale of
 * its block of 64 positions.  A scale is a power of two, 2^-120 to 2^111: the smallest that
 * brings the largest magnitude of the rows to 448 or less (beyond 448 * 2^111 values are cut
 * to that) where the block is written from its first position, growing with later rows
 * that need a larger one.  max_seq: a multiple of 64; head_dim 64 or 128
 * (SSD_ERR_UNSUPPORTED otherwise).  Codes need no initial value.  Scales need one, 0,
 * only where a sequence begins inside of a block (a padded batch whose pads are not
 * appended): what stands there counts as the scale of the positions in front. */
typedef struct {
  int32_t n_seq, n_kv_heads, head_dim, max_seq;
  void* k;
  void* v;
  float* k_scale;
  float* v_scale;
} ssd_kv8_cache;

/* Appends: rows m < rows[b] of sequence b (rows: device [n_seq], NULL: M each;
 * 0 leaves the sequence alone) go to positions pos[b] + m (pos: device [n_seq]).
 * k, v: device, dtype SSD_DTYPE_F32 or _BF16, row m of sequence b at element
 * (b M + m) row_stride, its heads one behind the other: a product's rows q | k | v
 * can be read in place; pointers and row_stride in multiples of 16 bytes.  M in 1 .. max_seq
 * (SSD_ERR_CAPACITY above, whatever rows says).
 * Positions from pos[b] on in its block count as free (a rollback needs no call).  Where
 * pos[b] is inside of a block, the larger of the scale that stands there and the new rows'
 * own becomes the block's; where that grows, the codes in front are rounded to it again
 * (nothing but values below 2^-6 of the new scale can change).  Codes from
 * pos[b] + rows[b] on are not written, but stand under a new scale in that block.
 * So rows that are rolled back leave a trace: the scale that they raised stays until the
 * block is written from its first position again, and what the codes in front lost
 * to it does not come back.
 * NaN and infinities are stored as NaN and take no part in a scale.
 * A sequence whose positions do not lie in 0 .. max_seq - 1, or whose rows[b] does
 * not in 0 .. M, is left alone, with its error bit; pos[b] is in 0 .. max_seq where rows[b]
 * is 0, too. */
ssd_status ssd_kv8_append(const ssd_kv8_cache* cache, const void* k, const void* v, int32_t dtype,
                          int64_t row_stride, int32_t M, const int32_t* pos, const int32_t* rows,
                          int32_t* err_dev, void* stream);

/* Bytes of device workspace that ssd_kv8_attention needs for these sizes,
 * whatever the lengths (256: it uses none, and takes NULL; 0: sizes that it refuses,
 * ssd_last_error(NULL) says why). */
size_t ssd_kv8_attention_bytes(const ssd_kv8_cache* cache, int32_t dtype, int32_t n_heads,
                               int32_t M);

/* Attention over the cache, softmax scale 1/sqrt(head_dim), query head h reading KV
 * head h / (n_heads / n_kv_heads): row m < rows[b] of sequence b sits at position
 * p = pos[b] + m and sees the keys j <= p with j >= first[b] (device [n_seq], NULL: 0;
 * a padded batch) and, with window > 0, j > p - window.  The rows' own keys must
 * have been appended.  q and out: device, dtype SSD_DTYPE_F32 or _BF16 (both the
 * same), row m of sequence b at element (b M + m) q_stride (out_stride), heads one
 * behind the other; pointers and strides in multiples of 16 bytes; out may
 * be q, then at the same stride, and overlaps it in no other way.
 * A row that sees no key is zero.  Rows from rows[b] on are left as they were,
 * and so are sequences with bad positions or row numbers (error bits as above).
 * What stands in a key or value that a row does not see never reaches it, NaN
 * neither.  Scores, sums and outputs are fp32.  bf16 query elements above 2^-28 of their
 * row's largest are exact, fp32 ones above 2^-15 keep 22 bits; a probability keeps 11
 * bits (fp32: 22) where its product with its value's scale is above 2^-20 (fp32: 2^-17) of
 * the row's largest probability times the largest value scale that the row sees.  Below
 * these they lose bits one by one.  Equal calls give equal bits.
 * Any M in 1 .. max_seq, any n_heads / n_kv_heads; SSD_ERR_CAPACITY for larger M, and where
 * n_seq x M x max_seq is so large that the work has more than 2^31 parts.  workspace: 256-byte
 * aligned, used by this call until it has run. */
ssd_status ssd_kv8_attention(const ssd_kv8_cache* cache, const void* q, int32_t dtype,
                             int32_t n_heads, int64_t q_stride, int32_t M, const int32_t* pos,
                             const int32_t* rows, const int32_t* first, int32_t window, void* out,
                             int64_t out_stride, void* workspace, size_t workspace_bytes,
                             int32_t* err_dev, void* stream);

#define SSD_MAX_TOP 32 /* most probable tokens of a row, at most */

/* Log-probabilities over rows of logits z at temperature t (0.001..1000; z / t is z times
 * 1 / t, which is rounded to fp32 once): of softmax(z / t), each row's lse = ln sum e^(z/t),
 * entropy in nats, the n_tokens given tokens' log-probabilities z/t - lse and the top_n (0..32)
 * most probable tokens (lower id first on ties) with theirs.  logits: device, dtype
 * SSD_DTYPE_F32 or _BF16, row r at element r row_stride (>= vocab; any alignment of an
 * element).  tokens: device [n_rows][n_tokens], logprob the same in fp32 (both may be NULL
 * when n_tokens is 0); id -1 marks a place without a token, its result is 0; any other id
 * outside [0, vocab) gives NaN and its error bit.  lse, entropy: device fp32 [n_rows], each may
 * be NULL.
 * top_id, top_logprob: device [n_rows][top_n], in descending order; where a row has
 * fewer than top_n logits above -inf, the places left are id -1, -inf.
 * A logit of -inf is a token of probability 0.  A row of nothing else has lse -inf,
 * its entropy and tokens NaN.  A NaN or +inf logit makes a row's lse, entropy and
 * log-probabilities NaN; its top_id are those of the numbers in it. */
ssd_status ssd_token_logprobs(const void* logits, int32_t dtype, int32_t n_rows, int32_t vocab,
                              int64_t row_stride, const int32_t* tokens, int32_t n_tokens,
                              float temperature, int32_t top_n, float* logprob, float* lse,
                              float* entropy, int32_t* top_id, float* top_logprob,
                              int32_t* err_dev, void* stream);

/* Test fixture: fills dst (device, n elements of dtype) with the seeded
 * synthetic weights of tensor `tid` (see synth/synth.h): element i is
 * synth_weight_f32(seed, tid, i, sigma), rounded to bf16 for SSD_DTYPE_BF16.
 * Enqueued on `stream`; no synchronisation. */
ssd_status ssd_synth_fill(void* dst, int32_t dtype, uint64_t n, uint32_t seed, uint32_t tid,
                          double sigma, void* stream);

/* Measurement fixture: reads `bytes` (multiple of 16) from src (device) with
 * the same streaming loads as the weight kernels and writes one checksum
 * word to sink (device).  Enqueued on `stream`. */
ssd_status ssd_read_probe(const void* src, uint64_t bytes, uint32_t* sink, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* SSD_OPS_H */
