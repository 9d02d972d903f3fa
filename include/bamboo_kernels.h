/*
 * bamboo_kernels.h -- C ABI of the individual layer kernels the Bamboo stage
 * is built from (arXiv 2204.12013, Section 5.1: FNC/BNC and FRC/BRC are the
 * same layer computation; the paper leaves the layer math to the models it
 * trains, Section 7 Table 1: BERT-Large, GPT-2).  Exposed so that each kernel
 * can be checked and timed on its own.
 *
 * All data pointers are device pointers owned by the caller; `stream` is a
 * hipStream_t passed as void*.  Calls enqueue and return.  dtype: 0 fp32,
 * 1 bf16 storage with fp32 accumulation.  impl: 0 automatic (MFMA kernel when it
 * covers the shape, vector-ALU kernel otherwise), 1 vector-ALU kernel,
 * 2 bf16 MFMA kernel, matrix products with one K chain per output tile (BAMBOO_E_STATE if it does not cover the
 * shape; matrix products: every dimension a multiple of 8).  fp32 matrix products run on the matrix cores too (impl 0),
 * except large ones that the vector ALU does faster.
 * Return: 0 or a negative bamboo_status (see bamboo_stage.h).
 * Tensors are row-major; "tokens" T = batch * seq.
 */
#ifndef BAMBOO_KERNELS_H
#define BAMBOO_KERNELS_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Y[T,N] = X[T,K] W[K,N] + bias[N] (+ res[T,N] if res != NULL).
 * If gelu_out != NULL (and res == NULL), with h = X W + bias kept in fp32:
 * gelu_out[T,N] = GELU(h) (erf form) and Y[T,N] = GELU'(h), the factor the
 * backward multiplies the incoming gradient by (so GELU is evaluated once, in
 * the forward, and the pre-activation itself is not kept). */
int bk_linear_fwd(int dtype, int impl, int T, int N, int K, const void* X, const void* W, const void* bias,
                  const void* res, void* Y, void* gelu_out, void* stream);

/* dX[T,K] = dY[T,N] W[K,N]^T (+ res[T,K] if res != NULL).
 * If mul != NULL (and res == NULL): dX = (dY W^T) * mul[T,K] elementwise (the
 * backward through an activation whose derivative the forward stored). */
int bk_linear_bwd_input(int dtype, int impl, int T, int K, int N, const void* dY, const void* W, const void* res,
                        const void* mul, void* dX, void* stream);

/* dW[K,N] (fp32) += X[T,K]^T dY[T,N]; if db != NULL also db[N] (fp32) += sum over
 * tokens of dY (the bias gradient of the same linear layer), with
 * partial = fp32 scratch of bk_colsum_scratch_floats(N) floats. */
int bk_linear_bwd_weight(int dtype, int impl, int T, int K, int N, const void* X, const void* dY, float* dW,
                         float* db, float* partial, void* stream);

/* n (1..4) weight gradients in one go: dW[i][K[i],N[i]] (fp32) += X[i][T[i],K[i]]^T dY[i][T[i],N[i]].
 * T, K, N: host int arrays; X, dY, dW: host arrays of device pointers.  Where one kernel covers all of them (bf16:
 * any T, K and N multiples of 8, aligned to 16 bytes; fp32: up to 1024 tiles of 32 x 32 each) and none writes what
 * another one reads or writes, they run as ONE launch whose workgroups are dealt over the problems, so that problems
 * that do not fill the chip on their own share its rounds; otherwise one launch each, in order.  The results do not
 * depend on which. */
int bk_linear_bwd_weight_group(int dtype, int n, const int* T, const int* K, const int* N, const void* const* X,
                               const void* const* dY, float* const* dW, void* stream);

/* out[N] (fp32) += sum over tokens of A[T,N]; partial: fp32 scratch of
 * bk_colsum_scratch_floats(N) floats.  Fixed summation order. */
int bk_colsum_acc(int dtype, int T, int N, const void* A, float* out, float* partial, void* stream);
uint64_t bk_colsum_scratch_floats(int N);

/* bk_colsum_acc for callers that cannot allocate device memory: code under HIP graph capture, tight
 * serving loops, harnesses that forbid hipMalloc.  Same result as bk_colsum_acc (the same two kernels
 * in the same order), but the partial rows live in a device array inside the library (2 MiB per GPU,
 * held until the process ends) instead of a caller buffer; the call allocates and frees nothing.
 * A, out: device pointers as for bk_colsum_acc (out is added to).  BAMBOO_E_ARG if the shape needs
 * more than bk_colsum_static_max_floats() = 2^19 floats of partial rows (partial rows x N; the launch
 * shape keeps that product below 2^18 until a single row exceeds the array, i.e. every N <= 524288
 * fits with any T), decided before anything is launched.  All calls on one GPU share that GPU's array: calls that overlap on one GPU (two
 * streams, two threads) race; calls on one stream, one after the other, are safe, and nothing needs
 * clearing between them. */
int bk_colsum_acc_static(int dtype, int T, int N, const void* A, float* out, void* stream);
uint64_t bk_colsum_static_max_floats(void);

/* Softmax attention.  qkv[T,3H] = queries | keys | values, head h = columns
 * h*d..(h+1)*d-1 of each third; scores scaled by 1/sqrt(d); causal != 0 masks
 * keys after the query.  ctx[T,H]; lse[batch,heads,seq] fp32 = log-sum-exp of
 * the scaled scores of each row. */
int bk_attention_fwd(int dtype, int impl, int batch, int seq, int heads, int d, int causal, const void* qkv, void* ctx,
                     float* lse, void* stream);
/* dqkv[T,3H] from dctx[T,H], recomputing the probabilities from lse.
 * delta: fp32 [batch,heads,seq], set to rowsum(ctx * dctx) of each head. */
int bk_attention_bwd(int dtype, int impl, int batch, int seq, int heads, int d, int causal, const void* qkv,
                     const void* ctx, const float* lse, const void* dctx, void* dqkv, float* delta, void* stream);

/* y = gamma * (r - mean) * rstd + beta per token row; stats[2t] = mean,
 * stats[2t+1] = rstd = 1/sqrt(biased variance + eps). */
int bk_layernorm_fwd(int dtype, int T, int H, float eps, const void* r, const void* gamma, const void* beta, void* y,
                     float* stats, void* stream);
/* dr = LayerNorm backward of dout (+ add[T,H] if add != NULL); dgamma, dbeta
 * (fp32) += their token sums.  partial: fp32 scratch of
 * bk_layernorm_bwd_scratch_floats(H) floats. */
int bk_layernorm_bwd(int dtype, int T, int H, const void* dout, const void* r, const float* stats, const void* gamma,
                     const void* add, void* dr, float* dgamma, float* dbeta, float* partial, void* stream);
uint64_t bk_layernorm_bwd_scratch_floats(int H);

/* One Adam step (Section 7 names the optimizer) over n parameters, n a multiple of 4, step >= 1:
 * g fp32 gradient; master, m, v fp32 master weights and moments, updated in place; w[n] (storage
 * dtype) = the new master weights rounded to storage.  All device pointers, 16-byte aligned. */
int bk_adam(int dtype, int64_t n, const float* g, float* master, float* m, float* v, void* w, float lr, float beta1,
            float beta2, float eps, int step, void* stream);

/* ---- the two ends of the model, worked on by the wrap-around stage only (Section 5.1: the last
 * node keeps the replica of the first node's layers and fetches the input samples itself).  The
 * paper does not spell them out; they are the textbook ends of the models it trains.
 *
 * Front: out[t,:] = E_tok[ids[t],:] + E_pos[t mod seq,:], the sum taken in fp32 and rounded to the
 * storage type.  ids: device int32 [T]; values outside [0, V) are clamped into the range (never
 * read out of bounds).  H a multiple of 8; E_tok [V,H], E_pos [seq,H], out [T,H] 32-byte aligned. */
int bk_embedding_fwd(int dtype, int T, int seq, int H, int V, const int32_t* ids, const void* E_tok, const void* E_pos,
                     void* out, void* stream);
/* dE_tok[V,H] (fp32) += rows of g[T,H] scattered by ids, dE_pos[seq,H] (fp32) += rows of g summed over
 * the samples.  No atomics: rows hit by several tokens are added in token order.  Any H and any alignment
 * (H a multiple of 8 with g 32-byte aligned is faster). */
int bk_embedding_bwd(int dtype, int T, int seq, int H, int V, const int32_t* ids, const void* g, float* dE_tok,
                     float* dE_pos, void* stream);
/* Back: per token t, lse[t] = log sum_v exp(logits[t,v]) and loss_tok[t] = lse[t] - logits[t,labels[t]]
 * (fp32, from the stored logits); V a multiple of 8, logits [T,V] 32-byte aligned. */
int bk_softmax_xent_fwd(int dtype, int T, int V, const void* logits, const int32_t* labels, float* lse,
                        float* loss_tok, void* stream);
/* dlogits[t,v] = (exp(logits[t,v] - lse[t]) - [v == labels[t]]) * scale; dlogits may be logits. */
int bk_softmax_xent_bwd(int dtype, int T, int V, const void* logits, const int32_t* labels, const float* lse,
                        float scale, void* dlogits, void* stream);
/* out[0] = scale * (in[0] + ... + in[n-1]) in a fixed order (the mean loss of a micro-batch). */
int bk_ordered_sum(int64_t n, const float* in, float scale, float* out, void* stream);

/* ---- operators of a training step around the stage: what a model that reads an encoder, or is trained further from
 * preferences or rewards, puts between the calls above.  Here a row of a matrix may be followed by other columns: ld* is
 * the distance between rows in elements.  Outputs must not overlap inputs or each other except where it says so
 * (columns of one matrix beside each other do not).  Calls work on the
 * current device, which the stream and all pointers belong to; nothing is kept from one call for the next.
 *
 * Rotary positions, between the QKV product and the attention: in each of `heads` heads of row t (columns h*d .. h*d+d-1),
 * pair i of the first rot features is turned by the angle pos[t] * freq[i]:
 *   (a, b) -> amplitude * (a cos - b sin, b cos + a sin),
 * the pair being features (i, i + rot/2), or (2i, 2i + 1) if interleaved != 0.  inverse != 0 turns the other way: the
 * backward, from the gradient at y to that at x.  Features rot .. d-1 are passed on.  y may be x (with ldy = ldx); for
 * queries and keys of a packed qkv[T,3H] in place: heads = 2 * heads, ldx = 3H.
 * pos: device int32 [T], any sign, or NULL for t mod seq.  freq: device double [rot/2] (bk_rotary_frequencies).  Angles
 * are formed in 64 bits.  2 <= rot <= d <= 512, rot even. */
int bk_rotary(int dtype, int T, int seq, int heads, int d, int rot, int interleaved, int inverse, const void* x,
              int64_t ldx, const int32_t* pos, const double* freq, float amplitude, void* y, int64_t ldy, void* stream);
/* freq (HOST double [rot/2]) = base^(-2i/rot), for a context stretched by `factor` >= 1:
 * scaling 0  as it is;  1  all divided by factor;  2  base * factor^(rot/(rot-2)) in the place of base (the slowest pair is
 * divided by factor, the fastest stays);  3  by parts: a pair that makes r turns in `length` positions is kept to
 * w = clamp((r - 1) / 31, 0, 1) and divided by factor to 1 - w, and *amplitude = 0.1 ln(factor) + 1 instead of 1.
 * length: the context the model was trained on (scaling 3 only).  amplitude may be NULL.  Runs on the host. */
int bk_rotary_frequencies(int rot, double base, int scaling, double factor, int length, double* freq, float* amplitude);

/* Softmax attention of queries over the states of an encoder, of another length.  Queries q[batch*sq, heads*d] (row
 * stride ldq), keys and values k, v[batch*sk, kv_heads*d] (row stride ldkv; halves of one packed projection, or two
 * matrices); query head h reads key head h / (heads / kv_heads); scores scaled by 1/sqrt(d); 1 <= d <= 128.
 * kv_len: device int32 [batch], keys that count of each sample (the first ones; clamped to 0 .. sk), or NULL for all; keys
 * and values behind them are never read.  ctx[batch*sq, heads*d] (row stride ldc), lse[batch,heads,sq] fp32.  A sample
 * without keys has ctx = 0 and lse = -inf.
 * scratch: fp32, bk_cross_attention_scratch_floats(..) floats, 16-byte aligned, used by this call alone.
 * impl: 0 automatic (2 for bf16 tensors, 1 for fp32 ones), 1 fp32 arithmetic on the matrix cores, 2 bf16 on them (BAMBOO_E_STATE for
 * fp32 tensors).  2 rounds the probabilities, and in the backward dS, to bf16 for the products that follow: gradients are 0.0022 to
 * 0.0029 of their norm off and ctx up to 0.0025, where the one rounding of a result is 0.0017; 1 on bf16 tensors rounds results alone, at
 * a sixteenth of the matrix rate.  Scores are taken to stay within 10^29.  bf16 is fastest with d 64 or 128, strides multiples of 8 and pointers aligned to 16 bytes. */
int bk_cross_attention_fwd(int dtype, int impl, int batch, int sq, int sk, int heads, int kv_heads, int d, const void* q,
                           int64_t ldq, const void* k, const void* v, int64_t ldkv, const int32_t* kv_len, void* ctx,
                           int64_t ldc, float* lse, float* scratch, void* stream);
/* dq, dk, dv (strides lddq, lddkv) from dctx (stride lddc), recomputing the probabilities from lse.  Keys that do not count
 * get zeros; the gradients of a key head are summed over the query heads that read it.  Fixed order, no atomics. */
int bk_cross_attention_bwd(int dtype, int impl, int batch, int sq, int sk, int heads, int kv_heads, int d, const void* q,
                           int64_t ldq, const void* k, const void* v, int64_t ldkv, const int32_t* kv_len,
                           const void* ctx, int64_t ldc, const float* lse, const void* dctx, int64_t lddc, void* dq,
                           int64_t lddq, void* dk, void* dv, int64_t lddkv, float* scratch, void* stream);
/* 0 for sizes that the calls refuse (the product of batch, kv_heads and the larger of sk and sq * heads / kv_heads has to stay below
 * 2^31). */
uint64_t bk_cross_attention_scratch_floats(int batch, int sq, int sk, int heads, int kv_heads, int d);

/* Clipped policy loss with a KL and an entropy term, and its gradient in the same pass.  Per token t, with
 * logp = log softmax(logits[t,:])[labels[t]], r = exp(logp - old_logp[t]), u = ref_logp[t] - logp:
 *   loss_tok[t] = -min(r adv[t], clip(r, 1 - clip_low, 1 + clip_high) adv[t]) + kl_coef (exp(u) - u - 1) - ent_coef H
 *   dlogits[t,:] = scale * d loss_tok[t] / d logits[t,:]       (where both sides of the min are equal: the unclipped one's)
 * H: entropy of the token's distribution.  mask: device bytes [T], 0 = the token does not count (its logits are not read;
 * all it gets is zeros), or NULL.  ref_logp NULL: no KL term.  Any V, strides ldl, ldd in elements; labels outside [0, V) are
 * clamped.  Outputs [T] fp32: logp, loss_tok, and, unless NULL, kl_tok (the term without its coefficient) and entropy;
 * dlogits NULL: no gradient; dlogits may be logits (with ldd = ldl).  T < 2^24, V <= 2^27.  Logits of -inf take no part; a NaN, +inf or a row
 * of -inf alone makes the row NaN.  The mean over the tokens: bk_ordered_sum. */
int bk_policy_loss(int dtype, int T, int V, const void* logits, int64_t ldl, const int32_t* labels, const uint8_t* mask,
                   const float* old_logp, const float* ref_logp, const float* adv, float clip_low, float clip_high,
                   float kl_coef, float ent_coef, float scale, float* logp, float* loss_tok, float* kl_tok,
                   float* entropy, void* dlogits, int64_t ldd, void* stream);

/* Preference loss over pairs of sequences.  logits[2*pairs*seq, V]: the chosen sequences, then the rejected ones in the
 * same order.  logp_seq[2*pairs] = sums of the counting tokens' log-probabilities, and per pair
 *   margin = beta ((logp_chosen - ref_chosen) - (logp_rejected - ref_rejected))
 *   loss = -(1 - smoothing) log sigmoid(margin) - smoothing log sigmoid(-margin)
 * ref_logp[2*pairs]: the reference model's sums.  mask, labels, V, ldl: as above.  lse[T], logp[T] (0 for tokens that do not
 * count), T = 2*pairs*seq < 2^24, margin[pairs], loss[pairs]: fp32 outputs; sums over a sequence are taken in 64 bits, of terms in
 * 64 bits: scratch, T doubles, used by this call alone. */
int bk_preference_loss_fwd(int dtype, int pairs, int seq, int V, const void* logits, int64_t ldl, const int32_t* labels,
                           const uint8_t* mask, const float* ref_logp, float beta, float smoothing, float* lse,
                           float* logp, float* logp_seq, float* margin, float* loss, double* scratch, void* stream);
/* dlogits[t,:] = scale * d loss[pair of t] / d logits[t,:]; dlogits may be logits (with ldd = ldl).  Probabilities are
 * exp(logits - lse): as fp32 holds lse, they are off by |lse| 2^-24 of themselves (a row whose logits all lie near -1e30 is not
 * normalised any more). */
int bk_preference_loss_bwd(int dtype, int pairs, int seq, int V, const void* logits, int64_t ldl, const int32_t* labels,
                           const uint8_t* mask, const float* lse, const float* margin, float beta, float smoothing,
                           float scale, void* dlogits, int64_t ldd, void* stream);

/* One AdamW step over n tensors, step >= 1.  Host arrays of n: numel (0 is allowed, below 2^34 - 1023), device pointers g (fp32 gradients),
 * master (fp32 weights), m, v, w (storage dtype, = the new master weights rounded), decay (the tensor's weight decay):
 *   m <- beta1 m + (1-beta1) g,  v <- beta2 v + (1-beta2) g^2,
 *   master <- master (1 - lr decay) - lr (m / (1-beta1^step)) / (sqrt(v / (1-beta2^step)) + eps)
 * moment_bits 32: m, v fp32; m_scale, v_scale NULL.  8: m, v codes of one byte (e4m3) and m_scale, v_scale fp32
 * [ceil(numel/256)]: element i of m is code * m_scale[i/256], the ROOT of element i of v is code * v_scale[i/256]; all
 * zero bits are zero moments.  The step uses the moments before they are rounded to codes; the rounding goes up or down by
 * bits that depend on (seed, step, the tensor's place in the list, the element) alone, so that replicas that make the
 * same calls stay equal to the bit (a captured call repeats its own step number and rate).  With 8 bits a gradient that is NaN makes its element's moments NaN, an infinite one its
 * whole block's (and a finite one whose square is not, the block's second moments).  No two tensors may overlap.  Any alignment of an element; the fast form takes pointers aligned to 16
 * bytes (w and codes: to four elements). */
int bk_adamw_group(int dtype, int moment_bits, int n, const int64_t* numel, const float* const* g, float* const* master,
                   void* const* m, void* const* v, float* const* m_scale, float* const* v_scale, void* const* w,
                   const double* decay, double lr, double beta1, double beta2, double eps, int step, uint32_t seed,
                   void* stream);

#ifdef __cplusplus
}
#endif
#endif /* BAMBOO_KERNELS_H */
