/* softsync_learn.h -- operators around the parameter server for language models: what a learner computes on the weights it
 * pulled (token log probabilities, a clipped policy loss, a preference loss, each with its gradient with respect to the logits)
 * and what a server does with pushed gradients beside momentum SGD (their global norm, an AdamW step over many tensors with
 * moments in 32 or in 8 bits).  Same library, status codes and conventions as softsync_ps.h:
 *   - *_dev pointers are device memory of the current GPU; host arrays are copied before the call returns;
 *   - the library allocates no device memory: the caller owns every buffer and workspace;
 *   - work is enqueued on `stream` (a cudaStream_t) and the call returns at once; nothing is read back;
 *   - negative return values are errors (ps_status) and nothing has been enqueued, except after PS_ERR_CUDA.
 * The paper has none of these operators; its weighting of a stale gradient (Section 2.4, Eq. 3) enters as the scales. */
#ifndef SOFTSYNC_LEARN_H
#define SOFTSYNC_LEARN_H

#include "softsync_ps.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------------------------------------------------------
 * A list of tensors: parameters of a model, each with gradients of the same length.
 *
 * Moments of all tensors lie in one array (a state array) each, tensor after tensor, every tensor starting at a multiple of
 * PS_STATE_BLOCK elements; elements between the tensors are never read or written.  ps_tensors_sizes gives the length.
 * ------------------------------------------------------------------------------------------------------------------ */
#define PS_STATE_BLOCK 256                /* elements of 8-bit moments that share one exponent; the tensors' alignment in a state array */
#define PS_LIST_MAX_GRADS 256             /* most gradients in one weighted sum */

typedef struct ps_tensors ps_tensors_t;   /* opaque; one GPU; not thread-safe */

/* Elements of a state array and bytes of the device workspace of a list (either pointer may be NULL).  Needs no GPU. */
int ps_tensors_sizes(int num_tensors, const int64_t *sizes_host, int64_t *state_elems, int64_t *workspace_bytes);

/* A list of num_tensors >= 1 tensors with sizes_host[k] >= 0 elements.  workspace_dev: 16-byte aligned, at least
 * the bytes that ps_tensors_sizes gives, the list's own until ps_tensors_destroy: it holds the table of the tensors (uploaded here, on
 * `stream`, which this call waits for) and the partial sums of ps_grad_norm; so calls on one list must not overlap in time. */
int ps_tensors_create(ps_tensors_t **out, int num_tensors, const int64_t *sizes_host, void *workspace_dev, int64_t workspace_bytes,
                      void *stream);
int ps_tensors_destroy(ps_tensors_t *list);

/* Binds what ps_adamw_step updates.  weights_host[k]: device pointer of tensor k's fp32 weights.  mirrors_host: device pointers of
 * bf16 copies that every step rewrites, or NULL (single entries may be NULL too).  lr_mult_host, decay_mult_host: a learning-rate
 * and a weight-decay multiplier for each tensor, or NULL (1).  state_bits 32: m_dev and v_dev are fp32 state arrays, the scales NULL.  state_bits 8: they are byte
 * state arrays, and m_scale_dev, v_scale_dev have one byte for each PS_STATE_BLOCK elements (state array length / PS_STATE_BLOCK).
 * All zeros are the moments' start in either form.  State arrays are 16-byte aligned; weights 4-byte, mirrors 2-byte (16- and 8-byte
 * alignment is faster).  Uploads a table on `stream` and waits for it.  No two arrays may overlap. */
int ps_tensors_bind_adamw(ps_tensors_t *list, float *const *weights_host, void *const *mirrors_host,
                          const float *lr_mult_host, const float *decay_mult_host, int state_bits,
                          void *m_dev, void *v_dev, uint8_t *m_scale_dev, uint8_t *v_scale_dev, void *stream);

/* Global norm of the weighted sum of c gradients over all tensors:
 *     g = scales[0] g_0 + ... + scales[c-1] g_{c-1};   out_dev[0] = |g|_2;
 *     out_dev[1] = max_norm / |g| where |g| > max_norm, else 1 (NaN where the norm is NaN)
 * grads_host: c * num_tensors device pointers, gradient after gradient, of grad_dtype (ps_grad_dtype) values.  scales_host: c fp32
 * factors (Eq. 3 and the 1/c of Eq. 2 are the caller's), or NULL for 1.  Products and sums of g are rounded one by one in fp32, in the
 * order given; squares are added in fp32 up to a few dozen at a time (so one above 3.4e38 makes the norm infinite) and in fp64 beyond
 * that, in a fixed order: the same call gives the same bits. */
int ps_grad_norm(ps_tensors_t *list, const void *const *grads_host, int c, const float *scales_host, int grad_dtype,
                 float max_norm, float *out_dev, void *stream);

/* The hyper-parameters of one AdamW step.  step: its number t >= 1 (for the bias corrections).  seed: for the random rounding of
 * 8-bit moments; the same seed, step and inputs give the same bits. */
typedef struct ps_adamw_config {
    double lr, beta1, beta2, eps, weight_decay;
    int64_t step;
    uint64_t seed;
} ps_adamw_config;

/* One AdamW step of every bound tensor in one pass: with g as in ps_grad_norm and, if clip_dev != NULL, g = g * clip_dev[1]
 * (clip_dev: what ps_grad_norm wrote; where clip_dev[0] is not finite the step changes nothing at all),
 *     m = beta1 m + (1 - beta1) g;     v = beta2 v + (1 - beta2) g^2
 *     w = w (1 - lr wd) - lr / (1 - beta1^t) * m / (sqrt(v) / sqrt(1 - beta2^t) + eps)
 * with lr times the tensor's lr_mult and wd = weight_decay times its decay_mult.  Every product, sum, quotient and root is rounded once
 * to fp32, in the order ((m*, (1-beta1)*g), (v*, (1-beta2)*(g*g)), root * (1/sqrt(1-beta2^t)) + eps, quotient, * step size).  Of a quotient
 * below 2^-126 it is left open whether it is rounded to a subnormal before the product or only with it.
 *
 * Moments in 8 bits: the PS_STATE_BLOCK elements of a block share a power of two 2^(scale - 127); m is a sign, 3 exponent bits and 4
 * fraction bits with bias 7, v 4 exponent bits and 4 fraction bits with bias 15, both with subnormals.  The step computes with the
 * fp32 values and rounds what it keeps at random to one of the two neighbours, so that the expectation stays: an average
 * that moves by less than half a code step would otherwise never move.  A v above zero keeps at least the smallest code, so that no
 * quotient loses its denominator.  A block that meets an infinity, a NaN or
 * a magnitude of 31/16 * 2^126 decodes to infinities and NaN from then on. */
int ps_adamw_step(ps_tensors_t *list, const void *const *grads_host, int c, const float *scales_host, int grad_dtype,
                  const ps_adamw_config *config, const float *clip_dev, void *stream);

/* PS_OK if ps_adamw_step takes this configuration, else what it would return for it.  Needs no GPU. */
int ps_adamw_check(const ps_adamw_config *config);

/* The bound 8-bit moments as the values they stand for, exactly, in bf16 state arrays (16-byte aligned).  state_bits 8 only. */
int ps_adamw_moments(ps_tensors_t *list, void *m_bf16_dev, void *v_bf16_dev, void *stream);

/* ------------------------------------------------------------------------------------------------------------------
 * Losses from logits.  Row t of the logits holds the unnormalised log probabilities of one position's vocabulary; with a
 * temperature T, z = logits / T, p = softmax(z), and for the row's token a
 *     logp = z_a - lse(z),     lse(z) = log sum_j exp(z_j),     entropy = -sum_j p_j log p_j
 * Rows with a weight of exactly zero (prompts, padding) are not read, whatever they or their token hold: their outputs are zero.
 * Minus infinity is a valid logit (a barred entry: p = 0).  A row of minus infinities, or with a NaN or plus infinity, has NaN results, and
 * so has a row whose token lies outside [0, vocab).  Sums over a row and over rows are fp32 and fp64; two calls give the same bits.
 * ------------------------------------------------------------------------------------------------------------------ */
typedef struct ps_logits {
    const void *data_dev;                 /* rows of `vocab` values, aligned to their type; 16-byte aligned rows are faster */
    int dtype;                            /* ps_grad_dtype: fp32 or bf16 */
    int64_t rows, vocab, row_stride;      /* row_stride >= vocab: elements from one row to the next */
    const int64_t *tokens_dev;            /* rows token ids */
    const float *weights_dev;             /* rows weights, or NULL: 1 for every row */
    float temperature;                    /* > 0 */
} ps_logits;

/* Bytes of the device workspace that the two losses need for `rows` rows and `sequences` sequences (0 for the policy loss).  Its first
 * four bytes must be zero before its first use; every call leaves them so, whatever its sizes, and keeps nothing else there.
 * Calls that share a workspace must not overlap in time. */
int ps_loss_workspace(int64_t rows, int64_t sequences, int64_t *bytes);

/* logp, lse, entropy (fp32, rows each; lse and entropy may be NULL): one pass over the logits. */
int ps_token_logprob(const ps_logits *logits, float *logp_dev, float *lse_dev, float *entropy_dev, void *stream);

/* The clipped policy loss on tokens that a policy of older weights sampled (in an asynchronous training every learner's are), with
 *     rho = exp(logp - old_logp),   d = ref_logp - logp,   share_t = w_t / sum w    (0 where sum w is 0)
 *     l = -min(rho A, clamp(rho, 1 - clip_low, 1 + clip_high) A) + kl_coef (exp(d) - d - 1) - entropy_coef H
 *     loss = sum_t share_t l_t
 * and its gradient with respect to the logits
 *     dlogits_tj = share_t / T ( a_t (1[j = token] - p_j) + entropy_coef p_j (log p_j + H) )
 *     a = (-rho A where rho A <= clamp(rho) A, else 0) + kl_coef (1 - exp(d)).
 * ref_logp_dev may be NULL: no KL term (kl_coef is ignored).  dlogits_dev: logits' dtype, rows of vocab values dlogits_stride elements
 * apart; it may be the logits' own memory (same stride): the gradient then replaces them; else it must not overlap them.  NULL: no gradient.
 * A row that lies at the same place within 16 bytes in both is written in vectors, others (a dense gradient of padded rows) element by element.
 * stats_dev: 5 fp32, weighted means of loss, clipped term, KL term, entropy, and the share of clipped tokens.
 * logp_dev, entropy_dev: rows fp32 each (zero where the weight is zero); entropy_dev may be NULL. */
typedef struct ps_policy_inputs {
    const float *old_logp_dev, *advantages_dev, *ref_logp_dev;
    float clip_low, clip_high, kl_coef, entropy_coef;
} ps_policy_inputs;
int ps_policy_loss(const ps_logits *logits, const ps_policy_inputs *in, float *stats_dev, float *logp_dev, float *entropy_dev,
                   void *dlogits_dev, int64_t dlogits_stride, void *workspace_dev, int64_t workspace_bytes, void *stream);

/* The preference loss on `pairs` pairs of sequences: sequence k is rows [offsets[k], offsets[k+1]); sequences 2i and 2i + 1 are the
 * preferred and the other answer of pair i.  With pi_k = sum over its rows of w_t logp_t and ref_logp_k the same under the reference,
 *     margin_i = beta ((pi_2i - ref_2i) - (pi_2i+1 - ref_2i+1))
 *     loss = mean_i ( -(1 - s) log sigmoid(margin_i) - s log sigmoid(-margin_i) ),     s = label_smoothing
 *     dlogits_tj = +-g_i w_t / T (1[j = token] - p_j),   + for sequence 2i,   g_i = beta / pairs (s sigmoid(margin_i) - (1 - s) sigmoid(-margin_i))
 * offsets_dev: 2 * pairs + 1 ascending row numbers (a sequence may be empty); rows outside every sequence get a zero gradient.
 * stats_dev: 3 fp32, loss, share of positive margins, mean margin.  seq_logp_dev: 2 * pairs fp32.  dlogits as above. */
typedef struct ps_preference_inputs {
    const int64_t *offsets_dev;
    const float *ref_logp_dev;
    int64_t pairs;
    float beta, label_smoothing;
} ps_preference_inputs;
int ps_preference_loss(const ps_logits *logits, const ps_preference_inputs *in, float *stats_dev, float *seq_logp_dev,
                       void *dlogits_dev, int64_t dlogits_stride, void *workspace_dev, int64_t workspace_bytes, void *stream);

/* ------------------------------------------------------------------------------------------------------------------
 * Losses without logits.  The logits of a position are the products of its hidden state with the rows of the output matrix (the head),
 *     z_tj = hidden_t . head_j / T,     lse_t = log sum_j exp(z_tj),     logp_t = z_t,token - lse_t
 * They are computed a tile at a time (tensor cores, fp32 sums) and never leave the chip.  The tensor cores cut a running sum to 24 bits towards zero at each addition of 16 terms, so
 * their sums are of 1,024 terms at most (of 4,096 in gradients that are rounded to bf16) and are added to nearest in fp32.  The gradients go through the vocabulary piece by piece; of a piece
 * the rounded bf16 values
 *     G_tj = a_t (p_tj - 1[j = token])
 * (a_t relative to a power of two near the largest |a_t|, so that the size of all of them together does not matter)
 * are held in the workspace, for the two products  dhidden = scale G head  and  dhead = scale G^T hidden  (sums in fp32, in a fixed order).  A piece is as wide as
 * 1 GiB of G allows (or as many bytes as the hidden states have, where that is more); ps_head_cross_entropy keeps the exponentials of the last piece from
 * its statistics (16 bits each, 10 of fraction), the other pieces' logits are computed again.
 * Rows with a weight (or a dlogp) of exactly zero take no part, whatever they or their token hold: they are not read, their outputs and their
 * dhidden are zero.  A token outside [0, vocab) makes its row's results NaN; so does a NaN or an infinity in a row, or a product that is plus infinity.  An entry of the head
 * whose product with a row is minus infinity is barred (p = 0); a row of nothing else is NaN, and infinities of the head make dhidden NaN.  NaN
 * results of a row that takes part reach the loss and dhead.  Outputs must not overlap inputs.
 * ------------------------------------------------------------------------------------------------------------------ */
typedef struct ps_head {
    const void *hidden_dev;               /* bf16, rows of `width` values, hidden_stride elements apart */
    const void *head_dev;                 /* bf16, vocab rows of `width` values, head_stride elements apart */
    int64_t rows, width, vocab, hidden_stride, head_stride;
    const int64_t *tokens_dev;            /* rows token ids */
    float temperature;                    /* > 0, log2(e) / temperature a number of fp32 */
} ps_head;

/* Bytes of the device workspace (256-byte aligned) of the calls below; grad: of those with gradients.  It need not be initialised and holds nothing
 * between calls; calls that share one must not overlap in time.  Where the width is no multiple of 8, or a matrix is not aligned to 16 bytes
 * (address and stride), the workspace has room for an aligned copy of it, and with gradients for a piece's rows of dhead.
 * What it holds: 2 bytes for each row and entry of a piece (G: half of what the logits of the piece take in fp32, so a call whose logits are fewer than half a billion holds that much for
 * them), the hidden states that take part, 8 bytes for each row and 128 entries, and the sums of split tiles (256 KB each; none where a contraction is below 1,024, at most 58 MB
 * for each gradient). */
int ps_head_workspace(const ps_head *head, int grad, int64_t *bytes);

/* logp, lse (fp32, rows each) of the rows with a weight; zeros elsewhere.  weights_dev: rows fp32, or NULL (all). */
int ps_head_logprob(const ps_head *head, const float *weights_dev, float *logp_dev, float *lse_dev, void *workspace_dev, int64_t workspace_bytes,
                    void *stream);

/* The gradients of any loss of the log probabilities, from dlogp_t = dloss/dlogp_t and lse (of ps_head_logprob): a_t = -dlogp_t, scale = 1 / T.
 * p is exp(z - lse): off by lse's rounding to fp32 (2^-20 of p at an lse of 16, 2^-15 at 512), which is what is left of p - 1 where a row is that sure of its token.
 * dhidden_dev: rows x width, dhead_dev: vocab x width, dense, 16-byte aligned, bf16; either may be NULL. */
int ps_head_logprob_grad(const ps_head *head, const float *lse_dev, const float *dlogp_dev, void *dhidden_dev, void *dhead_dev, void *workspace_dev,
                         int64_t workspace_bytes, void *stream);

/* loss = -sum w_t logp_t / sum w (0 where sum w is 0) and its gradients: a_t = w_t, scale = 1 / (T sum w).  stats_dev: 2 fp32, loss and sum of the
 * weights.  logp_dev, lse_dev: rows fp32.  dhidden_dev, dhead_dev: as above. */
int ps_head_cross_entropy(const ps_head *head, const float *weights_dev, float *stats_dev, float *logp_dev, float *lse_dev, void *dhidden_dev, void *dhead_dev,
                          void *workspace_dev, int64_t workspace_bytes, void *stream);

/* ------------------------------------------------------------------------------------------------------------------
 * Activations in 8 bits.  PS_PACK_BLOCK columns of a row share a power of two u = 2^(s - 127), s a byte:
 *     u = 2^(floor(log2 max|x|) - 6), at least 2^-126;     code = x / u rounded to the nearest integer (ties to even), cut to +-127;     value = code u
 * A block with an infinity or a NaN has s = 255 and reads back as NaN.  Rows of codes are padded with zeros to a multiple of PS_PACK_BLOCK:
 * codes_dev: rows * round_up(cols, PS_PACK_BLOCK) bytes, 16-byte aligned; scales_dev: rows * ceil(cols / PS_PACK_BLOCK) bytes.  Values are exact in bf16
 * and fp32.  dtype: ps_grad_dtype of the activations (fp32 or bf16).
 * ------------------------------------------------------------------------------------------------------------------ */
#define PS_PACK_BLOCK 32

int ps_pack8(const void *x_dev, int dtype, int64_t rows, int64_t cols, int64_t row_stride, int8_t *codes_dev, uint8_t *scales_dev, void *stream);
int ps_unpack8(const int8_t *codes_dev, const uint8_t *scales_dev, int64_t rows, int64_t cols, void *out_dev, int dtype, int64_t row_stride, void *stream);

/* Root-mean-square norm of the residual stream, row by row:
 *     total = x + residual, rounded to dtype (x where residual_dev is NULL);     r = 1 / sqrt(mean(total^2) + eps);     n = total r
 * (r to fp32's accuracy wherever it is a number of fp32, whether or not the squares are);
 *     out = n gain, rounded to dtype (n where gain_dev is NULL);     codes, scales = 8 bits of n (before the gain, which the backward pass and
 *     ps_packed_weight_grad apply)
 * total_dev (total_stride elements a row) may be NULL, or the memory of x or of residual (with the same stride); out_dev (dense) may be NULL, or x's memory where
 * its rows are dense too; codes_dev and scales_dev may both be NULL.  rstd_dev: r, rows fp32.  Other overlaps are refused or undefined. */
typedef struct ps_norm {
    const void *x_dev, *residual_dev, *gain_dev;
    int dtype, gain_dtype;                /* ps_grad_dtype each */
    int64_t rows, cols, x_stride, residual_stride, total_stride;
    float eps;                            /* >= 0 */
    void *total_dev, *out_dev;
    int8_t *codes_dev;
    uint8_t *scales_dev;
    float *rstd_dev;
} ps_norm;
int ps_rms_norm(const ps_norm *norm, void *stream);

/* Its backward pass, from the 8 bits (codes_dev, scales_dev) or, where those are NULL, from total:
 *     g = dout gain;     dx = r (g - n mean(g n)) + dtotal, rounded to dtype: the gradient of x and of residual;     dgain = sum over rows of dout n
 * dtotal_dev (what comes back along the residual stream) and gain_dev may be NULL; dgain_dev: cols values of gain_dtype, or NULL.  dx_dev: dense; it may be
 * dout's or dtotal's memory where that is dense (dout's not beyond 8192 columns with a dgain).  Sums have a fixed order.  The workspace (16-byte aligned) is for
 * dgain: it need not be initialised and holds nothing between calls; calls that share one must not overlap in time. */
typedef struct ps_norm_grad {
    const void *dout_dev, *total_dev, *gain_dev, *dtotal_dev;
    const int8_t *codes_dev;
    const uint8_t *scales_dev;
    const float *rstd_dev;
    int dtype, gain_dtype;
    int64_t rows, cols, dout_stride, total_stride, dtotal_stride;
    void *dx_dev, *dgain_dev;
} ps_norm_grad;
int ps_norm_grad_workspace(int64_t rows, int64_t cols, int64_t *bytes);
int ps_rms_norm_grad(const ps_norm_grad *grad, void *workspace_dev, int64_t workspace_bytes, void *stream);

/* The gradient of a weight matrix (outs x cols) whose product took the kept activations n, times a gain, as input:
 *     dweight_jk = gain_k sum_t dout_tj n_tk
 * dout_dev: bf16, rows of `outs` values; n: the 8 bits, which enter the tensor cores exactly; sums in fp32, in a fixed order.  gain_dev: cols values of
 * gain_dtype, or NULL.  dweight_dev: outs x cols, dense, 16-byte aligned, of out_dtype; no input's memory.  The workspace (256-byte aligned, as above) has room for the
 * values of the codes in bf16, for the sums of split tiles (as above), and where cols is no multiple of 8 for aligned rows of the result. */
typedef struct ps_packed_grad {
    const void *dout_dev, *gain_dev;
    const int8_t *codes_dev;
    const uint8_t *scales_dev;
    int gain_dtype, out_dtype;
    int64_t rows, outs, cols, dout_stride;
    void *dweight_dev;
} ps_packed_grad;
int ps_packed_grad_workspace(const ps_packed_grad *grad, int64_t *bytes);
int ps_packed_weight_grad(const ps_packed_grad *grad, void *workspace_dev, int64_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SOFTSYNC_LEARN_H */
