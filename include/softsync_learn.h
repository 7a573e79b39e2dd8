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

#ifdef __cplusplus
}
#endif
#endif /* SOFTSYNC_LEARN_H */
