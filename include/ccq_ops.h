/*
 * ccq_ops.h -- C ABI of the operators around the CCQ token mixer: the embedding
 * lookup that feeds a stack of mixers, the gated group norm after the mixer's
 * read, the clipped policy loss at the end of the stack, and the AdamW update of
 * its weights.  Same library and conventions as ccq.h:
 *   - pointers are DEVICE pointers owned by the caller (host arrays are named so),
 *     nothing is allocated, calls are asynchronous on `stream`, argument errors
 *     are reported through the return value and ccq_last_error();
 *   - row strides are in elements; the elements of a row are contiguous.  Any
 *     stride >= the row's length and any base address that the element type
 *     allows is accepted; rows that start on 16-byte boundaries are faster;
 *   - sums, statistics and exponentials are fp32 whatever the storage type, and
 *     every sum has a fixed order: the same call gives the same bits;
 *   - an index outside its range leaves CCQ_ERR_INDEX for ccq_device_status().
 */
#ifndef CCQ_OPS_H_
#define CCQ_OPS_H_

#include "ccq.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------ embedding */

/*
 * out[i, :] = scale * table[ids[i], :], i < n.
 *   table     [rows, width] in dtype, row stride table_stride.
 *   ids       [n], id_bytes 4 (int32) or 8 (int64).
 *   out       [n, width] in dtype, row stride out_stride.
 * The product is formed in fp32 and rounded once.  An id outside [0, rows) gives a
 * zero row and CCQ_ERR_INDEX.
 */
CCQ_API ccq_status ccq_embed(const void *table, ccq_dtype dtype, int64_t table_stride, const void *ids,
                             int id_bytes, int64_t n, int64_t rows, int width, float scale, void *out,
                             int64_t out_stride, void *stream);

/*
 * The gradient of the table: dtable[r, :] = scale * sum over i with ids[i] = r of
 * dout[i, :], for every row r (rows that no id names are zero).
 *   dout       [n, width] in dtype, row stride dout_stride.
 *   padding_id an id whose row gets no gradient (zero), or negative: none.  Its rows of
 *              dout are not read.
 *   dtable     [rows, width] in grad_dtype, row stride dtable_stride; written in full.
 *   workspace  ccq_embed_grad_workspace_size() bytes, 16-byte aligned (NULL where that is 0).
 * The ids are sorted (stably), then every run of equal ids is summed in fp32 in ascending
 * i within pieces whose bounds depend on the ids alone, and the pieces in a fixed order.  An id
 * outside [0, rows) contributes nothing and leaves CCQ_ERR_INDEX.
 * n <= 2^30, rows <= 2^23.
 */
CCQ_API ccq_status ccq_embed_grad(const void *dout, ccq_dtype dtype, int64_t dout_stride, const void *ids,
                                  int id_bytes, int64_t n, int64_t rows, int width, float scale,
                                  int64_t padding_id, void *dtable, ccq_dtype grad_dtype,
                                  int64_t dtable_stride, void *workspace, size_t workspace_bytes,
                                  void *stream);

/* Workspace bytes ccq_embed_grad needs.  Host-only. */
CCQ_API ccq_status ccq_embed_grad_workspace_size(int64_t n, int64_t rows, int width, size_t *bytes);

/* ------------------------------------------------------- group norm, activation */

typedef enum { CCQ_ACT_NONE = 0, CCQ_ACT_SILU = 1, CCQ_ACT_SIGMOID = 2 } ccq_activation;

/*
 * Group norm of tokens with channels last, and an activation.  The statistics are per
 * token and group, so a token's result depends on no other token; with groups = heads it is
 * what follows the mixer's read (o viewed as [tokens, H * Dv]).  For each token and each
 * group of d = channels / groups channels
 *   mu   = mean(x) (0 with centered = 0),  rstd = 1 / sqrt(mean((x - mu)^2) + eps)
 *   u    = (x - mu) rstd * weight + bias
 *   y    = u * act(gate)  with a gate,   act(u)  without.
 *   x, gate, y     [tokens, channels] in dtype, with row strides (gate may be NULL).
 *   weight, bias   [channels] in param_dtype (each may be NULL: 1 and 0).
 * tokens and row strides below 2^31, channels up to 2^24.
 */
CCQ_API ccq_status ccq_group_norm(const void *x, int64_t x_stride, const void *gate, int64_t gate_stride,
                                  const void *weight, const void *bias, ccq_dtype dtype,
                                  ccq_dtype param_dtype, void *y, int64_t y_stride, int64_t tokens,
                                  int channels, int groups, int centered, float eps, ccq_activation act,
                                  void *stream);

/*
 * Gradients of ccq_group_norm for a given dy.  Nothing is kept from the forward: the
 * statistics are formed again from x.
 *   dy [tokens, channels] with its row stride; dx, dgate [tokens, channels] in dtype with
 *   row strides (dgate NULL exactly when gate is); dweight, dbias [channels] in param_dtype
 *   (each may be NULL).
 *   workspace  ccq_group_norm_bwd_workspace_size() bytes, 16-byte aligned: the partial sums of
 *              dweight and dbias.
 */
CCQ_API ccq_status ccq_group_norm_bwd(const void *x, int64_t x_stride, const void *gate, int64_t gate_stride,
                                      const void *weight, const void *bias, const void *dy,
                                      int64_t dy_stride, ccq_dtype dtype, ccq_dtype param_dtype, void *dx,
                                      int64_t dx_stride, void *dgate, int64_t dgate_stride, void *dweight,
                                      void *dbias, int64_t tokens, int channels, int groups, int centered,
                                      float eps, ccq_activation act, void *workspace,
                                      size_t workspace_bytes, void *stream);

/* Workspace bytes ccq_group_norm_bwd needs.  Host-only. */
CCQ_API ccq_status ccq_group_norm_bwd_workspace_size(int64_t tokens, int channels, int groups,
                                                     ccq_dtype dtype, size_t *bytes);

/* ---------------------------------------------------------------- policy loss */

typedef struct {
    float clip_low, clip_high; /* the ratio is held in [1 - clip_low, 1 + clip_high]      */
    float kl_coef;             /* weight of the KL term; 0 or no reference: none            */
    float temperature;         /* the logits are divided by it; 4.3e-39 to 1e30             */
    float grad_scale;          /* factor of dlogits (not of the loss)                       */
} ccq_policy_params;

/* clip 0.2 and 0.2, kl_coef 0, temperature 1, grad_scale 1. */
CCQ_API void ccq_default_policy_params(ccq_policy_params *p);

/*
 * Clipped policy loss with a KL term over token logits, and its gradient, in one call.
 * With z = logits / temperature, logp_i = z_i[a_i] - log sum_j exp z_i[j],
 * r_i = exp(logp_i - old_i) and d_i = ref_i - logp_i:
 *   loss = sum_i w_i (-min(r_i A_i, clip(r_i, 1 - clip_low, 1 + clip_high) A_i)
 *                     + kl_coef (exp(d_i) - d_i - 1))
 *   dlogits_i[j] = grad_scale dloss / dlogits_i[j]   (old, ref, A, w are constants)
 *   logits    [n, vocab] in dtype, row stride logits_stride (-inf entries allowed).
 *   actions   [n], id_bytes 4 or 8.
 *   old_logp, advantages [n] fp32; ref_logp [n] fp32 or NULL; weights [n] fp32 or NULL (1 / n).
 *   loss      [1] fp32;  logp [n] fp32 or NULL;
 *   dlogits   [n, vocab] in dtype, row stride dlogits_stride, or NULL (loss and logp alone).
 *             May be the logits themselves (same address and stride).
 *   workspace ccq_policy_loss_workspace_size() bytes, 16-byte aligned.
 * A token of weight 0 is masked: its logits are not read, its action, advantage and
 * log-probabilities (which may be anything) not used, its logp and its row of dlogits are 0.
 * An action outside [0, vocab) masks its token in the same way and, where the weight is not 0,
 * leaves CCQ_ERR_INDEX.
 */
CCQ_API ccq_status ccq_policy_loss(const void *logits, ccq_dtype dtype, int64_t logits_stride,
                                   const void *actions, int id_bytes, const float *old_logp,
                                   const float *ref_logp, const float *advantages, const float *weights,
                                   int64_t n, int vocab, const ccq_policy_params *p, float *loss,
                                   float *logp, void *dlogits, int64_t dlogits_stride, void *workspace,
                                   size_t workspace_bytes, void *stream);

/* Workspace bytes ccq_policy_loss needs.  Host-only. */
CCQ_API ccq_status ccq_policy_loss_workspace_size(int64_t n, size_t *bytes);

/*
 * logp[i] = log softmax(logits_i / temperature)[a_i]: the old and reference
 * log-probabilities of a policy loss.  An action outside [0, vocab) gives NaN and
 * CCQ_ERR_INDEX.
 */
CCQ_API ccq_status ccq_token_logp(const void *logits, ccq_dtype dtype, int64_t logits_stride,
                                  const void *actions, int id_bytes, int64_t n, int vocab,
                                  float temperature, float *logp, void *stream);

/* --------------------------------------------------------------------- AdamW */

/* Elements that share a scale in the 8-bit state. */
#define CCQ_ADAMW_BLOCK 256

/* One tensor of an update: device pointers, and its number of elements. */
typedef struct {
    void *param;      /* n, in param_dtype                                                  */
    const void *grad; /* n, in grad_dtype                                                   */
    void *m, *v;      /* n: fp32, or one e4m3 byte each with 8-bit states                     */
    float *scale;     /* 8-bit states: [ceil(n / CCQ_ADAMW_BLOCK)][2], the scales of m and v  */
    float *master;    /* n fp32, or NULL                                                    */
    int64_t n;
} ccq_adamw_tensor;

typedef struct {
    double lr, beta1, beta2, eps, weight_decay; /* double: 1 - beta is formed before it is rounded */
    int64_t step;                               /* 1 for the first update                          */
} ccq_adamw_params;

/*
 * One AdamW update of `count` tensors (HOST array), in place:
 *   g = grad * (grad_scale ? *grad_scale : 1)      (a device scalar, e.g. from gradient clipping)
 *   m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2
 *   p = p (1 - lr weight_decay) - lr / (1 - beta1^step) * m / (sqrt(v) / sqrt(1 - beta2^step) + eps)
 * in fp32; eps is 0 or at least 2^-126.  With a master copy p is the master, and param receives its rounded value; master is
 * NULL for all tensors or for none, and needs param_dtype BF16.
 * state_bits 32: m and v are fp32.
 * state_bits 8: per element one e4m3 byte for m and one for sqrt(v), over a power-of-two scale
 * for each CCQ_ADAMW_BLOCK consecutive elements (the smallest 2^e >= 2^-100 with every finite value
 * <= 448 * 2^e).  The update uses the unrounded moments; storing them rounds up where the
 * fraction between two neighbouring e4m3 values reaches a threshold that moves with the
 * element's index i and the step by Weyl's sequence, t = (i 0x6A09E667 + step 0x9E3779B1) mod 2^32
 * (1 - t 2^-32 for v, its complement for m), so that over the steps the stored moments follow
 * changes far below an e4m3 step: beta2 = 0.999 moves v by a thousandth where its neighbours are an
 * eighth apart, which rounding to nearest would lose for good.  A v > 0 is never stored as 0.
 * Moments that are not finite are stored as NaN in their own element.
 * A tensor with n = 0 is skipped.  Any number of tensors; 482 share a launch.
 * `params` is read by the call: a call captured in a graph keeps its lr and step, and with the step the bias
 * corrections and the thresholds of the 8-bit rounding, at every replay (grad_scale, a device
 * scalar, is read anew).  A training step's graph ends before this call.
 */
CCQ_API ccq_status ccq_adamw_step(const ccq_adamw_tensor *tensors, int count, ccq_dtype param_dtype,
                                  ccq_dtype grad_dtype, int state_bits, const ccq_adamw_params *p,
                                  const float *grad_scale, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* CCQ_OPS_H_ */
