/*
 * evospec_adapt.h -- what the draft model learns from the events that evospec_kl_gate admits (Path B of the EvoSpec paper,
 * Sec. "Online parameter update"): low-rank adapters beside a projection, forward and backward, for the requests of a batch
 * at once; the distillation loss on the retained support (Eq. 5) with its gradient; and an AdamW step over many tensors.
 * Conventions (errors, pointers, streams, workspaces) are those of evospec.h.  What a call writes (outputs, tensors updated in place, its
 * workspace) shares no memory with what it reads, nor one with another; rows of one buffer may lie between one another.  The entries below do not
 * look for that; the Python binding does.
 */
#ifndef EVOSPEC_ADAPT_H
#define EVOSPEC_ADAPT_H

#include "evospec_decode.h"      /* evospec_type */

#ifdef __cplusplus
extern "C" {
#endif

/*
 * `n` adapters of rank `r` (a multiple of 8, at most EVOSPEC_LORA_R_MAX) for one projection from d_in to d_out elements
 * (multiples of 8, at most 2^20).  Smaller ranks are padded with zeros, which changes nothing.
 *   a      dev bf16 [n][r][d_in]      b dev bf16 [n][d_out][r]      scale dev fp32 [n] or NULL (1)
 */
#define EVOSPEC_LORA_R_MAX 64
typedef struct evospec_lora {
    const void *a, *b;
    const float *scale;
    int n, r, d_in, d_out;
} evospec_lora;

/*
 * y[t] += scale * (x[t] A^T) B^T with the adapter of the request that row t belongs to: rows [row_off[s], row_off[s+1]) have
 * adapter[s].  Rows of a request whose adapter is not in [0, n), and rows of none, are left as they are.
 *   x         dev bf16 [T, d_in], rows x_stride elements apart, 16-B aligned
 *   row_off   dev int32 [S + 1], non-decreasing, values clamped to [0, T]       adapter dev int32 [S]
 *   y         dev bf16 [T, d_out], rows y_stride elements apart, 16-B aligned; no overlap with x.  Rounded once.
 *   out_h     dev fp32 [r, T] or NULL: h = x A^T, transposed, for evospec_lora_backward; zeros in columns of rows without an
 *             adapter
 * Sums are fp32.  h goes into the second product as three bf16 numbers, which are all of its 24 bits.  (So a product of an infinity and a
 * finite number may be NaN, not infinite; the same in the backward pass.)
 * T below 2^24, S at most 2^16, strides at most 2^26.
 */
int evospec_lora_forward(const evospec_lora *lora, const void *x, long long x_stride, const int32_t *row_off,
                         const int32_t *adapter, int S, int T, void *y, long long y_stride, float *out_h, void *stream);

/*
 * Its backward pass from dy, the gradient of y:  g = scale * dy B,  dx += g A,  dA = sum_t g[t]^T x[t],
 * dB = sum_t dy[t]^T (scale * h[t]), over all rows of an adapter.
 *   dy        dev bf16 [T, d_out], rows dy_stride elements apart, 16-B aligned
 *   h         dev fp32 [r, T] as evospec_lora_forward left it, or NULL: computed again from x
 *   dx        dev bf16 [T, d_in], rows dx_stride elements apart, 16-B aligned, or NULL; rounded once; no overlap with x or dy
 *   out_da    dev fp32 [n][r][d_in], 16-B aligned      out_db dev fp32 [n][d_out][r], 16-B aligned: written whole (zeros where an
 *             adapter has no rows)
 *   workspace dev, 16-B aligned, at least evospec_lora_backward_workspace_bytes(...) bytes, scratch: enough for every call of
 *             as many rows or fewer, whatever the requests
 * n (d_in + d_out) / 64 below 2^22 (rank 33 and more) or 2^23.
 * Sums are fp32 in an order that depends on the sizes, row_off and adapter only: the same inputs give the same bits.
 */
int evospec_lora_backward_workspace_bytes(const evospec_lora *lora, int S, int T, size_t *out_bytes /*host*/);
int evospec_lora_backward(const evospec_lora *lora, const void *x, long long x_stride, const float *h, const void *dy,
                          long long dy_stride, const int32_t *row_off, const int32_t *adapter, int S, int T, void *dx,
                          long long dx_stride, float *out_da, float *out_db, void *workspace, size_t workspace_bytes,
                          void *stream);

/*
 * Distillation on the retained support.  For event e, with z_j = h[e] . W_lm[support[e, j]] (as evospec_kl_gate's draft logits),
 * p = softmax(target[e] / T) and q = softmax(z / T) over the event's support:
 *   loss[e] = weight[e] T^2 sum_j p_j (log p_j - log q_j)          d loss[e] / d h[e] = weight[e] T sum_j (q_j - p_j) W_lm[support[e, j]]
 * An entry whose id is not in [0, V) is not in the support (evospec_kl_gate leaves -1).  An event without an entry, or whose
 * target logits are all -inf, has loss 0 and gradient 0; a NaN among another event's numbers makes both NaN.
 *   h         dev bf16 [E, d]         W_lm dev bf16 [V, d], both 16-B aligned; d a multiple of 8, at most EVOSPEC_KD_D_MAX
 *   support   dev int32 [E, K], K at most EVOSPEC_KD_K_MAX         target dev fp32 [E, K]         weight dev fp32 [E] or NULL (1)
 *   out_loss  dev fp32 [E]            out_dh dev `type` (EVOSPEC_BF16 or EVOSPEC_FP32) [E, d], 16-B aligned
 *   out_draft dev fp32 [E, K]: z, NaN where the entry is not in the support.  No output overlaps an input.
 *   workspace dev, 16-B aligned, at least evospec_kd_loss_workspace_bytes(E, K, d) bytes, scratch (fewer events can need more: their rows
 *             are split)
 * T at least 2^-126 and finite.  Logits and gradients are summed in fp32, the loss in 64 bits from the logits.  (The gradient
 * is a difference of two such sums: its error is relative to sum (p + q) |W|, also where p is nearly q.)  A logit of -inf (a sum past fp32's range)
 * is a share of zero; one of +inf makes its event's loss and gradient NaN.  E < 2^20.
 */
#define EVOSPEC_KD_K_MAX 1024
#define EVOSPEC_KD_D_MAX 16384
int evospec_kd_loss_workspace_bytes(int E, int K, int d, size_t *out_bytes /*host*/);
int evospec_kd_loss(const void *h, int E, int d, const void *W_lm, int V, const int32_t *support, const float *target,
                    const float *weight, int K, float T, int type, float *out_loss, void *out_dh, float *out_draft,
                    void *workspace, size_t workspace_bytes, void *stream);

/* What the moments of AdamW are kept in. */
typedef enum evospec_moments { EVOSPEC_MOMENTS_FP32 = 0, EVOSPEC_MOMENTS_8BIT = 1 } evospec_moments;
#define EVOSPEC_ADAMW_BLOCK 256  /* elements that share a scale */

/* A parameter of n elements and its gradient, contiguous, 16-B aligned. */
typedef struct evospec_adamw_tensor {
    void *param;
    const void *grad;
    long long n;
} evospec_adamw_tensor;

/*
 * (A tensor has at most 2^33 elements.)  Blocks of EVOSPEC_ADAMW_BLOCK elements of the flat buffers below, in which the tensors follow one another, each from a block
 * of its own on (elements behind a tensor's last are zeros once a step has run).
 */
int evospec_adamw_blocks(const evospec_adamw_tensor *tensors /*host [count]*/, int count, long long *out_blocks /*host*/);

/*
 * One step of AdamW over `count` tensors, for every element, with g = grad * grad_scale:
 *   m = beta1 m + (1 - beta1) g      v = beta2 v + (1 - beta2) g^2
 *   p = p (1 - lr weight_decay) - lr (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps)
 * in fp32, from the moments before they are rounded.  (A v below 2^-126 may count as 0; root and reciprocal are right to about the last bit.)
 * The moments' products and sums are rounded one by one, so that their codes are the same wherever the formulas are computed in that order.
 *   param_type  of all parameters (fp16, bf16, fp32); grad_type: the same, or EVOSPEC_FP32
 *   kind        EVOSPEC_MOMENTS_FP32: m and v dev fp32 [blocks * 256], scales NULL
 *               EVOSPEC_MOMENTS_8BIT: m and v dev uint8 [blocks * 256], scales dev fp32 [blocks][2], of m and of v
 *   master      dev fp32 [blocks * 256] or NULL: what p is read from and written to; the parameters become its rounded values.
 *               NULL: p is the parameter.
 *   t           >= 1, the number of this step            eps at least 2^-126, as fp32
 *   schedule    dev fp32 [2] or NULL: {lr, t} read on the GPU in place of the arguments, for a captured graph that is replayed
 *   grad_scale  dev fp32 [1] or NULL (1).  If it is infinite or NaN, the step changes nothing.
 * 8 bits: a value is code * scale, the scale of a block the least power of two from 2^-100 to 2^100 that takes its largest finite
 * magnitude (larger ones saturate).  m is e4m3 (largest 448, 0x7f is NaN).  v has 5 exponent bits (bias 15) and 3 mantissa bits and no sign, largest 61440
 * (code 0xf7); a v above zero has code 1 at least.  The low 20 of fp32's 23 mantissa bits are dropped after 16 random
 * bits are added at their top (magnitudes below the smallest normal number: with its exponent), so that a moment is right
 * on average: it moves by less than half a step of 3 mantissa bits at a time, and rounding to nearest would leave it where it
 * is.  The random bits of an element are a hash of its place in the flat buffers, seed and t: its low half is m's, its high half v's,
 *   x = place * 0x9e3779b1 + seed * 0x85ebca6b + t * 0xc2b2ae35;  x = (x ^ x >> 16) * 0x21f0aaad;  x = (x ^ x >> 15) * 0x735a2d97;  x ^ x >> 15
 * in 32 bits.  An element whose moments are not finite gets NaN for m and the largest code for v.
 */
int evospec_adamw_step(const evospec_adamw_tensor *tensors /*host [count]*/, int count, int param_type, int grad_type, int kind,
                       void *m, void *v, float *scales, float *master, double lr, double beta1, double beta2, double eps,
                       double weight_decay, long long t, uint32_t seed, const float *schedule, const float *grad_scale,
                       void *stream);

/* Moments of 8 bits as values: out_m, out_v dev `type` (EVOSPEC_BF16 or EVOSPEC_FP32) [blocks * 256], 16-B aligned. */
int evospec_adamw_moments(const void *m, const void *v, const float *scales, long long blocks, int type, void *out_m, void *out_v,
                          void *stream);

#ifdef __cplusplus
}
#endif
#endif /* EVOSPEC_ADAPT_H */
