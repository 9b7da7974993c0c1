/*
 * ozimmu layers -- the feed-forward layer of a language model on MI355X (gfx950): a linear layer with its epilogue, its
 * gradients, the AdamW step that uses them, and a mixture-of-experts layer for the few tokens of a serving step.
 *
 * Conventions, those of ozimmu.h where they apply
 *   - Matrices hold one token, or one output feature of a weight, per row; the entries of a row are contiguous and rows
 *     are `ld` entries apart (ld >= the entries of a row).  As column-major matrices they are the transposes: one column
 *     a token.
 *   - All matrix, state and workspace pointers are DEVICE pointers owned by the caller, aligned to their element (a
 *     workspace to 256 bytes).  The library allocates nothing and keeps nothing from one call to the next.  Pointers marked [host]
 *     are host pointers.
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream).  Calls are asynchronous on that stream, record
 *     into HIP graphs (kernels only) and return one of the OZIMMU_* status codes; nothing throws or aborts.
 *   - Outputs must not overlap inputs or each other unless an entry point says so.
 *   - Sums, activations and statistics are formed in 32 bits; what is written in 16 bits is rounded to nearest once.
 *     Results are deterministic (no atomics on floating-point values; the order of every sum is fixed by the sizes).
 *   - NaN and infinities go where the formulas take them; no entry point looks for them.
 *   - Sizes of 0 are accepted: no tokens or no output features write nothing, n_in = 0 gives products of 0.  Sizes up to
 *     2^30 - 1 (ozimmu_moe's width and hidden: 2^24), offsets in 64 bits.
 */
#ifndef OZIMMU_LAYERS_H
#define OZIMMU_LAYERS_H

#include <stddef.h>
#include <stdint.h>

#include "ozimmu.h"

#ifdef __cplusplus
extern "C" {
#endif

/* element types */
#define OZIMMU_BF16 0
#define OZIMMU_F16 1
#define OZIMMU_F32 2
#define OZIMMU_E4M3 3 /* 8 bits, AdamW's states only */

/* activations */
#define OZIMMU_ACT_NONE 0
#define OZIMMU_ACT_RELU 1
#define OZIMMU_ACT_GELU 2      /* z Phi(z), Phi the normal distribution function */
#define OZIMMU_ACT_GELU_TANH 3 /* z (1 + tanh(sqrt(2 / pi) (z + 0.044715 z^3))) / 2 */
#define OZIMMU_ACT_SILU 4      /* z / (1 + exp(-z)) */

/*
 * y = act(x w^T + bias) + residual
 *   x [tokens, n_in], w [n_out, n_in], bias [n_out], residual, pre and y [tokens, n_out], all of `type` (BF16, F16, F32).
 *   bias, residual and pre may be NULL.  pre receives x w^T + bias, which ozimmu_linear_grad takes.
 *   residual may be y itself (same pointer and ld).
 * Workspace: ozimmu_linear_workspace_bytes (partial sums where the contraction is divided among work-groups; it may be
 * 0, then NULL is accepted).  aligned = 1: every row of x and w starts on 16 bytes.  Otherwise the size has room for copies of them in
 * such rows; with less, down to the size for aligned = 1, a slower way is taken where they are not.
 */
size_t ozimmu_linear_workspace_bytes(int tokens, int n_in, int n_out, int type, int aligned);
int ozimmu_linear(int tokens, int n_in, int n_out, int type, const void *x, int ldx, const void *w, int ldw, const void *bias,
                  const void *residual, int ldr, int activation, void *pre, int ldpre, void *y, int ldy, void *workspace,
                  size_t workspace_bytes, void *stream);

/*
 * Gradients of ozimmu_linear.  With dz = dy * act'(pre), rounded to `type` for the products (one rounding, to the
 * type the matrix cores take; a float16 dz beyond 65504 becomes an infinity; the bias gradient is summed from the unrounded values):
 *   dx = dz w   [tokens, n_in],   dw = dz^T x   [n_out, n_in],   db = the sum of dz over the tokens   [n_out]
 * (the gradient of the residual is dy itself).  dx, dw and db may each be NULL and are then not formed; pre may be NULL for
 * OZIMMU_ACT_NONE; x may be NULL without dw, w without dx.  act'(0) = 0 for OZIMMU_ACT_RELU.
 * Workspace: as for ozimmu_linear, `aligned` of dy, x and w.
 */
size_t ozimmu_linear_grad_workspace_bytes(int tokens, int n_in, int n_out, int type, int activation, int aligned);
int ozimmu_linear_grad(int tokens, int n_in, int n_out, int type, const void *dy, int lddy, const void *x, int ldx, const void *w,
                       int ldw, const void *pre, int ldpre, int activation, void *dx, int lddx, void *dw, int lddw, void *db,
                       void *workspace, size_t workspace_bytes, void *stream);

/*
 * One AdamW step, in place, over `tensors` tensors of `list` [host, read before the call returns]:
 *   m = beta1 m + (1 - beta1) g,   v = beta2 v + (1 - beta2) g^2,
 *   p = (1 - lr weight_decay) p - lr / (1 - beta1^step)  m / (sqrt(v) / sqrt(1 - beta2^step) + eps)
 * in 32 bits, m and v rounded operation by operation, the quotient to two units.  step counts from 1.
 *   grads [host]  the gradients' pointers, or NULL: those of the list.
 *   state_type OZIMMU_F32: m and v are floats.  OZIMMU_E4M3: blocks of 256 consecutive values (the last one of a tensor may
 *     be shorter) hold m and sqrt(v) as m[i] * m_scale[i / 256] and v[i] * v_scale[i / 256], m[i] and v[i] e4m3 (a sign bit,
 *     4 of exponent, 3 of mantissa, largest value 448, 0x7f a NaN) and the scales float, 1/448 of the block's largest finite
 *     magnitude.  A value between two codes goes to the upper one with the probability of its distance from the
 *     lower, by 32-bit words that depend on the value's place, step and seed only; sqrt(v) > 0 does not become 0.  A NaN or an infinity makes its own m and v NaN,
 *     the others of the block stay what they are.  Where a block's
 *     largest magnitude is below 2^-100, m is held as zeros and sqrt(v) > 0 as the smallest code.
 *   copy, may be NULL: receives p in 16 bits (copy_type BF16 or F16), the weights of the next forward pass.
 * Tensors are arrays of `count` contiguous values at any alignment of their type; they must not overlap.  A launch takes up to 48
 * tensors of the same types that stand behind one another in the list.
 */
typedef struct {
    void *param;
    const void *grad;
    void *m, *v;
    float *m_scale, *v_scale; /* OZIMMU_E4M3 only: (count + 255) / 256 of each */
    void *copy;
    int64_t count;
    int param_type, grad_type, state_type, copy_type;
} ozimmu_adamw_tensor;

int ozimmu_adamw(int tensors, const ozimmu_adamw_tensor *list, const void *const *grads, double lr, double beta1, double beta2,
                 double eps, double weight_decay, long long step, uint32_t seed, void *stream);

/*
 * A mixture-of-experts layer for the tokens of a serving step, 0 <= tokens <= OZIMMU_MOE_TOKENS:
 *   logits = x router^T;  the top_k experts of a token are those of its largest logits, ties to the lowest index;
 *   gate = exp(logit) / the sum of exp(logit) over all experts, or over the chosen ones where `normalise` is not 0;
 *   y = sum over the chosen experts e of  gate_e w_out[e] (silu(w_in[e][0 ... hidden) x) * (w_in[e][hidden ... 2 hidden) x))
 *   x, y [tokens, width]; router [experts, width], w_in [experts, 2 hidden, width], w_out [experts, width, hidden] contiguous;
 *   all of `type`.  chosen [tokens, top_k]: the experts of each token in ascending order; gates: theirs, float.
 * The values of the hidden layer, with their gate, go into the second product as one float or as the sum of two numbers of
 * 16 bits: bfloat16 to 2^-16 of them, float16 to 2^-22, but to no less than 2^-25 (beyond float16's range to 2^-18).  A NaN logit
 * counts as larger than any number.
 * 1 <= top_k <= experts <= OZIMMU_MOE_EXPERTS, top_k <= OZIMMU_MOE_TOP_K.
 */
#define OZIMMU_MOE_TOKENS 64
#define OZIMMU_MOE_EXPERTS 512
#define OZIMMU_MOE_TOP_K 16
size_t ozimmu_moe_workspace_bytes(int tokens, int width, int hidden, int experts, int top_k, int type);
int ozimmu_moe(int tokens, int width, int hidden, int experts, int top_k, int type, int normalise, const void *x, int ldx,
               const void *router, const void *w_in, const void *w_out, int32_t *chosen, float *gates, void *y, int ldy,
               void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif
