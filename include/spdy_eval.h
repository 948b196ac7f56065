/*
 * spdy_eval.h - C ABI of the operators around the search: evaluating a stitched model and tuning the pruned one
 * (NVIDIA B200, sm_100a; part of libspdy_dp.so).
 *
 * SPDY's search (Section 3.3, Algorithm 4) asks its caller for the calibration loss of the model stitched together
 * for a profile (Section 3.4); the pruned model is then tuned against the dense one.  The operators here carry that
 * work on the device: linear layers with their epilogue, layer normalisation with its gradients, log probabilities
 * of given tokens with entropy and top alternatives, from logits or straight from an output layer's input and weight with the
 * gradients by both, the distillation loss against the dense model's top log probabilities with its gradient, and AdamW steps.
 * spdy_linear has no backward call: its input's gradient is the product with the transposed
 * weight, its weight's gradient is left to the caller.
 *
 * Common rules
 *   - All pointers are device pointers on the current device unless they say "host"; the work is enqueued on
 *     `cuda_stream` (a cudaStream_t as void*, NULL = the default stream) and the call returns.  Nothing is
 *     allocated and nothing is kept between calls, so every call may be captured into a CUDA graph.
 *   - Matrices are row-major with unit column stride; ld... is the row stride in elements and at least the row
 *     length.  Pointers need the alignment of their element type only; wide accesses are used where the addresses
 *     allow.  Outputs may not overlap inputs except where a function says so.
 *   - Sums, statistics and gradients of parameters are held in fp32; 16-bit outputs (an output layer's dweight among them) are
 *     rounded once.  No atomics on floating-point data: the same call on the same data gives the same bits.
 *   - Rows may be zero in number, and spdy_linear's columns: the call is a no-op (parameter gradients of no rows are written as
 *     0).  Rows of no columns (D = 0, V = 0) have no mean and no distribution: SPDY_ERR_INVALID_ARG.
 *   - At most 2^31 - 1 blocks per launch: rows beyond that number (times up to 8 for long rows) are SPDY_ERR_UNSUPPORTED.
 * Errors: SPDY_ERR_INVALID_ARG (null pointer, size or stride out of range, unknown type, bad alignment),
 * SPDY_ERR_WORKSPACE_TOO_SMALL, SPDY_ERR_UNSUPPORTED (a size beyond a stated limit), SPDY_ERR_CUDA.
 */
#ifndef SPDY_EVAL_H
#define SPDY_EVAL_H

#include "spdy_dp.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum spdy_dtype { SPDY_F32 = 0, SPDY_BF16 = 1, SPDY_F16 = 2 } spdy_dtype;

typedef enum spdy_activation {
    SPDY_ACT_NONE = 0,
    SPDY_ACT_RELU = 1, /* max(z, 0); NaN stays NaN */
    SPDY_ACT_GELU = 2, /* z (1 + erf(z / sqrt 2)) / 2, within 2^-20 (1 + z^2 / 16) of itself, the negative tail too; 0 at -inf */
    SPDY_ACT_SILU = 3  /* z / (1 + exp(-z)), within 2^-20 (1 + |z| / 8) of itself; 0 at -inf */
} spdy_activation;

/*
 * y[m][n] = act(sum_k x[m][k] w[n][k] + bias[n]) + residual[m][n]
 *   x [M][K], w [N][K], residual [M][N]: `dtype` (SPDY_BF16 or SPDY_F16; fp32 operands are refused), products summed in
 *   fp32.  bias [N] of `bias_dtype` (`dtype` or SPDY_F32) and residual may be NULL.  y [M][N] is `out_dtype`: `dtype` or
 *   SPDY_F32.  y may be the residual itself (same pointer, stride and type).
 *   workspace: spdy_linear_workspace_bytes(...) bytes, 256-byte aligned, contents undefined afterwards; 0 bytes (and NULL)
 *   when the query says 0.  It holds copies of operands whose rows do not start on 16-byte boundaries.
 *   K = 0 gives act(bias) + residual.
 */
size_t spdy_linear_workspace_bytes(const void *x, int64_t ldx, const void *w, int64_t ldw, int dtype, int64_t M, int64_t N,
                                   int64_t K);
int spdy_linear(const void *x, int64_t ldx, const void *w, int64_t ldw, int dtype, const void *bias, int bias_dtype,
                const void *residual, int64_t ldres, int activation, int64_t M, int64_t N, int64_t K, void *y, int64_t ldy,
                int out_dtype, void *workspace, size_t workspace_bytes, void *cuda_stream);
/*
 * The kernels of spdy_linear wait on barriers between their warps with a limit of about two seconds of polling (time in which
 * the kernel is preempted does not count); a wait that runs out is counted and what was waited for is NaN in y (never seen; it
 * would mean a broken device or library).  Reads and clears that
 * count on the current device, waiting for `cuda_stream`: SPDY_OK, or SPDY_ERR_INTERNAL if it was not zero.
 */
int spdy_linear_check_status(void *cuda_stream);

/*
 * Layer normalisation over the D columns of each row:
 *   mean = sum x / D,  rstd = 1 / sqrt(sum (x - mean)^2 / D + eps),  y = (x - mean) rstd weight + bias
 *   x, y [R][D] of `dtype`; weight, bias [D] of `param_dtype` (`dtype` or SPDY_F32), either may be NULL (1 and 0);
 *   mean, rstd [R] fp32, either may be NULL.  y may be x itself.  eps >= 0 and finite.
 */
int spdy_layer_norm(const void *x, int64_t ldx, int dtype, const void *weight, const void *bias, int param_dtype, int64_t R,
                    int64_t D, float eps, void *y, int64_t ldy, float *mean, float *rstd, void *cuda_stream);

/*
 * Its gradients, with u = dy weight and h = (x - mean) rstd of a row:
 *   dx = rstd (u - sum u / D - h sum(u h) / D),  dweight = sum over rows of dy h,  dbias = sum over rows of dy
 *   dx [R][D] of `dtype` (may be dy or x itself); dweight, dbias [D] fp32, either may be NULL.  The rows' contributions are
 *   added in a fixed order through `workspace` (spdy_layer_norm_backward_workspace_bytes(R, D, dtype) bytes, 256-byte aligned).
 */
size_t spdy_layer_norm_backward_workspace_bytes(int64_t R, int64_t D, int dtype);
int spdy_layer_norm_backward(const void *dy, int64_t lddy, const void *x, int64_t ldx, int dtype, const void *weight,
                             int param_dtype, const float *mean, const float *rstd, int64_t R, int64_t D, void *dx,
                             int64_t lddx, float *dweight, float *dbias, void *workspace, size_t workspace_bytes,
                             void *cuda_stream);

/*
 * Log probabilities of given tokens under softmax(logits / temperature), with each row's entropy and its most probable
 * alternatives:
 *   lse = log sum_v exp(x_v / T),  logprob = x_token / T - lse,  entropy = - sum_v p_v log p_v
 *   logits [R][V] of `dtype` (V <= 2^31 - 65); tokens [R] int32 or int64 (`index_bits` 32 or 64), may be NULL when logprob is;
 *   logprob, entropy, lse [R] fp32, each may be NULL.  top_ids [R][top_k] int32 and top_logprobs [R][top_k] fp32: the top_k
 *   largest logits in descending order, equal ones by ascending id; 0 <= top_k <= SPDY_TOP_MAX, top_k <= V.
 *   temperature > 0, finite.
 *   A negative token means "no token": logprob 0, no gradient.  A token >= V gives NaN (logprob and the row's gradient).
 *   -inf marks ids that are not allowed: probability 0, nothing added to the entropy.  A row with nothing left (all -inf)
 *   has lse = -inf, logprob = -inf, entropy = 0, top_logprobs = -inf and gradient 0.  A row holding NaN or +inf has lse,
 *   logprob and entropy NaN; among the alternatives NaN ranks below -inf.
 */
#define SPDY_TOP_MAX 128
int spdy_token_logprobs(const void *logits, int64_t ld, int dtype, const void *tokens, int index_bits, int64_t R, int64_t V,
                        float temperature, int32_t top_k, float *logprob, float *entropy, float *lse, int32_t *top_ids,
                        float *top_logprobs, void *cuda_stream);

/*
 * The gradient of sum_r grad_logprob[r] logprob[r] + grad_entropy[r] entropy[r]:
 *   dlogits_v = (grad_logprob ([v = token] - p_v) - grad_entropy p_v (log p_v + entropy)) / T
 *   lse, entropy [R]: what the forward call gave (entropy may be NULL when grad_entropy is); grad_logprob, grad_entropy [R]
 *   fp32, either may be NULL (0).  dlogits [R][V] of `dtype`, may be the logits themselves.
 * An lse in fp32 is off by up to 2^-24 |lse|, and every p from it by that much relative to itself; in rows whose largest logit
 * over T is beyond 1e7 (an all-masked row under a finite mask of -1e9) it no longer tells how many ids share the mass: p is then at
 * most 1 each.  spdy_token_logprobs_with_grad does the forward and this in one call: memory is read once as far as the rows in flight
 * fit on chip, and the gradient comes from the sums themselves, whatever their size.  lse (and entropy with grad_entropy) are
 * required there too.
 */
int spdy_token_logprobs_backward(const void *logits, int64_t ld, int dtype, const void *tokens, int index_bits, int64_t R,
                                 int64_t V, float temperature, const float *lse, const float *entropy,
                                 const float *grad_logprob, const float *grad_entropy, void *dlogits, int64_t lddl,
                                 void *cuda_stream);
int spdy_token_logprobs_with_grad(const void *logits, int64_t ld, int dtype, const void *tokens, int index_bits, int64_t R,
                                  int64_t V, float temperature, const float *grad_logprob, const float *grad_entropy,
                                  float *logprob, float *entropy, float *lse, void *dlogits, int64_t lddl,
                                  void *cuda_stream);

/*
 * The same values under softmax((hidden weight^T + bias) / temperature), straight from a head's input and weight: the logits
 *   x_rv = sum_d hidden[r][d] weight[v][d] + bias[v]   (products summed in fp32)
 * are never kept.
 *   hidden [R][D], weight [V][D]: `dtype` (SPDY_BF16 or SPDY_F16), D >= 1; bias [V] of `bias_dtype` (`dtype` or SPDY_F32), may be NULL;
 *   a bias of -inf marks ids that are not allowed.  R, V and D below 2^31 - 65536.
 *   tokens, logprob, entropy, lse, rows with nothing left, NaN and infinities: as spdy_token_logprobs has them.  A logit is the fp32 sum
 *   of the tensor cores' sums of up to 384 products, which are cut where fp32 additions round: each is short by at most 3e-6 of its
 *   magnitudes (measured: lse by 4e-7 of itself, 1.2e-6 where all products are positive).  What fp32 holds exactly is exact, and columns
 *   of zeros change nothing.  Up to 4 rows are added up in fp32.
 * Gradients of sum_r grad_logprob[r] logprob[r] + grad_entropy[r] entropy[r], with g_rv the gradient by x_rv
 * (spdy_token_logprobs_backward's dlogits):
 *   dhidden[r][d] = sum_v g_rv weight[v][d],   dweight[v][d] = sum_r g_rv hidden[r][d],   dbias[v] = sum_r g_rv
 *   dhidden [R][D] and dweight [V][D] of `dtype`, dbias [V] fp32 (from sums in fp32); each may be NULL.  They may not overlap the inputs.
 *   g is computed in fp32 and rounded to 16 bits once, as the operand of the two products (in half precision times a power of two that
 *   brings its largest row near 2^14); for up to 64 rows it is their operand as the sum of two such numbers.  ..._with_grad may keep the
 *   logits in between, as logarithms in 16 bits (with dbias 23): p is then within 3.5e-4 of itself (half precision 1.8e-4; with dbias 2.8e-6 and 1.4e-6), and 0 where it is 2^-64 (2^-32) of a neighbouring
 *   id's; at the token g comes from its logit in fp32.  A row of hidden that is not finite spoils dweight, with or without a token.
 *   ..._backward takes lse (and entropy with grad_entropy) from the forward call, ..._with_grad computes all in one call.
 *   workspace: ..._workspace_bytes(...) bytes, 256-byte aligned, contents undefined afterwards; `forward` and `gradients` say what the
 *   call computes (gradients: 0 none, 1 without dbias, 2 with it).  Of g it holds as many ids at a time as 256 MB hold
 *   (2048 at least), or, in ..._with_grad, as many rows as 512 MB hold, and then 4 V D bytes of dweight's sums; of few
 *   tiles (V x D small) the sums lie there in up to 64 parts.
 * spdy_linear_check_status reports for these kernels too.
 */
size_t spdy_linear_token_logprobs_workspace_bytes(const void *hidden, int64_t ldh, const void *weight, int64_t ldw, int dtype,
                                                  int64_t R, int64_t V, int64_t D, int forward, int gradients);
int spdy_linear_token_logprobs(const void *hidden, int64_t ldh, const void *weight, int64_t ldw, int dtype, const void *bias,
                               int bias_dtype, const void *tokens, int index_bits, int64_t R, int64_t V, int64_t D,
                               float temperature, float *logprob, float *entropy, float *lse, void *workspace,
                               size_t workspace_bytes, void *cuda_stream);
int spdy_linear_token_logprobs_backward(const void *hidden, int64_t ldh, const void *weight, int64_t ldw, int dtype,
                                        const void *bias, int bias_dtype, const void *tokens, int index_bits, int64_t R,
                                        int64_t V, int64_t D, float temperature, const float *lse, const float *entropy,
                                        const float *grad_logprob, const float *grad_entropy, void *dhidden, int64_t lddh,
                                        void *dweight, int64_t lddw, float *dbias, void *workspace, size_t workspace_bytes,
                                        void *cuda_stream);
int spdy_linear_token_logprobs_with_grad(const void *hidden, int64_t ldh, const void *weight, int64_t ldw, int dtype,
                                         const void *bias, int bias_dtype, const void *tokens, int index_bits, int64_t R,
                                         int64_t V, int64_t D, float temperature, const float *grad_logprob,
                                         const float *grad_entropy, float *logprob, float *entropy, float *lse, void *dhidden,
                                         int64_t lddh, void *dweight, int64_t lddw, float *dbias, void *workspace,
                                         size_t workspace_bytes, void *cuda_stream);

/*
 * Distillation from a teacher's top log probabilities.  p = softmax(logits / temperature) is the student's row, S the ids a
 * row of `ids` names, and
 *   tail != 0: q_j = exp(top_logprobs_j), left = max(0, 1 - sum_j q_j), p_rest = the student's probability outside S,
 *              loss = sum_j q_j (log q_j - log p_{id_j}) + left (log left - log p_rest)
 *   tail == 0: q = softmax(top_logprobs) over the entries (any offset per row is immaterial), loss without the last term
 *   (the divergence from the teacher's distribution over "each of S, or something else", or over S alone).
 *   logits [R][V] of `dtype`; ids [R][K] int32 or int64 with row stride K; top_logprobs [R][K] fp32 with row stride K, taken at
 *   the same temperature; 1 <= K <= SPDY_DISTILL_MAX.  loss, lse, rest [R] fp32 (rest: the log of the sum outside S, written
 *   when tail != 0), each may be NULL in the forward call.
 *   The ids of a row should be distinct; an id that comes twice adds both entries' terms and is in S once.  A negative id is an
 *   entry that is not there; an id >= V makes the row's loss and gradient NaN.  A row without entries has no teacher: with
 *   tail == 0 loss 0 and gradient 0.  Where the student has nothing left outside S (rest = -inf) the tail term is dropped.
 *   A student's row of -inf alone: lse = -inf, loss +inf (0 if no q_j > 0), gradient 0.
 * Gradient of sum_r grad_loss[r] loss[r], with A = sum_j q_j + left (left counted where the tail term is):
 *   dlogits_v = grad_loss / T (A p_v - sum of q_j with id_j = v)   in S
 *               grad_loss / T (A p_v - left p_v / p_rest)          outside
 *   (without the tail A p_v outside).  dlogits [R][V] of `dtype`, may be the logits themselves.
 * From saved sums the gradient is as exact as an fp32 lse and rest let it be (see spdy_token_logprobs_backward), p and p / p_rest at
 * most 1.  spdy_distill_loss_with_grad works from the sums themselves; lse, and rest with the tail, are required there too.
 */
#define SPDY_DISTILL_MAX 256
int spdy_distill_loss(const void *logits, int64_t ld, int dtype, const void *ids, int index_bits, const float *top_logprobs,
                      int64_t R, int64_t V, int32_t K, float temperature, int tail, float *loss, float *lse, float *rest,
                      void *cuda_stream);
int spdy_distill_loss_backward(const void *logits, int64_t ld, int dtype, const void *ids, int index_bits,
                               const float *top_logprobs, int64_t R, int64_t V, int32_t K, float temperature, int tail,
                               const float *lse, const float *rest, const float *grad_loss, void *dlogits, int64_t lddl,
                               void *cuda_stream);
int spdy_distill_loss_with_grad(const void *logits, int64_t ld, int dtype, const void *ids, int index_bits,
                                const float *top_logprobs, int64_t R, int64_t V, int32_t K, float temperature, int tail,
                                const float *grad_loss, float *loss, float *lse, float *rest, void *dlogits, int64_t lddl,
                                void *cuda_stream);

/*
 * An AdamW step over many tensors at once.  For each element, with t = step:
 *   g = grad grad_scale,   m = beta1 m + (1 - beta1) g,   v = beta2 v + (1 - beta2) g^2
 *   param = param (1 - lr weight_decay) - lr / (1 - beta1^t) m / (sqrt(v / (1 - beta2^t)) + eps)
 * in fp32, each operation rounded; the square root and the quotient within 2^-21 of themselves.  With a master copy it is the
 * copy that is stepped, and param that is rounded from it.
 *   tensors, options: host memory, read before the call returns.  A tensor is n contiguous elements; param, grad and master need
 *   the alignment of their types, m and v 16 bytes.  grad NULL: the tensor is left alone.  Memory that is written may belong to one
 *   tensor only.
 *   state_bits 32: m, v fp32 [n].  state_bits 8: m, v bytes [n], m_exp, v_exp bytes [ceil(n / 32)]; all 0 to begin with.
 *     32 consecutive elements share E, the fp32 exponent field (at least 1) of the largest magnitude among them; E = 255: the block
 *     holds a value that is not finite, or one from 2^127 on, and all of it reads as NaN.  Relative to 2^(E - 127) an element is a
 *     floating-point number with 3 bits of mantissa: m has a sign and 4 bits of exponent, field 14 being the binade of the largest
 *     (so that m ends at 2^-16 to 2^-17 of the largest); v has 5 bits, field 30 (2^-31 to 2^-32).  Rounding is stochastic, by 20 random
 *     bits; a positive v is never rounded to 0.  The update uses m and v as they are before this rounding.
 *   keep_zeros: elements whose weight (master, where there is one) is 0 stay 0, and so do their m and v: pruned weights stay pruned.
 *   rounding of 16-bit params without a master: 0 to nearest, 1 stochastic (a change of less than half a step is lost to nearest).
 *   Random bits are a hash of (seed, t modulo 2^32, index in `tensors`, element): the same call gives the same bits.
 *   step >= 1.  step_device, lr_device: device scalars used instead of step and lr, read when the kernel runs, for captured steps
 *   (lr_device needs step_device; a step below 1 counts as 1).  grad_scale, skip: device scalars or NULL; with *skip != 0 nothing is
 *   changed.  Infinities and NaN in grad are not looked for.
 */
typedef struct spdy_adamw_tensor {
    void *param;
    const void *grad;
    float *master; /* NULL, or fp32 [n]: only with 16-bit params */
    void *m, *v;
    uint8_t *m_exp, *v_exp;
    int64_t n;
    float weight_decay;
    int32_t param_dtype, grad_dtype; /* grad: param's type or SPDY_F32 */
    int32_t state_bits, keep_zeros;
    int32_t reserved; /* 0 */
} spdy_adamw_tensor;

typedef struct spdy_adamw_options {
    double lr, beta1, beta2, eps; /* 0 <= beta < 1, eps >= 0 */
    int64_t step;
    uint32_t seed;
    int32_t rounding;
    const float *lr_device;
    const int64_t *step_device;
    const float *grad_scale, *skip;
} spdy_adamw_options;

int spdy_adamw_step(const spdy_adamw_tensor *tensors, int32_t count, const spdy_adamw_options *options, void *cuda_stream);

/*
 * The moments of tensors with state_bits 8 as numbers: m_out[i], v_out[i] (host arrays of device pointers) receive n elements of
 * `out_dtype`, SPDY_F32 or SPDY_BF16 (both hold them exactly; below 2^-133 bf16 rounds).  param, grad and master are not looked at.
 */
int spdy_adamw_moments(const spdy_adamw_tensor *tensors, int32_t count, void *const *m_out, void *const *v_out, int out_dtype,
                       void *cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* SPDY_EVAL_H */
