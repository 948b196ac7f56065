// The distillation loss against a teacher's top log probabilities and its gradient: C entries (spdy_eval.h).
#include "eval_loss.cuh"

using namespace spdy_eval;

namespace {

bool teacher_ok(const void *ids, int bits, const float *top_lp, int64_t R, int32_t K)
{
    return (bits == 32 || bits == 64) && K >= 1 && K <= SPDY_DISTILL_MAX && (R == 0 || (ids && top_lp)) && aligned(ids, bits / 8) && aligned(top_lp, 4);
}

LossArgs base_args(const void *logits, int64_t ld, const void *ids, int bits, const float *top_lp, int64_t R, int64_t V, int32_t K, float temperature)
{
    LossArgs a = {};
    a.logits = logits, a.ld = ld, a.R = R, a.V = V, a.K = K;
    a.c = kLog2e / temperature, a.inv_t = 1.f / temperature, a.temperature = temperature, a.lower = temperature == 1.f ? 0.f : 1.8e-7f;
    a.ids = ids, a.index_bits = bits, a.top_lp = top_lp;
    return a;
}

int run_forward(const LossArgs &a, int dtype, int tail, cudaStream_t stream)
{
    if (tail) return SPDY_EVAL_BY_TYPE(dtype, (rows<T, kDistillTail, kNoGrad>(a, stream)));
    return SPDY_EVAL_BY_TYPE(dtype, (rows<T, kDistill, kNoGrad>(a, stream)));
}

int run_backward(const LossArgs &a, int dtype, int tail, cudaStream_t stream)
{
    if (tail) return SPDY_EVAL_BY_TYPE(dtype, (backward<T, kDistillTail>(a, stream)));
    return SPDY_EVAL_BY_TYPE(dtype, (backward<T, kDistill>(a, stream)));
}

}  // namespace

extern "C" {

int spdy_distill_loss(const void *logits, int64_t ld, int dtype, const void *ids, int index_bits, const float *top_logprobs, int64_t R, int64_t V,
                      int32_t K, float temperature, int tail, float *loss, float *lse, float *rest, void *cuda_stream)
{
    if (!rows_ok(logits, ld, dtype, R, V) || !temperature_ok(temperature) || !teacher_ok(ids, index_bits, top_logprobs, R, K)) return SPDY_ERR_INVALID_ARG;
    if (R == 0) return SPDY_OK;
    LossArgs a = base_args(logits, ld, ids, index_bits, top_logprobs, R, V, K, temperature);
    a.loss = loss, a.lse = lse, a.rest = rest;
    return run_forward(a, dtype, tail, static_cast<cudaStream_t>(cuda_stream));
}

int spdy_distill_loss_backward(const void *logits, int64_t ld, int dtype, const void *ids, int index_bits, const float *top_logprobs, int64_t R,
                               int64_t V, int32_t K, float temperature, int tail, const float *lse, const float *rest, const float *grad_loss,
                               void *dlogits, int64_t lddl, void *cuda_stream)
{
    if (!rows_ok(logits, ld, dtype, R, V) || !rows_ok(dlogits, lddl, dtype, R, V) || !temperature_ok(temperature) ||
        !teacher_ok(ids, index_bits, top_logprobs, R, K))
        return SPDY_ERR_INVALID_ARG;
    if (R == 0) return SPDY_OK;
    if (!lse || !grad_loss || (tail && !rest)) return SPDY_ERR_INVALID_ARG;
    LossArgs a = base_args(logits, ld, ids, index_bits, top_logprobs, R, V, K, temperature);
    a.in_lse = lse, a.in_rest = rest, a.grad = grad_loss, a.dlogits = dlogits, a.lddl = lddl;
    return run_backward(a, dtype, tail, static_cast<cudaStream_t>(cuda_stream));
}

int spdy_distill_loss_with_grad(const void *logits, int64_t ld, int dtype, const void *ids, int index_bits, const float *top_logprobs, int64_t R,
                                int64_t V, int32_t K, float temperature, int tail, const float *grad_loss, float *loss, float *lse, float *rest,
                                void *dlogits, int64_t lddl, void *cuda_stream)
{
    if (!rows_ok(logits, ld, dtype, R, V) || !rows_ok(dlogits, lddl, dtype, R, V) || !temperature_ok(temperature) ||
        !teacher_ok(ids, index_bits, top_logprobs, R, K))
        return SPDY_ERR_INVALID_ARG;
    if (R == 0) return SPDY_OK;
    if (!lse || !grad_loss || (tail && !rest)) return SPDY_ERR_INVALID_ARG;
    LossArgs a = base_args(logits, ld, ids, index_bits, top_logprobs, R, V, K, temperature);
    a.loss = loss, a.lse = lse, a.rest = rest, a.grad = grad_loss, a.dlogits = dlogits, a.lddl = lddl;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (tail) return SPDY_EVAL_BY_TYPE(dtype, (rows<T, kDistillTail, kGrad>(a, stream)));
    return SPDY_EVAL_BY_TYPE(dtype, (rows<T, kDistill, kGrad>(a, stream)));
}

}  // extern "C"
