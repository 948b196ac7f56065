// Log probabilities of given tokens, entropy, top alternatives and their gradients: C entries (spdy_eval.h).
#include "eval_loss.cuh"

namespace spdy_eval {

int sm_count()
{
    static int counts[64];  // 0 = not asked yet; asking twice gives the same answer
    int device = 0;
    if (cudaGetDevice(&device) != cudaSuccess || device < 0 || device >= 64) return 148;
    int n = __atomic_load_n(&counts[device], __ATOMIC_RELAXED);
    if (n == 0) {
        if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device) != cudaSuccess || n <= 0) n = 148;
        __atomic_store_n(&counts[device], n, __ATOMIC_RELAXED);
    }
    return n;
}

}  // namespace spdy_eval

using namespace spdy_eval;

namespace {

bool tokens_ok(const void *tokens, int bits) { return (bits == 32 || bits == 64) && aligned(tokens, bits / 8); }

LossArgs base_args(const void *logits, int64_t ld, const void *tokens, int bits, int64_t R, int64_t V, float temperature)
{
    LossArgs a = {};
    a.logits = logits, a.ld = ld, a.R = R, a.V = V;
    a.c = kLog2e / temperature, a.inv_t = 1.f / temperature, a.temperature = temperature, a.lower = temperature == 1.f ? 0.f : 1.8e-7f;
    a.ids = tokens, a.index_bits = bits;
    return a;
}

}  // namespace

extern "C" {

int spdy_token_logprobs(const void *logits, int64_t ld, int dtype, const void *tokens, int index_bits, int64_t R, int64_t V, float temperature,
                        int32_t top_k, float *logprob, float *entropy, float *lse, int32_t *top_ids, float *top_logprobs, void *cuda_stream)
{
    if (!rows_ok(logits, ld, dtype, R, V) || !temperature_ok(temperature) || !tokens_ok(tokens, index_bits)) return SPDY_ERR_INVALID_ARG;
    if (top_k < 0 || top_k > SPDY_TOP_MAX || top_k > V) return SPDY_ERR_INVALID_ARG;
    if (R == 0) return SPDY_OK;
    if ((logprob && !tokens) || (top_k > 0 && (!top_ids || !top_logprobs))) return SPDY_ERR_INVALID_ARG;
    LossArgs a = base_args(logits, ld, tokens, index_bits, R, V, temperature);
    a.K = top_k;
    a.logprob = logprob, a.entropy = entropy, a.lse = lse, a.top_ids = top_ids, a.top_logprobs = top_logprobs;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (top_k) return SPDY_EVAL_BY_TYPE(dtype, (rows<T, kLogprobsTop, kNoGrad>(a, stream)));
    return SPDY_EVAL_BY_TYPE(dtype, (rows<T, kLogprobs, kNoGrad>(a, stream)));
}

int spdy_token_logprobs_backward(const void *logits, int64_t ld, int dtype, const void *tokens, int index_bits, int64_t R, int64_t V, float temperature,
                                 const float *lse, const float *entropy, const float *grad_logprob, const float *grad_entropy, void *dlogits,
                                 int64_t lddl, void *cuda_stream)
{
    if (!rows_ok(logits, ld, dtype, R, V) || !rows_ok(dlogits, lddl, dtype, R, V) || !temperature_ok(temperature) || !tokens_ok(tokens, index_bits))
        return SPDY_ERR_INVALID_ARG;
    if (R == 0) return SPDY_OK;
    if (!lse || (grad_logprob && !tokens) || (grad_entropy && !entropy)) return SPDY_ERR_INVALID_ARG;
    LossArgs a = base_args(logits, ld, tokens, index_bits, R, V, temperature);
    a.in_lse = lse, a.in_entropy = entropy, a.grad = grad_logprob, a.grad_entropy = grad_entropy, a.dlogits = dlogits, a.lddl = lddl;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    return SPDY_EVAL_BY_TYPE(dtype, (backward<T, kLogprobs>(a, stream)));
}

int spdy_token_logprobs_with_grad(const void *logits, int64_t ld, int dtype, const void *tokens, int index_bits, int64_t R, int64_t V, float temperature,
                                  const float *grad_logprob, const float *grad_entropy, float *logprob, float *entropy, float *lse, void *dlogits,
                                  int64_t lddl, void *cuda_stream)
{
    if (!rows_ok(logits, ld, dtype, R, V) || !rows_ok(dlogits, lddl, dtype, R, V) || !temperature_ok(temperature) || !tokens_ok(tokens, index_bits))
        return SPDY_ERR_INVALID_ARG;
    if (R == 0) return SPDY_OK;
    if (((logprob || grad_logprob) && !tokens) || !lse || (grad_entropy && !entropy)) return SPDY_ERR_INVALID_ARG;
    LossArgs a = base_args(logits, ld, tokens, index_bits, R, V, temperature);
    a.logprob = logprob, a.entropy = entropy, a.lse = lse, a.grad = grad_logprob, a.grad_entropy = grad_entropy, a.dlogits = dlogits, a.lddl = lddl;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    return SPDY_EVAL_BY_TYPE(dtype, (rows<T, kLogprobs, kGrad>(a, stream)));
}

}  // extern "C"
