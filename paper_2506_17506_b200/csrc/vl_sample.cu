// vl_token_sample: checks and dispatch (the kernels are in vl_sample.cuh).
#include <math.h>

#include "vl_sample.cuh"

// (rows of that many entries are short ones, whatever their type and wherever they start: at most 251 vectors of fp32, 126 of 16 bits)
extern "C" uint64_t vl_sample_work(uint64_t n_rows, uint32_t n_vocab) { return n_vocab <= 1000 ? 0 : 4 * n_rows; }

extern "C" int vl_token_sample(int device, const vl_logits *x, const vl_sampling *rules, const float *d_uniform, void *d_tokens,
                               uint32_t token_bytes, float *d_logprob, float *d_drawn_logprob, int32_t *d_kept, void *d_work, uint64_t work_bytes,
                               void *stream)
{
    LogitRows q;
    const int rc = vl_logit_rows(x, &q);
    if (rc != VL_OK) return rc;
    if (x->tokens || !rules) return VL_ERR_INVALID_ARG;
    if (!(rules->top_p > 0.0 && rules->top_p <= 1.0) || !(rules->min_p >= 0.0 && rules->min_p <= 1.0)) return VL_ERR_INVALID_ARG;
    if ((token_bytes != 2 && token_bytes != 4 && token_bytes != 8) || (token_bytes == 2 && q.V > 65535)) return VL_ERR_INVALID_ARG;
    if ((uintptr_t)d_tokens % token_bytes) return VL_ERR_INVALID_ARG;
    if (((uintptr_t)d_uniform | (uintptr_t)d_logprob | (uintptr_t)d_drawn_logprob | (uintptr_t)d_kept) & 3) return VL_ERR_INVALID_ARG;
    if (q.n_rows == 0) return VL_OK;
    const uint64_t work = vl_sample_work(q.n_rows, q.V);
    if (!d_uniform || !d_tokens || (work && (!d_work || ((uintptr_t)d_work & 3) || work_bytes < work))) return VL_ERR_INVALID_ARG;
    const DeviceScope scope(device);
    if (scope.error != cudaSuccess) return VL_ERR_CUDA;
    const SampleRules s{d_uniform, rules->top_k, rules->top_p, rules->min_p,
                        rules->min_p > 0.0 ? log(rules->min_p) / (double)x->scale : -HUGE_VAL, static_cast<uint32_t *>(d_work)};
    const SampleOut o{d_tokens, token_bytes, d_logprob, d_drawn_logprob, d_kept};
    const auto launch = x->dtype == VL_F32 ? vl_sample_f32 : x->dtype == VL_F16 ? vl_sample_f16 : vl_sample_bf16;
    return launch(q, s, o, device, (cudaStream_t)stream) == cudaSuccess ? VL_OK : VL_ERR_CUDA;
}
