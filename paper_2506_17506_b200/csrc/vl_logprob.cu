// vl_token_logprobs: checks and dispatch (the kernels are in vl_logprob.cuh).
#include "vl_logits.cuh"

int vl_logit_rows(const vl_logits *x, LogitRows *q)
{
    if (!x || x->n_vocab == 0 || x->n_vocab > VL_MAX_VOCAB) return VL_ERR_INVALID_ARG;
    if (x->dtype != VL_F32 && x->dtype != VL_F16 && x->dtype != VL_BF16) return VL_ERR_INVALID_ARG;
    const uint32_t size = x->dtype == VL_F32 ? 4 : 2;
    if (x->n_rows > 1 && x->row_stride < x->n_vocab) return VL_ERR_INVALID_ARG;
    if (x->n_rows && (!x->logits || (uintptr_t)x->logits % size)) return VL_ERR_INVALID_ARG;
    if (x->n_rows > (1ull << 40) || x->row_stride > (1ull << 40)) return VL_ERR_INVALID_ARG;
    if (x->n_rows > 1 && x->row_stride > (1ull << 56) / x->n_rows) return VL_ERR_INVALID_ARG;  // (no such memory)
    if (x->tokens && ((x->token_bytes != 2 && x->token_bytes != 4 && x->token_bytes != 8) || (uintptr_t)x->tokens % x->token_bytes))
        return VL_ERR_INVALID_ARG;
    if (((uintptr_t)x->occupied | (uintptr_t)x->mask_rows) & 3) return VL_ERR_INVALID_ARG;
    if (x->mask_rows && !x->occupied) return VL_ERR_INVALID_ARG;
    if (x->occupied && !x->mask_rows && x->n_masks < x->n_rows) return VL_ERR_INVALID_ARG;
    if (!(x->scale >= 1e-6f && x->scale <= 1e6f)) return VL_ERR_INVALID_ARG;
    q->x = x->logits; q->n_rows = x->n_rows; q->stride = x->row_stride;
    q->V = x->n_vocab; q->W = (x->n_vocab + 31) / 32;
    q->tokens = x->tokens; q->token_bytes = x->token_bytes;
    q->occupied = x->occupied; q->n_masks = (uint32_t)(x->n_masks < (1ull << 31) ? x->n_masks : (1ull << 31)); q->mask_rows = x->mask_rows; q->widths = x->widths;
    q->scale = x->scale;
    return VL_OK;
}

extern "C" int vl_token_logprobs(int device, const vl_logits *x, float *d_logprob, float *d_entropy, float *d_row_stats, uint32_t top,
                                 int32_t *d_top_ids, float *d_top_logprobs, void *stream)
{
    LogitRows q;
    const int rc = vl_logit_rows(x, &q);
    if (rc != VL_OK) return rc;
    if (((uintptr_t)d_logprob | (uintptr_t)d_entropy | (uintptr_t)d_top_ids | (uintptr_t)d_top_logprobs) & 3) return VL_ERR_INVALID_ARG;
    if ((uintptr_t)d_row_stats & 7) return VL_ERR_INVALID_ARG;
    if (d_logprob && !q.tokens && q.n_rows) return VL_ERR_INVALID_ARG;
    if (top > VL_MAX_ALTERNATIVES || (top && q.n_rows && (!d_top_ids || !d_top_logprobs))) return VL_ERR_INVALID_ARG;
    if (q.n_rows == 0) return VL_OK;
    const DeviceScope scope(device);
    if (scope.error != cudaSuccess) return VL_ERR_CUDA;
    const ScoreOut o{d_logprob, d_entropy, d_row_stats, top, d_top_ids, d_top_logprobs};
    const auto launch = x->dtype == VL_F32 ? vl_scores_f32 : x->dtype == VL_F16 ? vl_scores_f16 : vl_scores_bf16;
    return launch(q, o, device, (cudaStream_t)stream) == cudaSuccess ? VL_OK : VL_ERR_CUDA;
}
