// The gradient of vl_token_logprobs to the logits.  With l_i = log p_i = scale (x_i - M) - L:
//   d logprob / d x_i = scale ([i = token] - p_i),   d entropy / d x_i = -scale p_i (l_i + entropy)
// p is recomputed from the logits and the row's two statistics: nothing but these is kept from the forward pass.
#include "vl_logits.cuh"

namespace {

constexpr uint32_t GRAD_THREADS = 256;

struct GradIn {
    const float *stats, *entropy, *g, *h;
    void *dx;
    uint64_t stride;
};

template <typename T>
__global__ void __launch_bounds__(GRAD_THREADS) k_score_grad(const LogitRows q, const GradIn p)
{
    const float inf = __int_as_float(0x7f800000);
    for (uint64_t r = blockIdx.x; r < q.n_rows; r += gridDim.x) {
        const int64_t tok = row_token(q, r);
        const float M = p.stats[2 * r], L = p.stats[2 * r + 1];
        const T *x = static_cast<const T *>(q.x) + r * q.stride;
        T *dx = static_cast<T *>(p.dx) + r * p.stride;
        const RowMask mask = row_mask(q, r);
        const bool masked = mask.any(), dead = tok < 0 || L == -inf;
        const float H = p.h && !dead ? p.entropy[r] : 0.0f, h = p.h && !dead ? p.h[r] : 0.0f;
        const float g = !p.g || dead || (masked && mask.is_closed((uint32_t)tok)) ? 0.0f : p.g[r];
        for (uint32_t i = threadIdx.x; i < q.V; i += GRAD_THREADS) {
            float d = 0.0f;
            if (!dead && !(masked && mask.is_closed(i))) {
                const float l = (to_f32(x[i]) - M) * q.scale - L;
                const float e = expf(l);
                d = e == 0.0f ? 0.0f : -e * (g + h * (l + H));
                if ((int64_t)i == tok) d += g;
                d *= q.scale;
            }
            from_f32(dx[i], d);
        }
    }
}

}  // namespace

extern "C" int vl_token_logprobs_backward(int device, const vl_logits *x, const float *d_row_stats, const float *d_entropy,
                                          const float *d_g_logprob, const float *d_g_entropy, void *d_dlogits, uint64_t out_stride,
                                          void *stream)
{
    LogitRows q;
    const int rc = vl_logit_rows(x, &q);
    if (rc != VL_OK) return rc;
    if (((uintptr_t)d_entropy | (uintptr_t)d_g_logprob | (uintptr_t)d_g_entropy) & 3) return VL_ERR_INVALID_ARG;
    if ((uintptr_t)d_row_stats & 7) return VL_ERR_INVALID_ARG;
    if (d_g_entropy && !d_entropy) return VL_ERR_INVALID_ARG;
    if (d_g_logprob && !q.tokens) return VL_ERR_INVALID_ARG;
    if (q.n_rows > 1 && out_stride < q.V) return VL_ERR_INVALID_ARG;
    if (out_stride > (1ull << 40)) return VL_ERR_INVALID_ARG;
    if (q.n_rows && (!d_row_stats || !d_dlogits || (uintptr_t)d_dlogits % (x->dtype == VL_F32 ? 4 : 2))) return VL_ERR_INVALID_ARG;
    if (d_dlogits == x->logits && q.n_rows > 1 && out_stride != q.stride) return VL_ERR_INVALID_ARG;
    if (q.n_rows == 0) return VL_OK;
    const DeviceScope scope(device);
    if (scope.error != cudaSuccess) return VL_ERR_CUDA;
    const GradIn p{d_row_stats, d_entropy, d_g_logprob, d_g_entropy, d_dlogits, out_stride};
    const uint32_t blocks = (uint32_t)(q.n_rows < 0x7FFFFFFFull ? q.n_rows : 0x7FFFFFFFull);
    cudaStream_t st = (cudaStream_t)stream;
    if (x->dtype == VL_F32) k_score_grad<float><<<blocks, GRAD_THREADS, 0, st>>>(q, p);
    else if (x->dtype == VL_F16) k_score_grad<__half><<<blocks, GRAD_THREADS, 0, st>>>(q, p);
    else k_score_grad<__nv_bfloat16><<<blocks, GRAD_THREADS, 0, st>>>(q, p);
    g_vl_launches.fetch_add(1);
    return cudaGetLastError() == cudaSuccess ? VL_OK : VL_ERR_CUDA;
}
