// Log probabilities of given tokens, entropy and best alternatives of rows of logits, and their gradient: how likely the model
// behind the candidates found them (the autoregressive factorisation of Section 3.1), under the masks of vl_occupied_masks where
// it decodes around occupied registers (Section 4.5).
//
// With z = scale x over the open entries, M = max x, e_i = exp(scale (x_i - M)), L = ln sum e_i:
//   log p_i = scale (x_i - M) - L,   entropy = L - sum e_i scale (x_i - M) / sum e_i
// Both terms of the entropy are non-negative, so nothing cancels; the sums are held in 32 bits.
#include "vl_logits.cuh"

namespace {

constexpr uint32_t LP_THREADS = 256;

__device__ __forceinline__ float warp_max(float v)
{
#pragma unroll
    for (int d = 16; d; d >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, d));
    return v;
}
__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}

// A value and its place as one key: larger values first, lower places first among equals (zeros of both signs are equal).
__device__ __forceinline__ unsigned long long rank_key(float x, uint32_t i)
{
    const uint32_t b = __float_as_uint(x + 0.0f);
    const uint32_t order = (b & 0x80000000u) ? ~b : (b | 0x80000000u);
    return ((unsigned long long)order << 32) | (0xFFFFFFFFu - i);
}

struct ScoreOut {
    float *logprob, *entropy, *stats;
    uint32_t top;
    int32_t *ids;
    float *lps;
};

__device__ __forceinline__ void empty_row(const ScoreOut &o, uint64_t r, bool left_out, uint32_t tid, uint32_t nt)
{
    const float inf = __int_as_float(0x7f800000);
    if (tid == 0) {
        if (o.logprob) o.logprob[r] = left_out ? 0.0f : -inf;
        if (o.entropy) o.entropy[r] = 0.0f;
        if (o.stats) o.stats[2 * r] = o.stats[2 * r + 1] = left_out ? 0.0f : -inf;
    }
    for (uint32_t j = tid; j < o.top; j += nt) { o.ids[r * o.top + j] = -1; o.lps[r * o.top + j] = -inf; }
}

// One block per row: the maximum, the sums, then the alternatives one by one, each a pass over the row.
template <typename T>
__global__ void __launch_bounds__(LP_THREADS) k_score(const LogitRows q, const ScoreOut o)
{
    __shared__ float s_a[8], s_b[8];
    __shared__ unsigned long long s_k[8];
    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const float inf = __int_as_float(0x7f800000);
    for (uint64_t r = blockIdx.x; r < q.n_rows; r += gridDim.x) {
        const int64_t tok = row_token(q, r);
        if (tok < 0) { empty_row(o, r, true, tid, LP_THREADS); continue; }
        const T *x = static_cast<const T *>(q.x) + r * q.stride;
        const RowMask mask = row_mask(q, r);
        const bool masked = mask.any();
        float m = -inf;
        bool nan = false;
        for (uint32_t i = tid; i < q.V; i += LP_THREADS) {
            if (masked && mask.is_closed(i)) continue;
            const float v = to_f32(x[i]);
            nan = nan || v != v;
            m = fmaxf(m, v);
        }
        m = warp_max(m);
        __syncthreads();
        if (lane == 0) s_a[warp] = m;
        nan = __syncthreads_or(nan);
        m = s_a[0];
        for (int w = 1; w < 8; ++w) m = fmaxf(m, s_a[w]);
        if (m == -inf && !nan) { empty_row(o, r, false, tid, LP_THREADS); continue; }
        float s = 0.0f, t = 0.0f;
        for (uint32_t i = tid; i < q.V; i += LP_THREADS) {
            if (masked && mask.is_closed(i)) continue;
            const float d = (to_f32(x[i]) - m) * q.scale;
            const float e = expf(d);
            s += e;
            if (e != 0.0f) t += e * d;
        }
        s = warp_sum(s);
        t = warp_sum(t);
        __syncthreads();
        if (lane == 0) { s_a[warp] = s; s_b[warp] = t; }
        __syncthreads();
        s = t = 0.0f;
        for (int w = 0; w < 8; ++w) { s += s_a[w]; t += s_b[w]; }
        const float L = logf(s);
        if (tid == 0) {
            if (o.logprob)
                o.logprob[r] = masked && mask.is_closed((uint32_t)tok) ? -inf : (to_f32(x[tok]) - m) * q.scale - L;
            if (o.entropy) o.entropy[r] = L - t / s;
            if (o.stats) { o.stats[2 * r] = m; o.stats[2 * r + 1] = L; }
        }
        unsigned long long last = ~0ull;
        for (uint32_t j = 0; j < o.top; ++j) {
            unsigned long long best = 0;
            for (uint32_t i = tid; i < q.V; i += LP_THREADS) {
                if (masked && mask.is_closed(i)) continue;
                const float v = to_f32(x[i]);
                if (!(v > -inf)) continue;
                const unsigned long long k = rank_key(v, i);
                if (k < last && k > best) best = k;
            }
            for (int d = 16; d; d >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, d));
            __syncthreads();
            if (lane == 0) s_k[warp] = best;
            __syncthreads();
            for (int w = 0; w < 8; ++w) best = max(best, s_k[w]);
            if (tid == 0) {
                const uint32_t i = 0xFFFFFFFFu - (uint32_t)best;
                o.ids[r * o.top + j] = best ? (int32_t)i : -1;
                o.lps[r * o.top + j] = best ? (to_f32(x[i]) - m) * q.scale - L : -inf;
            }
            last = best;
        }
    }
}

struct GradIn {
    const float *stats, *entropy, *g, *h;
    void *dx;
    uint64_t stride;
};

// With l_i = log p_i: d logprob / d x_i = scale ([i = token] - p_i), d entropy / d x_i = -scale p_i (l_i + entropy).
template <typename T>
__global__ void __launch_bounds__(LP_THREADS) k_score_grad(const LogitRows q, const GradIn p)
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
        for (uint32_t i = threadIdx.x; i < q.V; i += LP_THREADS) {
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

template <typename F>
int by_type(int dtype, F &&f)
{
    switch (dtype) {
    case VL_F32: return f(float{});
    case VL_F16: return f(__half{});
    default: return f(__nv_bfloat16{});
    }
}

uint32_t row_blocks(uint64_t rows) { return (uint32_t)(rows < 0x7FFFFFFFull ? rows : 0x7FFFFFFFull); }

}  // namespace

int vl_logit_rows(const vl_logits *x, LogitRows *q)
{
    if (!x || x->n_vocab == 0 || x->n_vocab > VL_MAX_VOCAB) return VL_ERR_INVALID_ARG;
    if (x->dtype != VL_F32 && x->dtype != VL_F16 && x->dtype != VL_BF16) return VL_ERR_INVALID_ARG;
    const uint32_t size = x->dtype == VL_F32 ? 4 : 2;
    if (x->n_rows > 1 && x->row_stride < x->n_vocab) return VL_ERR_INVALID_ARG;
    if (x->n_rows && (!x->logits || (uintptr_t)x->logits % size)) return VL_ERR_INVALID_ARG;
    if (x->n_rows > (1ull << 40) || x->row_stride > (1ull << 40)) return VL_ERR_INVALID_ARG;
    if (x->tokens && ((x->token_bytes != 2 && x->token_bytes != 4 && x->token_bytes != 8) || (uintptr_t)x->tokens % x->token_bytes))
        return VL_ERR_INVALID_ARG;
    if (((uintptr_t)x->occupied | (uintptr_t)x->mask_rows) & 3) return VL_ERR_INVALID_ARG;
    if (x->mask_rows && !x->occupied) return VL_ERR_INVALID_ARG;
    if (x->occupied && !x->mask_rows && x->n_masks < x->n_rows) return VL_ERR_INVALID_ARG;
    if (!(x->scale > 0.0f) || x->scale > 3.0e38f) return VL_ERR_INVALID_ARG;
    q->x = x->logits; q->n_rows = x->n_rows; q->stride = x->row_stride;
    q->V = x->n_vocab; q->W = (x->n_vocab + 31) / 32;
    q->tokens = x->tokens; q->token_bytes = x->token_bytes;
    q->occupied = x->occupied; q->n_masks = x->n_masks; q->mask_rows = x->mask_rows; q->widths = x->widths;
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
    return by_type(x->dtype, [&](auto type) {
        k_score<decltype(type)><<<row_blocks(q.n_rows), LP_THREADS, 0, (cudaStream_t)stream>>>(q, o);
        g_vl_launches.fetch_add(1);
        return cudaGetLastError() == cudaSuccess ? VL_OK : VL_ERR_CUDA;
    });
}

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
    return by_type(x->dtype, [&](auto type) {
        k_score_grad<decltype(type)><<<row_blocks(q.n_rows), LP_THREADS, 0, (cudaStream_t)stream>>>(q, p);
        g_vl_launches.fetch_add(1);
        return cudaGetLastError() == cudaSuccess ? VL_OK : VL_ERR_CUDA;
    });
}
