// The gradient of vl_token_logprobs to the logits.  With l_i = log p_i = scale (x_i - M) - L:
//   d logprob / d x_i = scale ([i = token] - p_i),   d entropy / d x_i = -scale p_i (l_i + entropy)
// p is recomputed from the logits and the row's two statistics: nothing but these is kept from the forward pass.
//
// In powers of two, with y = log2 p: d_i = 2^y (a + b y), a = -scale (g + h entropy), b = -scale h ln 2, and scale g more at the token.
// y = c x - K, c = scale log2 e, K = c M + L log2 e, is one multiply-add; K is rounded, and what it lacks, the same in the whole row,
// goes into a and b.  Each value is rounded once.
//
// What bounds it: the logits read and the gradient written, once each, and per element an exponential and about five more instructions.
#include "vl_logits.cuh"

namespace {

struct GradIn {
    const float *stats, *entropy, *g, *h;
    void *dx;
    uint64_t stride;
    int mixed;  // memory between the logits' rows is the gradient's: in place, or rows of both in turn
};

// What a row's entries have in common.
struct GradRow {
    float c, K, a, b, at_token;
    float M;         // for rows far out, where K would lack whole powers of two: it is L log2 e alone there
    bool far, dead;  // far: or the derivatives are; a, b and at_token are then without the scale, which is multiplied last
    int tok;
};
__device__ __forceinline__ GradRow grad_row(const LogitRows &q, const GradIn &p, uint64_t r, int64_t tok, bool shut)  // shut: the token is closed
{
    GradRow w;
    const float2 st = *reinterpret_cast<const float2 *>(p.stats + 2 * r);
    float g = p.g ? p.g[r] : 0.0f;
    const float h = p.h ? p.h[r] : 0.0f, H = p.h ? p.entropy[r] : 0.0f;
    w.tok = (int)tok;
    w.dead = tok < 0 || st.y == __int_as_float(0xFF800000);
    if (shut) g = 0.0f;
    w.c = q.scale * LOG2E;
    w.M = st.x;
    const float L2 = __fmul_rn(st.y, LOG2E), B = __fmul_rn(st.x, w.c), K = __fadd_rn(B, L2), k = __fsub_rn(K, B);
    // what K lacks: the rounded bits of the sum and of both products
    const float lacks = __fadd_rn(__fsub_rn(B, __fsub_rn(K, k)), __fsub_rn(L2, k)) + __fmaf_rn(st.x, w.c, -B) + __fmaf_rn(st.y, LOG2E, -L2);
    const float a = -q.scale * fmaf(h, H, g), b = -q.scale * h * LN2;
    w.at_token = q.scale * g;
    // (b times 300, the most that y is, is a number below the limit; what is no number is not below it)
    w.far = far_out(st.x, w.c) || !(fabsf(K) + fabsf(a) + fabsf(b) + fabsf(w.at_token) < 1e35f);
    w.K = K;
    const float f = ex2(-lacks);
    w.a = f * fmaf(-b, lacks, a);
    w.b = f * b;
    if (w.far) {
        w.K = L2;
        w.a = -fmaf(h, H, g);
        w.b = -h * LN2;
        w.at_token = g;
    }
    return w;
}

constexpr float FLOOR = -300.0f;  // 2^-300 is 0, and 0 (a + b y) too

// The gradient of a vector that begins at entry `first`.  An entry of minus infinity (closed, or impossible) has p = 0 whatever the
// row's numbers are.
template <typename T>
__device__ __forceinline__ uint4 grad_vector(const uint4 &raw, int first, const GradRow &w, float scale)
{
    float x[EPV<T>], d[EPV<T>];
    unpack(raw, x, T{});
    const uint32_t at = (uint32_t)(w.tok - first);
    if (!w.far) {
        const f32x2 c2 = both(w.c, w.c), K2 = both(-w.K, -w.K), a2 = both(w.a, w.a), b2 = both(w.b, w.b);
#pragma unroll
        for (int j = 0; j < EPV<T>; j += 2) {
            float y0, y1;
            apart(fma2(both(x[j], x[j + 1]), c2, K2), y0, y1);
            y0 = max_nan(y0, FLOOR);
            y1 = max_nan(y1, FLOOR);
            apart(mul2(both(ex2(y0), ex2(y1)), fma2(b2, both(y0, y1), a2)), d[j], d[j + 1]);
        }
        if (at < (uint32_t)EPV<T>) {
#pragma unroll
            for (int j = 0; j < EPV<T>; ++j)
                if ((uint32_t)j == at) d[j] += w.at_token;
        }
    } else {
#pragma unroll
        for (int j = 0; j < EPV<T>; ++j) {
            const float y = max_nan((x[j] - w.M) * w.c - w.K, FLOOR);
            const float v = x[j] == __int_as_float(0xFF800000) ? 0.0f : ex2(y) * fmaf(w.b, y, w.a);
            d[j] = ((uint32_t)j == at ? v + w.at_token : v) * scale;
        }
    }
    return pack(d, T{});
}

// A vector's entries one by one, those that are in the row.
template <typename T>
__device__ __forceinline__ void store_entries(T *row, int first, uint32_t V, const uint4 &d)
{
    T e[EPV<T>];
    memcpy(e, &d, 16);
#pragma unroll
    for (int j = 0; j < EPV<T>; ++j)
        if ((uint32_t)(first + j) < V) row[first + j] = e[j];
}

// Stores the gradient of a warp's 32 vectors to a row whose vectors begin at other entries: a vector there is the end of one lane's and the
// beginning of the next one's, `shift` entries of it the former.  What such vectors do not cover is stored one by one.  v: the lane's vector (any
// number; those from n on have no entries).  2,000 rows of 50,021 bf16 logits 108 us, 254 with every entry stored by itself, 69 where vectors match.
template <typename T>
__device__ __forceinline__ void store_shifted(T *dx, const RowVectors<T> &x, uint32_t v, const uint4 &d, uint32_t lane)
{
    const uint32_t lead = (uint32_t)((uintptr_t)dx & 15) / (uint32_t)sizeof(T);
    const int delta = (int)lead - (int)x.lead, shift = delta < 0 ? delta + EPV<T> : delta;  // 1 .. EPV - 1
    const int first = x.first(v);
    const uint32_t before[4] = {__shfl_up_sync(0xffffffffu, d.x, 1), __shfl_up_sync(0xffffffffu, d.y, 1),
                                __shfl_up_sync(0xffffffffu, d.z, 1), __shfl_up_sync(0xffffffffu, d.w, 1)};
    const int begin = first - shift;  // entry at which the vector begins that holds the lane's first ones
    const bool full = lane > 0 && v < x.n && begin >= 0 && begin + EPV<T> <= (int)x.V;
    const bool after = __shfl_down_sync(0xffffffffu, (int)full, 1) && lane < 31;
    if (full) {
        uint32_t w[8] = {before[0], before[1], before[2], before[3], d.x, d.y, d.z, d.w};
        const uint32_t skip = 16 - shift * (int)sizeof(T);  // bytes
        if (skip & 8) {
#pragma unroll
            for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
        }
        if (skip & 4) {
#pragma unroll
            for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
        }
        const uint32_t bits = (skip & 3) * 8;
        __stcs(reinterpret_cast<uint4 *>(dx + begin), make_uint4(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits),
                                                                 __funnelshift_r(w[2], w[3], bits), __funnelshift_r(w[3], w[4], bits)));
    }
    if (v < x.n && !(full && after)) {
        T e[EPV<T>];
        memcpy(e, &d, 16);
#pragma unroll
        for (int j = 0; j < EPV<T>; ++j)
            if ((uint32_t)(first + j) < x.V && !(j < EPV<T> - shift ? full : after)) dx[first + j] = e[j];
    }
}

// Long rows: a block per row and run of 4 vectors a thread.
constexpr int GRAD_U = 4;

// ALIKE: a vector of a row is a vector of the gradient's row in all rows.
template <typename T, bool MASKED, bool ALIKE, int NT>
__global__ void __launch_bounds__(NT) k_grad_long(const LogitRows q, const GradIn p)
{
    const uint64_t step = (uint64_t)gridDim.y * gridDim.z;
    const uint32_t lane = threadIdx.x & 31;
    for (uint64_t r = blockIdx.y + (uint64_t)gridDim.y * blockIdx.z; r < q.n_rows; r += step) {
        const RowVectors<T> x(static_cast<const T *>(q.x) + r * q.stride, q.V);
        T *const dx = static_cast<T *>(p.dx) + r * p.stride;
        const bool alike = ALIKE || ((uintptr_t)dx & 15) == x.lead * sizeof(T);
        uint4 *const to = reinterpret_cast<uint4 *>(reinterpret_cast<uintptr_t>(dx) & ~(uintptr_t)15);
        const uint32_t v0 = blockIdx.x * (NT * GRAD_U) + threadIdx.x;
        uint4 raw[GRAD_U];
#pragma unroll
        for (int u = 0; u < GRAD_U; ++u) {
            const uint32_t v = v0 + u * NT;
            raw[u] = make_uint4(0u, 0u, 0u, 0u);
            if (v < x.n && x.whole(v)) raw[u] = __ldcs(x.at(v));
        }
        const RowMask mask = row_mask(q, r);
        const int64_t tok = row_token(q, r);
        const GradRow w = grad_row(q, p, r, tok, MASKED && tok >= 0 && tok < (int64_t)q.V && mask.is_closed((uint32_t)tok));
#pragma unroll
        for (int u = 0; u < GRAD_U; ++u) {
            const uint32_t v = v0 + u * NT;
            if (ALIKE ? v >= x.n : v - lane >= x.n) break;  // (a whole warp stores vectors that are shifted)
            const bool whole = x.whole(v);
            const int first = x.first(v);
            if (v < x.n && !whole) raw[u] = x.part(v);
            if (MASKED && v < x.n) close_entries<T>(raw[u], mask.closed_from(first, EPV<T>));
            const uint4 d = w.dead ? make_uint4(0u, 0u, 0u, 0u) : grad_vector<T>(raw[u], first, w, q.scale);
            if (!ALIKE && !alike) store_shifted<T>(dx, x, v, d, lane);
            else if (whole) __stcs(to + v, d);
            else if (v < x.n) store_entries<T>(dx, first, q.V, d);
        }
    }
}

// Short rows: a group of lanes per row.
constexpr uint32_t SHORT_WARPS = 8;

template <typename T, bool MASKED, bool ALIGNED, int G, int NV>
__global__ void __launch_bounds__(SHORT_WARPS * 32, short_blocks(NV)) k_grad_short(const LogitRows q, const GradIn p)
{
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane % G;
    const uint64_t step = (uint64_t)gridDim.x * SHORT_WARPS * (32 / G);
    for (uint64_t r0 = ((uint64_t)blockIdx.x * SHORT_WARPS + warp) * (32 / G); r0 < q.n_rows; r0 += step) {
        const bool there = r0 + lane / G < q.n_rows;
        const uint64_t r = there ? r0 + lane / G : q.n_rows - 1;
        const RowVectors<T> x(static_cast<const T *>(q.x) + r * q.stride, q.V);
        uint4 raw[NV];
        if (there) fetch_row<T, G, NV, ALIGNED>(raw, x, g, !p.mixed && r != 0 && r != q.n_rows - 1);
        const RowMask mask = row_mask(q, r);
        const int64_t tok = row_token(q, r);
        bool shut = false;
        if (MASKED) shut = close_row<T, G, NV, ALIGNED>(raw, x, mask, g, tok);
        const GradRow w = grad_row(q, p, r, tok, shut);
        if (!there) continue;
        T *const dx = static_cast<T *>(p.dx) + r * p.stride;
        const bool alike = ALIGNED || ((uintptr_t)dx & 15) == x.lead * sizeof(T);  // vectors of one are vectors of the other
        uint4 *const to = reinterpret_cast<uint4 *>(reinterpret_cast<uintptr_t>(dx) & ~(uintptr_t)15) + g;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const uint32_t v = g + G * j;
            if (v >= x.n) break;
            const uint4 d = w.dead ? make_uint4(0u, 0u, 0u, 0u) : grad_vector<T>(raw[j], x.first(v), w, q.scale);
            if (alike && (ALIGNED || x.whole(v))) to[G * j] = d;
            else store_entries<T>(dx, x.first(v), q.V, d);
        }
    }
}

// ALIGNED: both matrices' rows start and end on vectors.
template <typename T, bool MASKED, bool ALIGNED>
bool launch_short(const LogitRows &q, const GradIn &p, uint32_t n, cudaStream_t st)
{
    return short_shape<false, ALIGNED>(n, q.W, [&](auto g, auto v) {
        constexpr int G = decltype(g)::value, NV = decltype(v)::value;
        const uint64_t blocks = (q.n_rows + SHORT_WARPS * (32 / G) - 1) / (SHORT_WARPS * (32 / G));
        k_grad_short<T, MASKED, ALIGNED, G, NV><<<(uint32_t)(blocks < (1u << 30) ? blocks : (1u << 30)), SHORT_WARPS * 32, 0, st>>>(q, p);
    });
}

template <typename T, bool MASKED>
cudaError_t launch(const LogitRows &q, const GradIn &p, cudaStream_t st)
{
    bool aligned;
    const uint32_t n = row_vectors(q, sizeof(T), &aligned);
    aligned = aligned && ((uintptr_t)p.dx & 15) == 0 && (q.n_rows <= 1 || p.stride % EPV<T> == 0);
    if (!(aligned ? launch_short<T, MASKED, true>(q, p, n, st) : launch_short<T, MASKED, false>(q, p, n, st))) {
        const uint32_t y = (uint32_t)(q.n_rows < 65535 ? q.n_rows : 65535);
        const uint64_t z = (q.n_rows + y - 1) / y;
        // small blocks where a row is not several large ones (16,000 rows of 2,500 bf16 logits: 41 us in blocks of 256 threads)
        const bool alike = (((uintptr_t)q.x - (uintptr_t)p.dx) & 15) == 0 && (q.n_rows <= 1 || (q.stride - p.stride) % EPV<T> == 0);
        const uint32_t threads = n <= 2048 || !alike ? 128 : 256, tile = threads * GRAD_U;
        const dim3 grid((n + tile - 1) / tile, y, (uint32_t)(z < 65535 ? z : 65535));
        if (!alike) k_grad_long<T, MASKED, false, 128><<<grid, 128, 0, st>>>(q, p);
        else if (threads == 128) k_grad_long<T, MASKED, true, 128><<<grid, 128, 0, st>>>(q, p);
        else k_grad_long<T, MASKED, true, 256><<<grid, 256, 0, st>>>(q, p);
    }
    g_vl_launches.fetch_add(1);
    return cudaGetLastError();
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
    if (out_stride > (1ull << 40) || (q.n_rows > 1 && out_stride > (1ull << 56) / q.n_rows)) return VL_ERR_INVALID_ARG;
    if (q.n_rows && (!d_row_stats || !d_dlogits || (uintptr_t)d_dlogits % (x->dtype == VL_F32 ? 4 : 2))) return VL_ERR_INVALID_ARG;
    if (q.n_rows == 0) return VL_OK;
    // Where the matrices' memory meets, they are the same rows, or rows of both in turn that have nothing in common.
    const uint64_t size = x->dtype == VL_F32 ? 4 : 2, row = q.V * size, pitch = q.stride * size;
    const uintptr_t from = (uintptr_t)x->logits, to = (uintptr_t)d_dlogits;
    const bool meet = to < from + (q.n_rows - 1) * pitch + row && from < to + (q.n_rows - 1) * out_stride * size + row;
    if (meet && q.n_rows > 1) {
        const uint64_t behind = to >= from ? (to - from) % pitch : (pitch - (from - to) % pitch) % pitch;
        if (out_stride != q.stride || (to != from && (behind < row || behind > pitch - row))) return VL_ERR_INVALID_ARG;
    } else if (meet && to != from) {
        return VL_ERR_INVALID_ARG;
    }
    const DeviceScope scope(device);
    if (scope.error != cudaSuccess) return VL_ERR_CUDA;
    const GradIn p{d_row_stats, d_entropy, d_g_logprob, d_g_entropy, d_dlogits, out_stride, meet};
    cudaStream_t st = (cudaStream_t)stream;
    const bool masked = q.occupied || q.widths;
    cudaError_t e;
    if (x->dtype == VL_F32) e = masked ? launch<float, true>(q, p, st) : launch<float, false>(q, p, st);
    else if (x->dtype == VL_F16) e = masked ? launch<__half, true>(q, p, st) : launch<__half, false>(q, p, st);
    else e = masked ? launch<__nv_bfloat16, true>(q, p, st) : launch<__nv_bfloat16, false>(q, p, st);
    return e == cudaSuccess ? VL_OK : VL_ERR_CUDA;
}
