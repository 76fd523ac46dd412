// The loss that makes the verifier's verdicts a training signal (Section 6): rewards of the sampled candidates, advantages within
// the samples of each program, the clipped objective over their tokens, and its derivative to every token's log probability.
//
//   reward = [pass] - pair_cost conflict_pairs - bank_cost bank_conflicts,   A = reward - mean  (/ (std + eps))
//   d = logprob - old, rho = exp d,  token loss = -min(rho A, clip(rho) A) + kl (exp q - q - 1),  q = ref - logprob
// The loss rests on small differences (A sums to nothing within a program, rho is near 1): rewards, advantages and weights are worked out
// in 64 bits, rho - 1 comes from a series where it is small, and on which side of a border of the clip a token lies is decided as in exact
// arithmetic.  A token's difference, exponential and derivative are in 32 bits, the type they are given and wanted in; so are sums of up to four
// tokens' terms, less 1 where these are near 1, and all sums beyond that are in 64.
//
// Three kernels: k_advantages, a cluster or a block per program, leaves each candidate's weight and weighted advantage; k_policy_tokens
// streams the tokens, which is what bounds it (12 to 16 bytes a token), each warp a run of them, finding candidates by their
// offsets; k_policy_sum adds the blocks' sums in order.  Small losses take one kernel, k_policy_small.
#include <cooperative_groups.h>
#include <math.h>

#include "vl_logits.cuh"

namespace {

namespace cg = cooperative_groups;

constexpr uint32_t PL_GROUPS = 96;    // programs per launch (their pointers travel as kernel arguments)
constexpr uint32_t PL_THREADS = 256, PL_WARPS = PL_THREADS / 32;
constexpr uint32_t PL_STEP = 128;     // tokens of a warp at a time, four to a lane
constexpr uint32_t PL_MAX_BLOCKS = 2048;

struct GroupParams {
    const uint4 *out[PL_GROUPS];
    uint64_t K[PL_GROUPS], first[PL_GROUPS];  // first: candidate number of its first row
    double pair_cost, bank_cost, eps;
    const int64_t *off;
    uint64_t N, T;
    double2 *weights;  // [N] weight of a token of the candidate, and times the advantage
    float *advantage;
    int normalise, per_token;
};

__device__ __forceinline__ double reward_of(const uint4 &v, double pair_cost, double bank_cost)
{
    return ((v.x & VL_PASS) ? 1.0 : 0.0) - pair_cost * (double)v.z - bank_cost * (double)v.w;
}

// Sum over the block, the same in every thread and in the same order on every run.
__device__ __forceinline__ double block_sum(double v, double *s)
{
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.0;
    for (uint32_t w = 0; w < blockDim.x / 32; ++w) v += s[w];
    return v;
}

__device__ __forceinline__ int64_t inside(int64_t t, uint64_t T) { return min(max(t, (int64_t)0), (int64_t)T); }

// The advantages and weights of program j, by `step` threads of which this one is thread k0; total(v, at) sums over them, at = 0 the first
// time, 1 the second.  A thread's first KEEP rewards stay in registers.
template <uint32_t KEEP, typename F>
__device__ __forceinline__ void advantages(const GroupParams &q, uint32_t j, uint64_t step, uint64_t k0, double2 *weights, float *advantage, F &&total)
{
    const uint64_t K = q.K[j];
    const uint4 *out = q.out[j];
    // taken from the first one's: equal rewards leave exactly nothing, which a division by their deviation would blow up
    const double base = reward_of(__ldg(out), q.pair_cost, q.bank_cost);
    double keep[KEEP];
#pragma unroll
    for (uint32_t i = 0; i < KEEP; ++i)
        keep[i] = k0 + i * step < K ? reward_of(__ldg(out + k0 + i * step), q.pair_cost, q.bank_cost) - base : 0.0;
    auto each = [&](auto &&f) {
#pragma unroll
        for (uint32_t i = 0; i < KEEP; ++i)
            if (k0 + i * step < K) f(k0 + i * step, keep[i]);
        for (uint64_t k = k0 + KEEP * step; k < K; k += step) f(k, reward_of(__ldg(out + k), q.pair_cost, q.bank_cost) - base);
    };
    double sum = 0.0;
    each([&](uint64_t, double c) { sum += c; });
    const double mean = total(sum, 0u) / (double)K;
    double by = 1.0;
    if (q.normalise) {
        double var = 0.0;
        each([&](uint64_t, double c) { var += (c - mean) * (c - mean); });
        by = 1.0 / (sqrt(total(var, 1u) / (double)K) + q.eps);
    }
    const double per_token = 1.0 / (double)max(inside(q.off[q.N], q.T) - inside(q.off[0], q.T), (int64_t)1);
    each([&](uint64_t k, double c) {
        const double a = (c - mean) * by;
        const uint64_t at = q.first[j] + k;
        const double w = q.per_token ? per_token : 1.0 / ((double)q.N * (double)max(q.off[at + 1] - q.off[at], (int64_t)1));
        weights[at] = make_double2(w, w * a);
        if (advantage) advantage[at] = (float)a;
    });
}

// A block or a cluster of eight per program.
constexpr uint32_t ADV_THREADS = 1024;
__global__ void __launch_bounds__(ADV_THREADS) k_advantages(const __grid_constant__ GroupParams q)
{
    __shared__ double s[ADV_THREADS / 32], s_all[2][8];
    cg::cluster_group cluster = cg::this_cluster();
    const uint32_t parts = cluster.num_blocks(), part = cluster.block_rank();
    pdl_go();
    pdl_wait();
    auto total = [&](double v, uint32_t at) {  // over the cluster, in the blocks' order
        v = block_sum(v, s);
        if (parts == 1) return v;
        if (threadIdx.x < parts) *cluster.map_shared_rank(&s_all[at][part], threadIdx.x) = v;
        cluster.sync();
        v = 0.0;
        for (uint32_t b = 0; b < parts; ++b) v += s_all[at][b];
        return v;
    };
    if (parts > 1) cluster.sync();  // (all of them run)
    advantages<8>(q, blockIdx.x / parts, (uint64_t)parts * blockDim.x, (uint64_t)part * blockDim.x + threadIdx.x, q.weights, q.advantage, total);
}

struct TokenParams {
    const double2 *weights;
    const int64_t *off;
    uint64_t N, T, per_warp;  // per_warp: tokens of a warp, a multiple of PL_STEP
    const float *lp, *old, *ref;
    float hi, hi_rest, lo, lo_rest;  // the clip's borders as logarithms, in two parts
    double at_lo, at_hi, kl;
    int vectors;                     // every array on 16 bytes
    float *g;
    double *part;
};

// First of off[0 .. n) that is above t (n if none).  Every lane of the warp calls it with the same t: 31 places at a time.
__device__ __forceinline__ uint64_t first_above(const int64_t *off, uint64_t n, int64_t t, uint32_t lane)
{
    uint64_t a = 0, b = n;  // off[a - 1] <= t < off[b]
    while (a < b) {
        const uint64_t step = (b - a + 31) / 32;  // places a + step - 1, a + 2 step - 1, ... below b
        const uint64_t at = a + (lane + 1) * step - 1;
        const uint32_t above = __ballot_sync(0xffffffffu, at >= b || off[at] > t);
        const uint32_t f = above ? __ffs(above) - 1 : 32;
        const uint64_t from = a + f * step;
        b = min(b, from + step - 1);
        a = min(from, b);
    }
    return a;
}

// No exponential is above 2^122 = 5e36, so that nothing times it, and four of them together, are numbers.
constexpr float EXP_MOST = 122.0f;

// exp d, as such where |d| >= 0.35, or less 1 near 0, where the rest would have lost the digits of the difference; and exp d - 1 - d.
// Near 0 from the exponential series (its terms from the ninth on are below 2^-26 of the first), elsewhere from the exponential
// itself: within (5 + 2 |d|) u of its value, u = 2^-24 (its argument is rounded twice), and of 1 more in the difference.
struct Exp {
    float value, less;
    bool near;  // value is exp d - 1
    __device__ __forceinline__ float minus_1() const { return near ? value : value - 1.0f; }
};
__device__ __forceinline__ Exp exp_of(float d)
{
    float p = 1.0f / 40320.0f;
    p = fmaf(p, d, 1.0f / 5040.0f);
    p = fmaf(p, d, 1.0f / 720.0f);
    p = fmaf(p, d, 1.0f / 120.0f);
    p = fmaf(p, d, 1.0f / 24.0f);
    p = fmaf(p, d, 1.0f / 6.0f);
    p = fmaf(p, d, 0.5f);
    const float less = d * d * p, far = ex2(min_nan(d * LOG2E, EXP_MOST));
    const bool near = fabsf(d) < 0.35f;
    return {near ? d + less : far, near ? less : (far - 1.0f) - d, near};
}

// What tokens add to the loss of their candidate, of weight w and w times advantage wA: -wA (in + n_in + n_cut border) + kl w sum.
struct Part {
    float in, kl;  // sums over the tokens that are not clipped, of rho - 1 where it is near 1 (n_in of them) and of rho; and of exp q - q - 1
    int n_in, n_cut;
};
struct Weight {
    double w, wA;
    float wA32, wk32;  // and kl w
    bool up;           // a positive advantage: clipped above
};
__device__ __forceinline__ Weight weight_of(const TokenParams &q, uint64_t k)  // of candidate k - 1, or of none
{
    const double2 w = k > 0 && k <= q.N ? q.weights[k - 1] : make_double2(0.0, 0.0);
    return {w.x, w.y, (float)w.y, (float)(q.kl * w.x), w.y > 0.0};
}
template <bool REF>
__device__ __forceinline__ float token(const TokenParams &q, float lp, float old, float ref, const Weight &w, bool owned, Part &p)
{
    const bool counts = owned && fminf(fminf(lp, old), ref) != __int_as_float(0xFF800000);
    const float d = __fsub_rn(lp, old), border = w.up ? q.hi : q.lo;
    bool cut = w.up ? d > border : d < border;
    if (d == border) {  // what d lost to rounding decides (it is a 32-bit number, and so found exactly)
        const float back = __fsub_rn(d, lp), lost = __fsub_rn(__fsub_rn(lp, __fsub_rn(d, back)), __fadd_rn(old, back));
        cut = w.up ? lost > q.hi_rest : lost < q.lo_rest;
    }
    const Exp r = exp_of(d);
    const bool in = counts && !cut;
    p.in += in ? r.value : 0.0f;
    p.n_in += in && r.near;
    p.n_cut += counts && cut;
    float g = in ? -fmaf(w.wA32, r.value, r.near ? w.wA32 : 0.0f) : 0.0f;  // (a small rho keeps its digits)
    if (REF) {
        const Exp k = exp_of(__fsub_rn(ref, lp));
        p.kl += counts ? k.less : 0.0f;
        g = counts ? fmaf(-w.wk32, k.minus_1(), g) : 0.0f;
    }
    return g;
}
template <bool REF>
__device__ __forceinline__ double part_loss(const TokenParams &q, const Part &p, const Weight &w)
{
    const double in = (double)p.in + (double)p.n_in + (double)p.n_cut * (w.up ? q.at_hi : q.at_lo);
    return REF ? fma(q.kl * w.w, (double)p.kl, -w.wA * in) : -w.wA * in;
}

// A warp's run of tokens, `len` of them from `begin` on: their derivatives; the lanes' parts of the loss.
template <bool REF>
__device__ __forceinline__ double run_tokens(const TokenParams &q, uint64_t begin, uint32_t len, uint32_t lane)
{
    const float *const lp = q.lp + begin, *const old = (q.old ? q.old : q.lp) + begin, *const ref = (REF ? q.ref : q.lp) + begin;
    constexpr int FAR = 0x7FFFFFFF;
    auto offset = [&](uint64_t k) -> int {
        return k <= q.N ? (int)min(max(q.off[k] - (int64_t)begin, (int64_t)0), (int64_t)FAR) : FAR;
    };
    float4 nx, ny, nz;
    auto fetch = [&](uint32_t t) {
        if (q.vectors && t + 4 <= len) {
            nx = __ldcs(reinterpret_cast<const float4 *>(lp + t));
            ny = __ldcs(reinterpret_cast<const float4 *>(old + t));
            if (REF) nz = __ldcs(reinterpret_cast<const float4 *>(ref + t));
            else nz = nx;
        } else {
            auto one = [&](const float *a, uint32_t j) { return t + j < len ? a[t + j] : 0.0f; };
            nx = make_float4(one(lp, 0), one(lp, 1), one(lp, 2), one(lp, 3));
            ny = make_float4(one(old, 0), one(old, 1), one(old, 2), one(old, 3));
            nz = make_float4(one(ref, 0), one(ref, 1), one(ref, 2), one(ref, 3));
        }
    };
    double loss = 0.0;
    uint64_t k0 = 0;  // first offset above the step's first token
    if (len) {
        fetch(lane * 4);
        k0 = first_above(q.off, q.N + 1, (int64_t)begin, lane);
    }
    pdl_wait();       // for the weights
    int end0 = offset(k0);
    Weight w0 = weight_of(q, k0);
    bool owned0 = k0 > 0 && k0 <= q.N;
    for (uint32_t t0 = 0; t0 < len; t0 += PL_STEP) {
        const uint32_t t = t0 + lane * 4;
        const float x[4] = {nx.x, nx.y, nx.z, nx.w}, y[4] = {ny.x, ny.y, ny.z, ny.w}, z[4] = {nz.x, nz.y, nz.z, nz.w};
        if (t0 + PL_STEP < len) fetch(t + PL_STEP);
        float g[4];
        if (end0 >= (int)min(t0 + PL_STEP, len)) {  // one candidate's tokens, or nobody's
            Part p{0.0f, 0.0f, 0, 0};
#pragma unroll
            for (int j = 0; j < 4; ++j) g[j] = token<REF>(q, x[j], y[j], z[j], w0, owned0 && t + j < len, p);
            loss += part_loss<REF>(q, p, w0);
        } else {
            // the next 32 offsets; each lane walks to its tokens' from the last one at or below the first of them
            const int near = offset(k0 + lane);
            const bool many = __shfl_sync(0xffffffffu, near, 31) <= (int)(t0 + PL_STEP);  // they may end before the step does
            uint32_t n = 0;
#pragma unroll
            for (uint32_t d = 16; d; d /= 2)
                if (__shfl_sync(0xffffffffu, near, n + d - 1) <= (int)t) n += d;
            uint64_t k = k0 + n;
            Weight w = weight_of(q, k);
            Part p{0.0f, 0.0f, 0, 0};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint64_t to;
                if (many) {
                    uint64_t a = k0, b = q.N + 1;
                    while (a < b) {
                        const uint64_t mid = (a + b) >> 1;
                        if (offset(mid) <= (int)(t + j)) a = mid + 1; else b = mid;
                    }
                    to = a;
                } else {
                    for (;;) {
                        const int next = __shfl_sync(0xffffffffu, near, n);
                        const bool on = n < 31 && next <= (int)(t + j);
                        if (!__any_sync(0xffffffffu, on)) break;
                        n += on;
                    }
                    to = k0 + n;
                }
                if (to != k) {  // another candidate's
                    loss += part_loss<REF>(q, p, w);
                    p = Part{0.0f, 0.0f, 0, 0};
                    k = to;
                    w = weight_of(q, k);
                }
                g[j] = token<REF>(q, x[j], y[j], z[j], w, k > 0 && k <= q.N && t + j < len, p);
            }
            loss += part_loss<REF>(q, p, w);
            // first offset above the next step's first token
            if (many) k0 = first_above(q.off, q.N + 1, (int64_t)(begin + t0 + PL_STEP), lane);
            else k0 += __popc(__ballot_sync(0xffffffffu, near <= (int)(t0 + PL_STEP)));
            end0 = offset(k0);
            w0 = weight_of(q, k0);
            owned0 = k0 > 0 && k0 <= q.N;
        }
        if (q.g) {
            float *const to = q.g + begin + t;
            if (q.vectors && t + 4 <= len) {
                __stcs(reinterpret_cast<float4 *>(to), make_float4(g[0], g[1], g[2], g[3]));
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (t + j < len) to[j] = g[j];
            }
        }
    }
    return loss;
}

// Sum over the block's warps, in their order; in the first thread.
__device__ __forceinline__ double warps_sum(double v, double *s)
{
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.0;
    if (threadIdx.x == 0)
        for (uint32_t w = 0; w < PL_WARPS; ++w) v += s[w];
    return v;
}

template <bool REF>
__global__ void __launch_bounds__(PL_THREADS) k_policy_tokens(const TokenParams q)
{
    __shared__ double s[PL_WARPS];
    const uint64_t begin = ((uint64_t)blockIdx.x * PL_WARPS + (threadIdx.x >> 5)) * q.per_warp;
    pdl_go();
    const double loss = warps_sum(run_tokens<REF>(q, begin, begin < q.T ? (uint32_t)min(q.per_warp, q.T - begin) : 0, threadIdx.x & 31), s);
    if (threadIdx.x == 0) q.part[blockIdx.x] = loss;
}

// Small losses of one program: one launch of one cluster, each block with all the weights in its shared memory.  On the device it is no
// shorter than the three kernels that overlap (100 samples of 113 tokens 7.8 us and 7.3, 1,000 of 30 12.2 and 9.9), but the
// host makes one launch for three (15 us a call, 20).
constexpr uint32_t SMALL_BLOCKS = 8, SMALL_N = 256, SMALL_T = 16384;

template <bool REF>
__global__ void __launch_bounds__(PL_THREADS) k_policy_small(const __grid_constant__ GroupParams g, const __grid_constant__ TokenParams all,
                                                             float *out)
{
    __shared__ double2 s_weights[SMALL_N];
    __shared__ double s[PL_WARPS], s_part[SMALL_BLOCKS];
    cg::cluster_group cluster = cg::this_cluster();
    const uint32_t part = cluster.block_rank();
    TokenParams q = all;
    q.weights = s_weights;
    const uint64_t begin = ((uint64_t)part * PL_WARPS + (threadIdx.x >> 5)) * q.per_warp;
    advantages<SMALL_N / PL_THREADS>(g, 0, PL_THREADS, threadIdx.x, s_weights, part == 0 ? g.advantage : nullptr,
                                     [&](double v, uint32_t) { return block_sum(v, s); });
    cluster.sync();  // (the weights are there; all blocks run)
    const double loss = warps_sum(run_tokens<REF>(q, begin, begin < q.T ? (uint32_t)min(q.per_warp, q.T - begin) : 0, threadIdx.x & 31), s);
    if (threadIdx.x == 0) *cluster.map_shared_rank(&s_part[part], 0) = loss;
    cluster.sync();
    if (part == 0 && threadIdx.x == 0) {
        double v = 0.0;
        for (uint32_t b = 0; b < SMALL_BLOCKS; ++b) v += s_part[b];
        *out = (float)v;
    }
}

__global__ void __launch_bounds__(PL_THREADS) k_policy_sum(const double *part, uint32_t n, float *loss)
{
    __shared__ double s[PL_WARPS];
    pdl_wait();
    double v = 0.0;
    for (uint32_t i = threadIdx.x; i < n; i += PL_THREADS) v += part[i];
    v = block_sum(v, s);
    if (threadIdx.x == 0) *loss = (float)v;
}

template <typename... P, typename... A>
cudaError_t launch_cluster(void (*kernel)(P...), uint32_t blocks, uint32_t parts, uint32_t threads, cudaStream_t st, const A &...args)
{
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = parts;
    at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(blocks); cfg.blockDim = threads; cfg.stream = st;
    cfg.attrs = &at; cfg.numAttrs = 1;
    g_vl_launches.fetch_add(1);
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

}  // namespace

extern "C" uint64_t vl_policy_work(uint64_t n_candidates, uint64_t n_tokens)
{
    const uint64_t blocks = (n_tokens + PL_STEP * PL_WARPS - 1) / (PL_STEP * PL_WARPS);
    return 16 * n_candidates + 8 * (blocks < PL_MAX_BLOCKS ? blocks : PL_MAX_BLOCKS) + 16;
}

extern "C" int vl_policy_loss(int device, uint32_t n, const vl_verdict *const *d_out, const uint64_t *K, const int64_t *d_token_off,
                              uint64_t n_tokens, const float *d_logprob, const float *d_old_logprob, const float *d_ref_logprob,
                              const vl_policy_rules *rules, float *d_loss, float *d_advantage, float *d_g_logprob, void *d_work,
                              uint64_t work_bytes, void *stream)
{
    if (!rules || !d_loss || !d_token_off || (n && (!d_out || !K)) || (n_tokens && !d_logprob)) return VL_ERR_INVALID_ARG;
    if (((uintptr_t)d_token_off & 7) || ((uintptr_t)d_work & 15)) return VL_ERR_INVALID_ARG;
    if (((uintptr_t)d_logprob | (uintptr_t)d_old_logprob | (uintptr_t)d_ref_logprob | (uintptr_t)d_loss | (uintptr_t)d_advantage |
         (uintptr_t)d_g_logprob) & 3)
        return VL_ERR_INVALID_ARG;
    // (so that squares of rewards, a weight in 32 bits and what it is multiplied with are numbers)
    if (!(fabs(rules->pair_cost) <= 1e20 && fabs(rules->bank_cost) <= 1e20 && fabs(rules->kl) <= 1e30)) return VL_ERR_INVALID_ARG;
    if (!(rules->clip_lo >= 0.0 && rules->clip_hi >= 0.0) || (rules->kl != 0.0 && n_tokens && !d_ref_logprob)) return VL_ERR_INVALID_ARG;
    if (rules->normalise && !(rules->eps >= 1e-100 && isfinite(rules->eps))) return VL_ERR_INVALID_ARG;
    if (n_tokens > (1ull << 40)) return VL_ERR_INVALID_ARG;
    uint64_t N = 0;
    for (uint32_t j = 0; j < n; ++j) {
        if (K[j] > (1ull << 31) || (K[j] && (!d_out[j] || ((uintptr_t)d_out[j] & 15)))) return VL_ERR_INVALID_ARG;
        N += K[j];
    }
    if (!d_work || work_bytes < vl_policy_work(N, n_tokens)) return VL_ERR_INVALID_ARG;
    const DeviceScope scope(device);
    if (scope.error != cudaSuccess) return VL_ERR_CUDA;
    cudaStream_t st = (cudaStream_t)stream;
    GroupParams q;
    q.pair_cost = rules->pair_cost; q.bank_cost = rules->bank_cost; q.eps = rules->eps; q.normalise = rules->normalise;
    q.off = d_token_off; q.N = N; q.T = n_tokens;
    q.weights = static_cast<double2 *>(d_work); q.advantage = d_advantage; q.per_token = rules->per_token;
    double *const part = reinterpret_cast<double *>(q.weights + N);
    TokenParams t;
    t.weights = q.weights; t.off = d_token_off; t.N = N; t.T = n_tokens;
    t.lp = d_logprob; t.old = d_old_logprob; t.ref = d_ref_logprob;
    t.at_lo = rules->clip_lo < 1.0 ? 1.0 - rules->clip_lo : 0.0;
    t.at_hi = 1.0 + rules->clip_hi;
    const double lo = rules->clip_lo < 1.0 ? log1p(-rules->clip_lo) : -HUGE_VAL, hi = log1p(rules->clip_hi);
    t.lo = (float)lo; t.lo_rest = isfinite(lo) ? (float)(lo - t.lo) : 0.0f;
    t.hi = (float)hi; t.hi_rest = isfinite(hi) ? (float)(hi - t.hi) : 0.0f;
    if (!isfinite(t.at_hi)) t.at_hi = 0.0;  // (never taken)
    t.kl = rules->kl;
    t.g = d_g_logprob; t.part = part;
    t.vectors = !(((uintptr_t)d_logprob | (uintptr_t)d_old_logprob | (uintptr_t)(rules->kl != 0.0 ? d_ref_logprob : nullptr) | (uintptr_t)d_g_logprob) & 15);
    const uint64_t steps = (n_tokens + PL_STEP - 1) / PL_STEP;
    uint64_t first = 0;
    for (uint32_t j = 0; j < n;) {
        uint32_t m = 0;
        uint64_t most = 0;
        for (; j < n && m < PL_GROUPS; ++j) {
            if (!K[j]) continue;
            q.out[m] = reinterpret_cast<const uint4 *>(d_out[j]);
            q.K[m] = K[j];
            q.first[m++] = first;
            first += K[j];
            most = K[j] > most ? K[j] : most;
        }
        if (!m) break;
        if (m == 1 && q.K[0] == N && N <= SMALL_N && n_tokens <= SMALL_T) {
            t.per_warp = (steps + SMALL_BLOCKS * PL_WARPS - 1) / (SMALL_BLOCKS * PL_WARPS) * PL_STEP;
            const auto kernel = t.kl != 0.0 ? k_policy_small<true> : k_policy_small<false>;
            return launch_cluster(kernel, SMALL_BLOCKS, SMALL_BLOCKS, PL_THREADS, st, q, t, d_loss) == cudaSuccess ? VL_OK : VL_ERR_CUDA;
        }
        // a block, or a cluster for programs of many candidates
        const uint32_t parts = most > 2 * ADV_THREADS ? 8 : 1;
        const uint64_t threads = (most / parts + 31) / 32 * 32;
        if (launch_cluster(k_advantages, m * parts, parts, (uint32_t)(threads < 64 ? 64 : threads < ADV_THREADS ? threads : ADV_THREADS), st, q) != cudaSuccess)
            return VL_ERR_CUDA;
    }
    uint64_t blocks = (steps + PL_WARPS - 1) / PL_WARPS;
    const uint64_t resident = 8 * (uint64_t)vl_device_sm_count(device);
    const uint64_t at_most = resident < PL_MAX_BLOCKS ? resident : PL_MAX_BLOCKS;
    if (blocks > at_most) blocks = at_most;
    if (blocks) {
        t.per_warp = (steps + blocks * PL_WARPS - 1) / (blocks * PL_WARPS) * PL_STEP;
        if (launch_overlap(t.kl != 0.0 ? k_policy_tokens<true> : k_policy_tokens<false>, dim3((uint32_t)blocks), PL_THREADS, 0, st, N != 0, t) !=
            cudaSuccess)
            return VL_ERR_CUDA;
    }
    if (launch_overlap(k_policy_sum, dim3(1), PL_THREADS, 0, st, blocks != 0, (const double *)part, (uint32_t)blocks, d_loss) != cudaSuccess)
        return VL_ERR_CUDA;
    return VL_OK;
}
