// The loss that makes the verifier's verdicts a training signal (Section 6): rewards of the sampled candidates, advantages within
// the samples of each program, the clipped objective over their tokens, and its derivative to every token's log probability.
//
//   reward = [pass] - pair_cost conflict_pairs - bank_cost bank_conflicts,   A = reward - mean  (/ (std + eps))
//   d = logprob - old, rho = exp d,  token loss = -min(rho A, clip(rho) A) + kl (exp q - q - 1),  q = ref - logprob
// The sign of a token loss's sum rests on small differences (A sums to nothing within a program, rho is near 1): rewards,
// advantages and sums are held in 64 bits, rho - 1 comes from expm1, and the clip's borders are compared as logarithms in 64 bits.
#include <math.h>

#include "vl_logits.cuh"

namespace {

constexpr uint32_t PL_GROUPS = 96;    // programs per launch (their pointers travel as kernel arguments)
constexpr uint32_t PL_THREADS = 256;
constexpr uint32_t PL_TILE = 2048;    // tokens of a block

struct GroupParams {
    const uint4 *out[PL_GROUPS];
    uint64_t K[PL_GROUPS], first[PL_GROUPS];  // first: candidate number of its first row
    double pair_cost, bank_cost, eps;
    double *adv;
    float *advantage;
    int normalise;
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

// One block per program.
__global__ void __launch_bounds__(PL_THREADS) k_advantages(const GroupParams q)
{
    __shared__ double s[PL_THREADS / 32];
    const uint32_t j = blockIdx.x;
    const uint64_t K = q.K[j];
    const uint4 *out = q.out[j];
    // taken from the first one's: equal rewards leave exactly nothing, which a division by their deviation would blow up
    const double base = reward_of(__ldg(out), q.pair_cost, q.bank_cost);
    double sum = 0.0;
    for (uint64_t k = threadIdx.x; k < K; k += PL_THREADS) sum += reward_of(__ldg(out + k), q.pair_cost, q.bank_cost) - base;
    const double mean = block_sum(sum, s) / (double)K;
    double by = 1.0;
    if (q.normalise) {
        double var = 0.0;
        for (uint64_t k = threadIdx.x; k < K; k += PL_THREADS) {
            const double c = reward_of(__ldg(out + k), q.pair_cost, q.bank_cost) - base - mean;
            var += c * c;
        }
        by = 1.0 / (sqrt(block_sum(var, s) / (double)K) + q.eps);
    }
    for (uint64_t k = threadIdx.x; k < K; k += PL_THREADS) {
        const double a = (reward_of(__ldg(out + k), q.pair_cost, q.bank_cost) - base - mean) * by;
        q.adv[q.first[j] + k] = a;
        if (q.advantage) q.advantage[q.first[j] + k] = (float)a;
    }
}

struct TokenParams {
    const double *adv;
    const int64_t *off;
    uint64_t N, T;
    const float *lp, *old, *ref;
    double log_lo, log_hi, at_lo, at_hi, kl;
    int per_token;
    float *g;
    double *part;
};

__global__ void __launch_bounds__(PL_THREADS) k_policy_tokens(const TokenParams q)
{
    __shared__ double s[PL_THREADS / 32];
    const double inf = __longlong_as_double(0x7ff0000000000000ll);
    const int64_t span = min(max(q.off[q.N], (int64_t)0), (int64_t)q.T) - min(max(q.off[0], (int64_t)0), (int64_t)q.T);
    double loss = 0.0;
    for (uint32_t j = 0; j < PL_TILE / PL_THREADS; ++j) {
        const uint64_t t = (uint64_t)blockIdx.x * PL_TILE + j * PL_THREADS + threadIdx.x;
        if (t >= q.T) break;
        uint64_t a = 0, b = q.N + 1;  // the first offset above t
        while (a < b) {
            const uint64_t mid = (a + b) >> 1;
            if (q.off[mid] <= (int64_t)t) a = mid + 1; else b = mid;
        }
        float grad = 0.0f;
        if (a > 0 && a <= q.N) {
            const uint64_t k = a - 1;
            const double A = q.adv[k], lp = q.lp[t], old = q.old ? (double)q.old[t] : lp, ref = q.kl != 0.0 ? (double)q.ref[t] : lp;
            if (lp != -inf && old != -inf && ref != -inf) {
                const double w = 1.0 / (q.per_token ? (double)max(span, (int64_t)1)
                                                    : (double)q.N * (double)max(q.off[k + 1] - q.off[k], (int64_t)1));
                const double d = lp - old;
                const double Am = A * (double)expm1f((float)d);
                const bool outside = A > 0.0 ? d > q.log_hi : d < q.log_lo;
                double term = outside ? -A * (A > 0.0 ? q.at_hi : q.at_lo) : -(A + Am);
                double slope = outside ? 0.0 : -(A + Am);
                if (q.kl != 0.0) {
                    const double e = ref - lp, em = (double)expm1f((float)e);
                    term += q.kl * (em - e);
                    slope -= q.kl * em;
                }
                loss += w * term;
                grad = (float)(w * slope);
            }
        }
        if (q.g) q.g[t] = grad;
    }
    loss = block_sum(loss, s);
    if (threadIdx.x == 0) q.part[blockIdx.x] = loss;
}

__global__ void __launch_bounds__(PL_THREADS) k_policy_sum(const double *part, uint64_t n, float *loss)
{
    __shared__ double s[PL_THREADS / 32];
    double v = 0.0;
    for (uint64_t i = threadIdx.x; i < n; i += PL_THREADS) v += part[i];
    v = block_sum(v, s);
    if (threadIdx.x == 0) *loss = (float)v;
}

uint64_t policy_tiles(uint64_t n_tokens) { return (n_tokens + PL_TILE - 1) / PL_TILE; }

}  // namespace

extern "C" uint64_t vl_policy_work(uint64_t n_candidates, uint64_t n_tokens)
{
    return 8 * (n_candidates + policy_tiles(n_tokens) + 1);
}

extern "C" int vl_policy_loss(int device, uint32_t n, const vl_verdict *const *d_out, const uint64_t *K, const int64_t *d_token_off,
                              uint64_t n_tokens, const float *d_logprob, const float *d_old_logprob, const float *d_ref_logprob,
                              const vl_policy_rules *rules, float *d_loss, float *d_advantage, float *d_g_logprob, void *d_work,
                              uint64_t work_bytes, void *stream)
{
    if (!rules || !d_loss || !d_token_off || (n && (!d_out || !K)) || (n_tokens && !d_logprob)) return VL_ERR_INVALID_ARG;
    if (((uintptr_t)d_token_off & 7) || ((uintptr_t)d_work & 7)) return VL_ERR_INVALID_ARG;
    if (((uintptr_t)d_logprob | (uintptr_t)d_old_logprob | (uintptr_t)d_ref_logprob | (uintptr_t)d_loss | (uintptr_t)d_advantage |
         (uintptr_t)d_g_logprob) & 3)
        return VL_ERR_INVALID_ARG;
    if (!(isfinite(rules->pair_cost) && isfinite(rules->bank_cost) && isfinite(rules->kl))) return VL_ERR_INVALID_ARG;
    if (!(rules->clip_lo >= 0.0 && rules->clip_hi >= 0.0) || (rules->kl != 0.0 && n_tokens && !d_ref_logprob)) return VL_ERR_INVALID_ARG;
    if (rules->normalise && !(rules->eps > 0.0 && isfinite(rules->eps))) return VL_ERR_INVALID_ARG;
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
    double *adv = static_cast<double *>(d_work), *part = adv + N;
    GroupParams q;
    q.pair_cost = rules->pair_cost; q.bank_cost = rules->bank_cost; q.eps = rules->eps; q.normalise = rules->normalise;
    q.adv = adv; q.advantage = d_advantage;
    uint64_t first = 0;
    for (uint32_t j = 0; j < n;) {
        uint32_t m = 0;
        for (; j < n && m < PL_GROUPS; ++j) {
            if (!K[j]) continue;
            q.out[m] = reinterpret_cast<const uint4 *>(d_out[j]);
            q.K[m] = K[j];
            q.first[m++] = first;
            first += K[j];
        }
        if (!m) break;
        k_advantages<<<m, PL_THREADS, 0, st>>>(q);
        g_vl_launches.fetch_add(1);
    }
    TokenParams t;
    t.adv = adv; t.off = d_token_off; t.N = N; t.T = n_tokens;
    t.lp = d_logprob; t.old = d_old_logprob; t.ref = d_ref_logprob;
    t.at_lo = rules->clip_lo < 1.0 ? 1.0 - rules->clip_lo : 0.0;
    t.at_hi = 1.0 + rules->clip_hi;
    t.log_lo = rules->clip_lo < 1.0 ? log1p(-rules->clip_lo) : -HUGE_VAL;
    t.log_hi = log1p(rules->clip_hi);
    t.kl = rules->kl; t.per_token = rules->per_token;
    t.g = d_g_logprob; t.part = part;
    const uint64_t tiles = policy_tiles(n_tokens);
    if (tiles) {
        k_policy_tokens<<<(uint32_t)tiles, PL_THREADS, 0, st>>>(t);
        g_vl_launches.fetch_add(1);
    }
    k_policy_sum<<<1, PL_THREADS, 0, st>>>(part, tiles, d_loss);
    g_vl_launches.fetch_add(1);
    return cudaGetLastError() == cudaSuccess ? VL_OK : VL_ERR_CUDA;
}
