// One token of every row of logits from a given random number, with temperature, top-k, top-p and min-p, under the masks of occupied
// registers: the draw of a candidate's registers (Section 3.1), around those that are taken (Section 4.5, last paragraph).
//
// With z_i = scale (x_i - M) over the open entries, M the largest of them, w_i = exp z_i.  In the order "larger logit first, lower number
// first among equals" the kept entries are a prefix: the shortest of the first top_k, of those whose sum reaches top_p times the sum of
// these, and of those with w >= min_p.  So they are told by a logit and a number: every entry above the logit, and the first m of those equal
// to it.  With T the sum of w over the kept ones the token is the lowest kept entry up to which (in the order of their numbers) the sum of w
// is above u T.
//
// Which entries are kept, and which one a number falls on, is decided as in 64 bits: sums of 32-bit terms are off by some 2^-20, which for
// rows of 100,000 entries is where a number falls on another token every tenth row.
#pragma once
#include "vl_rank.cuh"

struct SampleRules {
    const float *uniform;  // [n_rows]
    uint32_t top_k;        // 0: all
    double top_p, min_p;
};
struct SampleOut {
    void *tokens;
    uint32_t token_bytes;
    float *logprob, *drawn;  // null: not wanted
    int32_t *kept;
};
cudaError_t vl_sample_f32(const LogitRows &q, const SampleRules &s, const SampleOut &o, int device, cudaStream_t st);
cudaError_t vl_sample_f16(const LogitRows &q, const SampleRules &s, const SampleOut &o, int device, cudaStream_t st);
cudaError_t vl_sample_bf16(const LogitRows &q, const SampleRules &s, const SampleOut &o, int device, cudaStream_t st);

namespace {

constexpr uint32_t LEAST_KEY = 0x00800000u;  // of the lowest number; minus infinity lies below

__device__ __forceinline__ void put_sample(const SampleOut &o, uint64_t r, int64_t token, float logprob, float drawn, uint32_t kept)
{
    if (o.token_bytes == 2) static_cast<uint16_t *>(o.tokens)[r] = (uint16_t)token;
    else if (o.token_bytes == 4) static_cast<int32_t *>(o.tokens)[r] = (int32_t)token;
    else static_cast<int64_t *>(o.tokens)[r] = token;
    if (o.logprob) o.logprob[r] = logprob;
    if (o.drawn) o.drawn[r] = drawn;
    if (o.kept) o.kept[r] = (int32_t)kept;
}
__device__ __forceinline__ bool drawn_at_all(float u) { return u >= 0.0f && u < 1.0f; }

// ---- in 64 bits
// NT threads (a warp, or a block) at a row that they read as often as they need it, 32 entries of a warp at a time.  All threads hold
// the same results; every sum has one order.
template <int NT>
struct Team {
    static constexpr uint32_t NW = NT / 32;
    double *s_d;    // [2][NW]
    uint32_t *s_u;  // [2][NW][3]
    uint32_t turn = 0;
    __device__ __forceinline__ uint32_t lane() const { return threadIdx.x & 31; }
    __device__ __forceinline__ uint32_t warp() const { return NT == 32 ? 0 : threadIdx.x >> 5; }
    __device__ __forceinline__ double sum(double v)
    {
#pragma unroll
        for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
        if (NT == 32) return v;
        double *s = s_d + (turn++ & 1) * NW;  // (the set of two calls ago has been read before the barrier of the last one)
        if (lane() == 0) s[warp()] = v;
        __syncthreads();
        v = 0.0;
        for (uint32_t w = 0; w < NW; ++w) v += s[w];
        return v;
    }
    struct Three {
        uint32_t sum, least, most;
    };
    __device__ __forceinline__ Three three(Three v)
    {
        v.sum = __reduce_add_sync(0xffffffffu, v.sum);
        v.least = __reduce_min_sync(0xffffffffu, v.least);
        v.most = __reduce_max_sync(0xffffffffu, v.most);
        if (NT == 32) return v;
        uint32_t *s = s_u + (turn++ & 1) * (3 * NW);
        if (lane() == 0) { s[3 * warp()] = v.sum; s[3 * warp() + 1] = v.least; s[3 * warp() + 2] = v.most; }
        __syncthreads();
        v = Three{0u, 0xFFFFFFFFu, 0u};
        for (uint32_t w = 0; w < NW; ++w) {
            v.sum += s[3 * w];
            v.least = min(v.least, s[3 * w + 1]);
            v.most = max(v.most, s[3 * w + 2]);
        }
        return v;
    }
};

// Entry of a row, minus infinity if it is closed.  Word w of the mask is asked for by the whole warp.
template <typename T>
__device__ __forceinline__ float open_entry(const T *row, const RowMask &mask, bool masked, uint32_t w, uint32_t lane)
{
    const uint32_t i = w * 32 + lane;
    const float none = __int_as_float(0xFF800000);
    if (i >= mask.V) return none;
    if (masked && (mask.closed(w) >> lane & 1)) return none;
    return to_f32(row[i]);
}

template <typename T, int NT>
__device__ __noinline__ void sample_row_64(const LogitRows &q, const SampleRules &rules, const SampleOut &o, uint64_t r, double *s_d,
                                           uint32_t *s_u)
{
    Team<NT> team{s_d, s_u};
    constexpr uint32_t NW = Team<NT>::NW;
    const uint32_t lane = team.lane(), warp = team.warp();
    const float inf = __int_as_float(0x7f800000);
    const T *row = static_cast<const T *>(q.x) + r * q.stride;
    const RowMask mask = row_mask(q, r);
    const bool masked = mask.any();
    const uint32_t words = (q.V + 31) / 32;
    auto each = [&](auto &&f) {  // f(key): of the entries that are open and possible
        for (uint32_t w = warp; w < words; w += NW) {
            const float x = open_entry<T>(row, mask, masked, w, lane);
            if (x > -inf) f(ordered(x));
        }
    };
    // the largest, and whether something is no number
    uint32_t most = 0, bad = 0, n = 0;
    for (uint32_t w = warp; w < words; w += NW) {
        const float x = open_entry<T>(row, mask, masked, w, lane);
        if (!(x < inf)) bad = 1;
        if (x > -inf) { most = max(most, ordered(x)); ++n; }
    }
    const auto first = team.three({n, bad ? 0u : 1u, most});
    n = first.sum;
    most = first.most;
    const bool leader = NT == 32 ? lane == 0 : threadIdx.x == 0;
    if (first.least == 0) {
        if (leader) put_sample(o, r, -1, __int_as_float(0x7fc00000), __int_as_float(0x7fc00000), 0);
        return;
    }
    if (n == 0) {
        if (leader) put_sample(o, r, -1, -inf, -inf, 0);
        return;
    }
    const double M = (double)from_ordered(most), scale = (double)q.scale;
    auto weight = [&](uint32_t key) { return exp(scale * ((double)from_ordered(key) - M)); };

    // all of them
    double S = 0.0;
    each([&](uint32_t key) { S += weight(key); });
    S = team.sum(S);

    // kept: keys above `cut`, and the first `ties` of those equal to it
    uint32_t cut = LEAST_KEY - 1, ties = 0;
    double among = S;  // sum over these
    if (rules.top_k && rules.top_k < n) {
        // the largest key that top_k entries reach: at least lo, below hi
        uint32_t lo = LEAST_KEY, hi = most + 1, above = 0;
        while (hi - lo > 1) {
            const uint32_t mid = lo + (hi - lo) / 2;
            typename Team<NT>::Three t{0u, 0xFFFFFFFFu, 0u};
            each([&](uint32_t key) {
                if (key >= hi || key < lo) return;
                if (key >= mid) { ++t.sum; t.least = min(t.least, key); }
                else t.most = max(t.most, key);
            });
            t = team.three(t);
            if (above + t.sum >= rules.top_k) {
                lo = t.least;
            } else {
                above += t.sum;
                hi = t.most ? t.most + 1 : lo + 1;
            }
        }
        cut = lo;
        ties = rules.top_k - above;
        double sum = 0.0;
        each([&](uint32_t key) { if (key > cut) sum += weight(key); });
        among = team.sum(sum) + (double)ties * weight(cut);
    }
    if (rules.top_p < 1.0) {
        const double need = rules.top_p * among;
        uint32_t lo = cut, hi = most + 1;
        double above = 0.0;
        while (hi - lo > 1) {
            const uint32_t mid = lo + (hi - lo) / 2;
            typename Team<NT>::Three t{0u, 0xFFFFFFFFu, 0u};
            double sum = 0.0;
            each([&](uint32_t key) {
                if (key >= hi || key <= cut) return;
                if (key >= mid) { sum += weight(key); t.least = min(t.least, key); }
                else if (key > lo) t.most = max(t.most, key);
            });
            sum = above + team.sum(sum);
            t = team.three(t);
            if (sum >= need && t.least != 0xFFFFFFFFu) {
                lo = t.least;
            } else {
                above = sum;
                hi = t.most ? t.most + 1 : lo + 1;
            }
        }
        // (lo is an entry's key, or the cut that was there)
        typename Team<NT>::Three t{0u, 0u, 0u};
        each([&](uint32_t key) { t.sum += key == lo; });
        const uint32_t there = lo == cut ? ties : team.three(t).sum;
        const double w = weight(lo);
        const double m = w > 0.0 ? ceil((need - above) / w) : 1.0;
        ties = lo == cut && ties == 0 ? 0 : (uint32_t)min(max(m, 1.0), (double)there);
        cut = lo;
    }
    if (rules.min_p > 0.0 && (cut < LEAST_KEY || weight(cut) < rules.min_p)) {
        uint32_t lo = max(cut, LEAST_KEY - 1), hi = most;  // the lowest key whose weight is enough: above lo, at most hi
        while (hi - lo > 1) {
            const uint32_t mid = lo + (hi - lo) / 2;
            if (weight(mid) >= rules.min_p) hi = mid;
            else lo = mid;
        }
        cut = hi - 1;
        ties = 0;
    }

    // what the warps' runs of entries hold of them; a run's ties are kept as far as there are some left
    const uint32_t per = (words + NW - 1) / NW, w0 = min(words, warp * per), w1 = min(words, w0 + per);
    double sum = 0.0;
    uint32_t count = 0, equal = 0;
    for (uint32_t w = w0; w < w1; ++w) {
        const float x = open_entry<T>(row, mask, masked, w, lane);
        if (!(x > -inf)) continue;
        const uint32_t key = ordered(x);
        if (key > cut) { sum += weight(key); ++count; }
        equal += key == cut;
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    count = __reduce_add_sync(0xffffffffu, count);
    equal = __reduce_add_sync(0xffffffffu, equal);
    const double level = ties ? weight(cut) : 0.0;
    double total = sum + (double)min(equal, ties) * level, base = 0.0;
    uint32_t before = 0, kept = count + min(equal, ties), mine = warp;
    if (NT > 32) {
        const uint32_t set = team.turn++ & 1;
        double *d = s_d + set * NW;
        uint32_t *u = s_u + set * (3 * NW);
        if (lane == 0) { d[warp] = sum; u[3 * warp] = count; u[3 * warp + 1] = equal; }
        __syncthreads();
        auto run = [&](uint32_t w, uint32_t &b) {  // kept weight of warp w, b ties in front of it
            const uint32_t m = min(u[3 * w + 1], ties - min(ties, b));
            b += u[3 * w + 1];
            return d[w] + (double)m * level;
        };
        total = 0.0;
        kept = 0;
        uint32_t b = 0;
        for (uint32_t w = 0; w < NW; ++w) {
            total += run(w, b);
            kept += u[3 * w];
        }
        kept += min(b, ties);
        // the run that the number falls into: the first up to whose end the sum is above it, or the last with something kept
        const double at = (double)rules.uniform[r] * total;
        double up = 0.0;
        b = 0;
        mine = 0xFFFFFFFFu;
        for (uint32_t w = 0; w < NW; ++w) {
            const uint32_t b0 = b;
            const double v = run(w, b), next = up + v;
            if (v > 0.0) {
                mine = w;
                base = up;
                before = b0;
                if (next > at) break;
            }
            up = next;
        }
    }
    if (warp != mine) return;
    const double at = (double)rules.uniform[r] * total;
    uint32_t token = 0xFFFFFFFFu;
    for (uint32_t w = w0; w < w1; ++w) {
        const float x = open_entry<T>(row, mask, masked, w, lane);
        const uint32_t key = x > -inf ? ordered(x) : 0u;
        const uint32_t same = __ballot_sync(0xffffffffu, key == cut && key);
        const bool in = key > cut || (key == cut && key && before + __popc(same & ((1u << lane) - 1)) < ties);
        before += __popc(same);
        const uint32_t ins = __ballot_sync(0xffffffffu, in);
        if (!ins) continue;
        double up = in ? weight(key) : 0.0;
        const double own = up;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const double v = __shfl_up_sync(0xffffffffu, up, d);
            if (lane >= d) up += v;
        }
        up += base;
        const uint32_t some = __ballot_sync(0xffffffffu, in && own > 0.0), past = __ballot_sync(0xffffffffu, in && own > 0.0 && up > at);
        base = __shfl_sync(0xffffffffu, up, 31);
        if (past) { token = w * 32 + __ffs(past) - 1; break; }
        if (some) token = w * 32 + 31 - __clz(some);  // (rounding may leave the number behind the last one)
    }
    if (lane == 0) {
        const double z = scale * ((double)to_f32(row[token]) - M);
        put_sample(o, r, token, (float)(z - log(S)), (float)(z - log(total)), kept);
    }
}

template <typename T, int NT>
__global__ void __launch_bounds__(NT == 32 ? 256 : NT) k_sample_64(const LogitRows q, const SampleRules s, const SampleOut o)
{
    __shared__ double s_d[2 * Team<NT>::NW];
    __shared__ uint32_t s_u[6 * Team<NT>::NW];
    const uint64_t teams = NT == 32 ? (uint64_t)gridDim.x * 8 : gridDim.x;
    for (uint64_t r = NT == 32 ? (uint64_t)blockIdx.x * 8 + (threadIdx.x >> 5) : blockIdx.x; r < q.n_rows; r += teams) {
        if (!drawn_at_all(s.uniform[r])) {
            if ((NT == 32 ? threadIdx.x & 31 : threadIdx.x) == 0) put_sample(o, r, -1, 0.0f, 0.0f, 0);
            continue;
        }
        sample_row_64<T, NT>(q, s, o, r, s_d, s_u);
        if (NT > 32) __syncthreads();  // (the next row's first sums may go where this row's last ones are read)
    }
}

}  // namespace
