// Drawing from short rows: a group of lanes, or a warp, holds a row in registers.
//
// Weights and sums are in 32 bits, u = 2^-24.  A weight is within (4 + 1.6 |y|) u of its value relatively, y its power of two (its
// roundings and the scale's, and the exponential's own error), and the mean of |y| over a row's probabilities is at most log2(entries / S), S the sum relative to
// the largest one (their entropy is at most that of equal ones).  With C the sum up to a border and T the whole one, C - a T is then known to
//     u T (4 * 2 a (1 - a) + 1.6 log2(entries / S) max(a, 1 - a) + a (additions of C and of T) + 4):
// the equal part of the errors is shared by C and T, the other one may be all on one side.  Where a border is nearer than that to the number
// that it is compared with, the warp works out the row in 64 bits (some hundred of 200,000 rows of 256 entries).
//
// What bounds them: instructions and the loads' latency.  200,000 rows of 256 bf16 logits (17 us of bytes) take 42 us without rules, 46 with min_p,
// 52 under masks and widths as well; a warp per row, which top_k and top_p take, is 189 with top_k 8, 432 with top_p 0.9.
#pragma once
#include "vl_sample.cuh"

namespace {

// Powers of two of a vector's entries relative to m.
template <typename T>
__device__ __forceinline__ void powers(const float (&x)[EPV<T>], float m, float c, bool far, float (&e)[EPV<T>])
{
    if (!far) {
        const float b = -__fmul_rn(m, c);
        const f32x2 c2 = both(c, c), low = both(b, b);
#pragma unroll
        for (int j = 0; j < EPV<T>; j += 2) {
            float y0, y1;
            apart(fma2(both(x[j], x[j + 1]), c2, low), y0, y1);
            e[j] = ex2(y0);
            e[j + 1] = ex2(y1);
        }
    } else {
#pragma unroll
        for (int j = 0; j < EPV<T>; ++j) e[j] = ex2((x[j] - m) * c);
    }
}
template <int N>
__device__ __forceinline__ float sum_of(const float (&e)[N])
{
    f32x2 s = both(e[0], e[1]);
#pragma unroll
    for (int j = 2; j < N; j += 2) s = add2(s, both(e[j], e[j + 1]));
    float a, b;
    apart(s, a, b);
    return a + b;
}
// ln of a sum of weights relative to m.
__device__ __forceinline__ float log_of(float s, float m, float c)
{
    const float l = logf(s);
    return max_nan(far_out(m, c) ? l : fmaf(LN2, __fmaf_rn(-m, c, __fmul_rn(m, c)), l), 0.0f);
}
__device__ __forceinline__ float log_ratio(float x, float m, float scale, float l) { return min_nan((0.5f * x - 0.5f * m) * (2.0f * scale) - l, 0.0f); }

// A vector's entries from a logit on, counted up: halves two at a time, as numbers of their own type (up to 64 of each half, which bf16 holds).
struct Count {
    uint32_t n;
    __device__ __forceinline__ explicit Count(float) : n(0) {}
    __device__ __forceinline__ void add(const uint4 &r, float from)
    {
        float x[4];
        unpack(r, x, 0.0f);
#pragma unroll
        for (int i = 0; i < 4; ++i) n += x[i] >= from;
    }
    __device__ __forceinline__ uint32_t sum() const { return n; }
};
template <typename P, typename T>
struct CountPairs {
    P n;
    __device__ __forceinline__ void add(const uint4 &r, const P &from)
    {
        P h[4];
        memcpy(h, &r, 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) n = __hadd2(n, __hge2(h[i], from));
    }
};
template <typename T>
struct Counter {
    Count c{0.0f};
    float from;
    __device__ __forceinline__ explicit Counter(float f) : from(f) {}
    __device__ __forceinline__ void add(const uint4 &r) { c.add(r, from); }
    __device__ __forceinline__ uint32_t sum() const { return c.n; }
};
template <>
struct Counter<__half> {
    CountPairs<__half2, __half> c;
    __half2 from;
    __device__ __forceinline__ explicit Counter(float f) : from(__half2half2(__float2half_ru(f))) { c.n = __float2half2_rn(0.0f); }
    __device__ __forceinline__ void add(const uint4 &r) { c.add(r, from); }
    __device__ __forceinline__ uint32_t sum() const { return (uint32_t)(__low2float(c.n) + __high2float(c.n)); }
};
template <>
struct Counter<__nv_bfloat16> {
    CountPairs<__nv_bfloat162, __nv_bfloat16> c;
    __nv_bfloat162 from;
    __device__ __forceinline__ explicit Counter(float f) : from(__bfloat162bfloat162(__float2bfloat16_ru(f))) { c.n = __float2bfloat162_rn(0.0f); }
    __device__ __forceinline__ void add(const uint4 &r) { c.add(r, from); }
    __device__ __forceinline__ uint32_t sum() const { return (uint32_t)(__low2float(c.n) + __high2float(c.n)); }
};

template <int G> __device__ __forceinline__ float group_sum(float v)
{
#pragma unroll
    for (int d = G / 2; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}

// Which entries of a row are kept: those from `from` on, and of each vector of a lane the first ties[j] of those equal to `level`.
template <int NV>
struct Keep {
    float from, level;
    uint32_t ties[NV];
};

// The token of a row that a group holds, from number u, where one is wanted and the sum S over the whole row (worked out here) is one.  The
// lane that has the token gets it in `token`, with its logit.  False where a border is too near, in every lane of the group.
template <typename T, int G, int NV, bool PART, bool TIES>
__device__ __forceinline__ bool draw(const uint4 (&raw)[NV], const Keep<NV> &keep, const RowVectors<T> &x, float u, float m, float c,
                                     uint32_t lane, bool wanted, int64_t *token, float *x_tok, float *all, float *total, uint32_t *kept)
{
    const uint32_t g = lane % G;
    const bool far = far_out(m, c);
    float v[NV];
    uint32_t n = 0;
    // PART: not all of them are kept
    float S = 0.0f, T_all = 0.0f;
    Counter<T> counter(LOWEST);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        float xs[EPV<T>], e[EPV<T>];
        unpack(raw[j], xs, T{});
        powers<T>(xs, m, c, far, e);
        if (!PART) counter.add(raw[j]);
        if (PART) {
            S += sum_of(e);
            uint32_t ties = TIES ? keep.ties[j] : 0u;
#pragma unroll
            for (int i = 0; i < EPV<T>; ++i) {
                bool k = xs[i] >= keep.from;
                if (TIES && xs[i] == keep.level && ties) { k = true; --ties; }
                if (!k) e[i] = 0.0f;
                n += k;
            }
        }
        v[j] = sum_of(e);
        T_all += v[j];
    }
    if (!PART) n = counter.sum();
    T_all = group_sum<G>(T_all);
    S = PART ? group_sum<G>(S) : T_all;
    *all = S;
    *total = T_all;
    const bool some = wanted && S > 0.0f && S < __int_as_float(0x7f800000);
#pragma unroll
    for (int d = G / 2; d; d >>= 1) n += __shfl_xor_sync(0xffffffffu, n, d);
    *kept = n;
    // round by round: the group's vectors that the number falls into, and what lies in front of them
    constexpr float ADDS = EPV<T> / 2 + NV + (G == 4 ? 2 : G == 8 ? 3 : G == 16 ? 4 : 5), MORE = ADDS - EPV<T> / 2 + EPV<T> + 1;  // of T, and of C beyond
    const float at = u * T_all;
    const float margin = T_all * 0x1p-24f * (8.0f * u * (1.0f - u) + POWER_ERROR * fmaxf(u, 1.0f - u) * __log2f((float)x.V / S) + u * (2.0f * ADDS + MORE) + 4.5f);
    float base = 0.0f, up = 0.0f, own = 0.0f;
    uint4 vector = raw[0];
    uint32_t ties = TIES ? keep.ties[0] : 0u, turn = 0;
    bool found = false;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        if (!found) {
            base = up;
            vector = raw[j];
            own = v[j];
            turn = j;
            if (TIES) ties = keep.ties[j];
        }
        up += NV == 1 ? T_all : group_sum<G>(v[j]);
        found = found || up > at;
    }
    float incl = own;
#pragma unroll
    for (int d = 1; d < G; d *= 2) {
        const float w = __shfl_up_sync(0xffffffffu, incl, d, G);
        if (g >= (uint32_t)d) incl += w;
    }
    uint32_t past = __ballot_sync(0xffffffffu, base + incl > at);
    if (G < 32) past = past >> (lane - g) & ((1u << (G & 31)) - 1);
    bool sure = false;
    *token = -1;
    if (some && past && g == __ffs(past) - 1u) {
        float xs[EPV<T>], e[EPV<T>], cum = base + (incl - own);
        unpack(vector, xs, T{});
        powers<T>(xs, m, c, far, e);
        bool open = true;
#pragma unroll
        for (int i = 0; i < EPV<T>; ++i) {
            bool k = !PART || xs[i] >= keep.from;
            if (TIES && xs[i] == keep.level && ties) { k = true; --ties; }
            const float next = k ? cum + e[i] : cum;
            if (open && next > at) {
                open = false;
                sure = at >= cum + margin && next >= at + margin;
                *token = (int64_t)x.first(g + G * turn) + i;
                *x_tok = xs[i];
            }
            cum = next;
        }
        if (!sure) *token = -1;
    }
    uint32_t ok = __ballot_sync(0xffffffffu, sure);
    if (G < 32) ok = ok >> (lane - g) & ((1u << (G & 31)) - 1);
    return ok != 0;
}

// Rows that a group could not settle, one after another by the whole warp.
template <typename T, int G>
__device__ __forceinline__ void settle(const LogitRows &q, const SampleRules &s, const SampleOut &o, uint64_t r, float m, bool open, uint32_t lane)
{
    uint32_t left = __ballot_sync(0xffffffffu, open && lane % G == 0);
    while (left) {
        const uint64_t which = __shfl_sync(0xffffffffu, (unsigned long long)r, __ffs(left) - 1);
        const uint32_t known = ordered(__shfl_sync(0xffffffffu, m, __ffs(left) - 1));
        left &= left - 1;
        sample_row_64<T, 32>(q, s, o, which, nullptr, nullptr, 1, 0, known);
    }
}

// No rules, or min_p: what is kept is told by a logit at once.
template <typename T, bool MASKED, bool ALIGNED, bool PART, int G, int NV>
__global__ void __launch_bounds__(SHORT_WARPS * 32, short_blocks(NV)) k_sample_short(const LogitRows q, const SampleRules s, const SampleOut o)
{
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane % G;
    const float c = q.scale * LOG2E, inf = __int_as_float(0x7f800000), nan = __int_as_float(0x7fc00000);
    const uint64_t r0 = ((uint64_t)blockIdx.x * SHORT_WARPS + warp) * (32 / G);
    if (r0 >= q.n_rows) return;
    uint64_t row = 0;
    float most = 0.0f;
    bool left;
    {
        const uint64_t r = min(r0 + lane / G, q.n_rows - 1);
        const bool there = r0 + lane / G < q.n_rows;  // (the warp's last rows may not be: it works on the last one instead)
        const RowVectors<T> x(static_cast<const T *>(q.x) + r * q.stride, q.V);
        uint4 raw[NV];
        fetch_row<T, G, NV, ALIGNED>(raw, x, g, r != 0 && r != q.n_rows - 1);
        const float u = s.uniform[r];
        if (MASKED) close_row<T, G, NV, ALIGNED>(raw, x, row_mask(q, r), g, -1);
        float m = vectors_max<NV>(raw, T{});
#pragma unroll
        for (int d = G / 2; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
        if (m == -inf) m = 0.0f;  // (nothing possible: every power is 0)
        const bool drawn = drawn_at_all(u);
        Keep<NV> keep;
        keep.from = fmaxf(__double2float_ru((double)m + s.drop), LOWEST);
        int64_t token;
        float x_tok = 0.0f, S, T_all;
        uint32_t kept;
        const bool sure = draw<T, G, NV, PART, false>(raw, keep, x, u, m, c, lane, there && drawn, &token, &x_tok, &S, &T_all, &kept);
        const bool some = there && drawn && S > 0.0f && S < inf;
        if (token >= 0) {
            const float lp = log_ratio(x_tok, m, q.scale, log_of(S, m, c));
            put_sample(o, r, token, lp, PART ? log_ratio(x_tok, m, q.scale, log_of(T_all, m, c)) : lp, kept);
        }
        if (there && !some && g == 0) {
            const float v = !drawn ? 0.0f : S == 0.0f ? -inf : nan;
            put_sample(o, r, -1, v, v, 0);
        }
        left = some && !sure;
        row = r;
        most = m;
    }
    settle<T, G>(q, s, o, row, most, left, lane);
}

// top_k or top_p: a warp per row.  FEW: up to 32 entries are kept, by top_k.
template <typename T, bool MASKED, bool ALIGNED, bool FEW, int NV>
__global__ void __launch_bounds__(SHORT_WARPS * 32, FEW ? (NV <= 4 ? 4 : 3) : NV <= 2 ? 4 : NV == 4 ? 3 : 2) k_sample_warp(const LogitRows q, const SampleRules s, const SampleOut o)
{
    __shared__ key_t64 s_cand[FEW ? SHORT_WARPS : 1][FEW ? SHORT_CAND : 1];
    __shared__ uint32_t s_n[SHORT_WARPS];
    __shared__ float s_runs[FEW ? 1 : SHORT_WARPS][FEW ? 1 : 1024];
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const float c = q.scale * LOG2E, inf = __int_as_float(0x7f800000), nan = __int_as_float(0x7fc00000);
    const uint64_t step = (uint64_t)gridDim.x * SHORT_WARPS;
    for (uint64_t r = (uint64_t)blockIdx.x * SHORT_WARPS + warp; r < q.n_rows; r += step) {
        const RowVectors<T> x(static_cast<const T *>(q.x) + r * q.stride, q.V);
        uint4 raw[NV];
        fetch_row<T, 32, NV, ALIGNED>(raw, x, lane, r != 0 && r != q.n_rows - 1);
        const float u = s.uniform[r];
        if (MASKED) close_row<T, 32, NV, ALIGNED>(raw, x, row_mask(q, r), lane, -1);
        const float own = vectors_max<NV>(raw, T{});
        float m = own;
#pragma unroll
        for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
        if (m == -inf) m = 0.0f;
        const bool far = far_out(m, c);
        auto each = [&](auto &&f) {  // f(entry, its weight), of the lane's entries
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                float xs[EPV<T>], e[EPV<T>];
                unpack(raw[j], xs, T{});
                powers<T>(xs, m, c, far, e);
#pragma unroll
                for (int i = 0; i < EPV<T>; ++i) f(xs[i], e[i]);
            }
        };
        float S = 0.0f;
        uint32_t n = 0;
        {
            float xs[EPV<T>], e[EPV<T>];
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                unpack(raw[j], xs, T{});
                powers<T>(xs, m, c, far, e);
                S += sum_of(e);
#pragma unroll
                for (int i = 0; i < EPV<T>; ++i) n += xs[i] > -inf;
            }
        }
        S = warp_sum(S);
        n = __reduce_add_sync(0xffffffffu, n);
        const bool drawn = drawn_at_all(u);
        if (!(drawn && S > 0.0f && S < inf)) {
            const float v = !drawn ? 0.0f : S == 0.0f ? -inf : nan;
            if (lane == 0) put_sample(o, r, -1, v, v, 0);
            continue;
        }
        const float L = log_of(S, m, c);
        if constexpr (FEW) {
            // the best, one to a lane in order; their weights and all that follows from them in 64 bits
            const key_t64 key = warp_alternatives<T, NV>(raw, own, x, lane, s.top_k, s_cand[warp], &s_n[warp]);
            const uint32_t best = min(n, s.top_k);
            const bool in = lane < best;
            const float xk = in ? key_value(key) : 0.0f;
            const double w = in ? exp((double)q.scale * ((double)xk - (double)m)) : 0.0;
            double sum = w;
#pragma unroll
            for (int d = 1; d < 32; d *= 2) {
                const double v = __shfl_up_sync(0xffffffffu, sum, d);
                if (lane >= (uint32_t)d) sum += v;
            }
            uint32_t kept = best;
            if (s.top_p < 1.0) {
                const double need = s.top_p * __shfl_sync(0xffffffffu, sum, best - 1);
                kept = min(kept, (uint32_t)__ffs(__ballot_sync(0xffffffffu, in && sum >= need)));
            }
            if (s.min_p > 0.0) kept = min(kept, (uint32_t)__popc(__ballot_sync(0xffffffffu, in && w >= s.min_p)));
            const double T_all = __shfl_sync(0xffffffffu, sum, kept - 1), at = (double)u * T_all;
            // up to an entry, in the order of the numbers: a lane's entry is behind those of lower ones
            const uint32_t place = in && lane < kept ? key_place(key) : 0xFFFFFFFFu;
            double up = 0.0;
            for (uint32_t j = 0; j < kept; ++j) {
                const double v = __shfl_sync(0xffffffffu, w, j);
                if (__shfl_sync(0xffffffffu, place, j) <= place) up += v;
            }
            const bool has = lane < kept && w > 0.0;
            uint32_t tok = __reduce_min_sync(0xffffffffu, has && up > at ? place : 0xFFFFFFFFu);
            if (tok == 0xFFFFFFFFu) tok = __reduce_max_sync(0xffffffffu, has ? place : 0u);  // (rounding may leave the number behind the last one)
            if (place == tok) {
                const float lt = (float)log(T_all);
                put_sample(o, r, tok, log_ratio(xk, m, q.scale, L), log_ratio(xk, m, q.scale, lt), kept);
            }
        } else {
        // the cut: a key, and how many of the entries equal to it are kept; found by halves between values, in 32 bits
        const uint32_t most = ordered(m);
        uint32_t cut = LEAST_KEY - 1, ties = 0, there = 0;
        float among = S;
        bool sure = true;
        auto halve = [&](uint32_t lo, uint32_t hi) {  // between the values, so that it comes near to where they are
            const uint32_t mid = ordered(0.5f * from_ordered(max(lo, LEAST_KEY)) + 0.5f * from_ordered(hi - 1));
            return min(max(mid, lo + 1), hi - 1);
        };
        if (s.top_k && s.top_k < n) {
            uint32_t lo = LEAST_KEY - 1, hi = most + 1, above = 0, at_lo = n;
            while (hi - lo > 1) {
                const float mid = from_ordered(halve(lo, hi)), low = from_ordered(lo);
                uint32_t count = 0;
                float least = inf, below = -inf;
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    float xs[EPV<T>];
                    unpack(raw[j], xs, T{});
#pragma unroll
                    for (int i = 0; i < EPV<T>; ++i) {
                        if (xs[i] >= mid) { ++count; least = fminf(least, xs[i]); }
                        else if (xs[i] >= low) below = fmaxf(below, xs[i]);
                    }
                }
                count = __reduce_add_sync(0xffffffffu, count);
                if (count >= s.top_k) {
                    lo = __reduce_min_sync(0xffffffffu, ordered(least));
                    at_lo = count;
                } else {
                    above = count;
                    hi = __reduce_max_sync(0xffffffffu, ordered(below)) + 1;
                }
            }
            cut = lo;
            ties = s.top_k - above;
            there = at_lo - above;
            float sum = 0.0f, w = 0.0f;
            const float level = from_ordered(cut);
            each([&](float v, float e) {
                if (v > level) sum += e;
                else if (v == level) w = e;
            });
            among = warp_sum(sum) + (float)ties * __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(w)));
        }
        if (s.top_p < 1.0) {
            // Where the cut lies: weights in 32 runs of half a power of two below the largest one, added up by every lane for its own entries and by a
            // lane for each run.  What is in the run of the cut, if a warp can hold it, is put in order; else the halves begin from it.
            const float need = (float)s.top_p * among, margin = among * 0x1p-24f * ((float)(NV * EPV<T>) + 50.0f + POWER_ERROR * __log2f((float)q.V));  // (a lane's additions, the warp's, and the weights' errors)
            uint32_t lo = cut, hi = most + 1;
            float above = 0.0f;
            const float over = cut < LEAST_KEY ? -inf : from_ordered(cut);
            float *const runs = s_runs[FEW ? 0 : warp] + lane;
#pragma unroll
            for (uint32_t k = 0; k < 32; ++k) runs[FEW ? 0 : 32 * k] = 0.0f;
            auto run_of = [&](float v) { return (uint32_t)fminf((m - v) * c * 2.0f, 31.0f); };
            each([&](float v, float e) {
                if (v > over) runs[FEW ? 0 : 32 * run_of(v)] += e;
            });
            __syncwarp();
            float in_run = 0.0f;
#pragma unroll
            for (uint32_t k = 0; k < 32; ++k) in_run += s_runs[FEW ? 0 : warp][FEW ? 0 : 32 * lane + ((k + lane) & 31)];
            __syncwarp();
            float up_to = in_run;
#pragma unroll
            for (int d = 1; d < 32; d *= 2) {
                const float v = __shfl_up_sync(0xffffffffu, up_to, d);
                if (lane >= (uint32_t)d) up_to += v;
            }
            const uint32_t past = __ballot_sync(0xffffffffu, up_to >= need);
            bool listed = false;
            if (past) {
                const uint32_t run = __ffs(past) - 1;
                const float front = __shfl_up_sync(0xffffffffu, up_to, 1);
                above = __shfl_sync(0xffffffffu, lane ? front : 0.0f, run);
                float least = inf, largest = -inf;
                uint32_t mine = 0;
                each([&](float v, float) {
                    if (v > over && run_of(v) == run) {
                        ++mine;
                        least = fminf(least, v);
                        largest = fmaxf(largest, v);
                    }
                });
                const uint32_t all = __reduce_add_sync(0xffffffffu, mine);
                uint32_t place = mine;
#pragma unroll
                for (int d = 1; d < 32; d *= 2) {
                    const uint32_t v = __shfl_up_sync(0xffffffffu, place, d);
                    if (lane >= (uint32_t)d) place += v;
                }
                place -= mine;
                if (all <= 32) {
                    listed = true;
                    float *const list = s_runs[FEW ? 0 : warp];
                    if (mine)
                        each([&](float v, float) {
                            if (v > over && run_of(v) == run) list[FEW ? 0 : place++] = v;
                        });
                    __syncwarp();
                    // the values in falling order, a lane at each, and their weights
                    const bool there_is = lane < all;
                    uint32_t key = there_is ? ordered(list[FEW ? 0 : lane]) : 0u;
#pragma unroll
                    for (uint32_t k = 2; k <= 32; k *= 2)
#pragma unroll
                        for (uint32_t d = k / 2; d; d /= 2) {
                            const uint32_t other = __shfl_xor_sync(0xffffffffu, key, d);
                            key = ((lane & d) == 0) == ((lane & k) == 0) ? max(key, other) : min(key, other);
                        }
                    const float v = there_is ? from_ordered(key) : m;
                    float w[EPV<T>], vs[EPV<T>];
#pragma unroll
                    for (int i = 0; i < EPV<T>; ++i) vs[i] = v;
                    powers<T>(vs, m, c, far, w);
                    float sum = there_is ? w[0] : 0.0f;
#pragma unroll
                    for (int d = 1; d < 32; d *= 2) {
                        const float t = __shfl_up_sync(0xffffffffu, sum, d);
                        if (lane >= (uint32_t)d) sum += t;
                    }
                    const uint32_t enough = __ballot_sync(0xffffffffu, there_is && above + sum >= need);
                    // (rounding: then it is the next run's first, which 64 bits find)
                    const uint32_t at = enough ? __ffs(enough) - 1 : 0;
                    lo = enough ? __shfl_sync(0xffffffffu, key, at) : LEAST_KEY - 1;
                    const uint32_t higher = __popc(__ballot_sync(0xffffffffu, there_is && key > lo));
                    above += higher ? __shfl_sync(0xffffffffu, sum, (higher - 1) & 31) : 0.0f;
                    __syncwarp();
                } else {
                    lo = __reduce_min_sync(0xffffffffu, ordered(least));
                    hi = __reduce_max_sync(0xffffffffu, ordered(largest)) + 1;
                }
            }
            while (!listed && hi - lo > 1) {
                const float mid = from_ordered(halve(lo, hi)), low = from_ordered(lo);
                float sum = 0.0f, least = inf, below = -inf;
                each([&](float v, float e) {
                    if (v >= mid) { sum += e; least = fminf(least, v); }
                    else if (v > low) below = fmaxf(below, v);
                });
                sum = warp_sum(sum);
                if (sum >= need) {
                    lo = __reduce_min_sync(0xffffffffu, ordered(least));
                } else {
                    above = sum;
                    const uint32_t next = __reduce_max_sync(0xffffffffu, ordered(below));
                    hi = max(next, lo) + 1;
                }
            }
            if (lo < LEAST_KEY) {
                sure = false;
            } else {
                float w = 0.0f;
                uint32_t equal = 0;
                const float level = from_ordered(lo);
                each([&](float v, float e) {
                    if (v == level) { w = e; ++equal; }
                });
                w = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(w)));
                equal = __reduce_add_sync(0xffffffffu, equal);
                const float k = fmaxf(ceilf((need - above) / w), 1.0f);
                const uint32_t most_ties = lo == cut ? ties : equal;
                sure = w > 0.0f && k <= (float)most_ties && fmaf(k, w, above) >= need + margin && (k == 1.0f ? above : fmaf(k - 1.0f, w, above)) <= need - margin;
                cut = lo;
                ties = sure ? (uint32_t)k : 0;
                there = equal;
            }
        }
        Keep<NV> keep;
        const float least = fmaxf(__double2float_ru((double)m + s.drop), LOWEST);
        keep.level = cut < LEAST_KEY ? -inf : from_ordered(cut);
        keep.from = cut < LEAST_KEY ? LOWEST : ties == there ? keep.level : from_ordered(cut + 1);
        const bool some_ties = sure && ties < there && keep.level >= least && cut >= LEAST_KEY;
        keep.from = fmaxf(keep.from, least);
        int64_t token = -1;
        float x_tok = 0.0f, T_all = 0.0f;
        uint32_t kept = 0;
        if (sure) {
            if (some_ties) {  // the first of them, in the order of the numbers: vector by vector of each round
                uint32_t before = 0;
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    float xs[EPV<T>];
                    unpack(raw[j], xs, T{});
                    uint32_t mine = 0;
#pragma unroll
                    for (int i = 0; i < EPV<T>; ++i) mine += xs[i] == keep.level;
                    uint32_t incl = mine;
#pragma unroll
                    for (int d = 1; d < 32; d *= 2) {
                        const uint32_t v = __shfl_up_sync(0xffffffffu, incl, d);
                        if (lane >= (uint32_t)d) incl += v;
                    }
                    const uint32_t front = before + incl - mine;
                    keep.ties[j] = front < ties ? ties - front : 0u;
                    before += __shfl_sync(0xffffffffu, incl, 31);
                }
                sure = draw<T, 32, NV, true, true>(raw, keep, x, u, m, c, lane, true, &token, &x_tok, &S, &T_all, &kept);
            } else {
                sure = draw<T, 32, NV, true, false>(raw, keep, x, u, m, c, lane, true, &token, &x_tok, &S, &T_all, &kept);
            }
        }
        if (token >= 0) put_sample(o, r, token, log_ratio(x_tok, m, q.scale, L), log_ratio(x_tok, m, q.scale, log_of(T_all, m, c)), kept);
        if (!sure) sample_row_64<T, 32>(q, s, o, r, nullptr, nullptr, 1, 0, ordered(m), s.top_p < 1.0 ? cut : 0u);
        }
    }
}

// The vectors of a lane for rows of at most n vectors that a warp holds with top_k or top_p: 1,024 entries and some (a lane for every word of a
// mask); longer ones are read twice instead.  16-bit rows of 129 to 256 vectors, 5,000 rows of 1,500 bf16 logits in us, as long rows and by a warp with
// eight vectors a lane: with favourites top_p 0.9 50, 72, top_k 50 67, 166, top_k 8 26, 17; broad ones 629, 148 (and of 1,100 with top_k 50, which is more
// than the long rows' groups tell, 853, 156).  The warp's kernels would take the compiler 7 minutes a type for 4.
template <typename T, typename F>
bool warp_shape(uint32_t n, F &&f)
{
    using std::integral_constant;
    if (n <= 32) f(integral_constant<int, 1>{});
    else if (n <= 64) f(integral_constant<int, 2>{});
    else if (n <= 128) f(integral_constant<int, 4>{});
    else if constexpr (sizeof(T) == 4) {
        if (n > 256) return false;
        f(integral_constant<int, 8>{});
    } else {
        return false;
    }
    return true;
}

template <typename T, bool MASKED, bool ALIGNED>
bool launch_sample_short(const LogitRows &q, const SampleRules &s, const SampleOut &o, uint32_t n, cudaStream_t st)
{
    const bool order = s.top_k || s.top_p < 1.0;
    auto run = [&](auto g, auto v) {
        constexpr int G = decltype(g)::value, NV = decltype(v)::value;
        const uint64_t blocks = (q.n_rows + SHORT_WARPS * (32 / G) - 1) / (SHORT_WARPS * (32 / G));
        const uint32_t grid = (uint32_t)blocks;  // (2^31 blocks have more rows than there is memory)
        if (s.min_p > 0.0) k_sample_short<T, MASKED, ALIGNED, true, G, NV><<<grid, SHORT_WARPS * 32, 0, st>>>(q, s, o);
        else k_sample_short<T, MASKED, ALIGNED, false, G, NV><<<grid, SHORT_WARPS * 32, 0, st>>>(q, s, o);
        g_vl_launches.fetch_add(1);
    };
    auto run_warp = [&](auto v) {
        constexpr int NV = decltype(v)::value;
        const uint64_t blocks = (q.n_rows + SHORT_WARPS - 1) / SHORT_WARPS;
        const uint32_t grid = (uint32_t)(blocks < (1u << 30) ? blocks : (1u << 30));
        if (s.top_k && s.top_k <= 32) k_sample_warp<T, MASKED, ALIGNED, true, NV><<<grid, SHORT_WARPS * 32, 0, st>>>(q, s, o);
        else k_sample_warp<T, MASKED, ALIGNED, false, NV><<<grid, SHORT_WARPS * 32, 0, st>>>(q, s, o);
        g_vl_launches.fetch_add(1);
    };
    return order ? warp_shape<T>(n, run_warp) : short_shape<false, ALIGNED>(n, q.W, run);
}

template <typename T>
bool launch_sample_short(const LogitRows &q, const SampleRules &s, const SampleOut &o, cudaStream_t st)
{
    bool aligned;
    const uint32_t n = row_vectors(q, sizeof(T), &aligned);
    if (q.occupied || q.widths) return aligned ? launch_sample_short<T, true, true>(q, s, o, n, st) : launch_sample_short<T, true, false>(q, s, o, n, st);
    return aligned ? launch_sample_short<T, false, true>(q, s, o, n, st) : launch_sample_short<T, false, false>(q, s, o, n, st);
}

}  // namespace
