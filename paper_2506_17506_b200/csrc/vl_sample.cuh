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
#include <cooperative_groups.h>

#include "vl_rank.cuh"

struct SampleRules {
    const float *uniform;  // [n_rows]
    uint32_t top_k;        // 0: all
    double top_p, min_p;
    uint8_t *left;         // [n_rows] working memory: rows that one kernel leaves to another
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

namespace cg = cooperative_groups;

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

template <typename T, bool MASKED>
__device__ __forceinline__ uint4 open_vector(const RowVectors<T> &x, const RowMask &mask, uint32_t v)
{
    uint4 raw = x.whole(v) ? *x.at(v) : x.part(v);
    if (MASKED) close_entries<T>(raw, mask.closed_from(x.first(v), EPV<T>));
    return raw;
}

// ---- in 64 bits
// exp z for z <= 0 after P. T. P. Tang, "Table-driven implementation of the exponential function", 1989: z = (64 k + j) ln 2 / 64 + r,
// 2^(j / 64) from a table, and a series for e^r - 1, |r| <= ln 2 / 128 (what it leaves out is below 2^-54).  Twelve operations of 64 bits for the
// library function's thirty; below e^-700, which no sum here holds, 0.
constexpr double LN2_64 = 0.693147180559945309417232121458;
constexpr uint32_t EXP_TABLE = 64;
__device__ __forceinline__ double exp_below_1(double z, const double *table)
{
    const double t = fma(z, (double)EXP_TABLE / LN2_64, 6755399441055744.0);  // rounds to a whole number: its low word
    const int n = __double2loint(t);
    const double r = fma(t - 6755399441055744.0, -LN2_64 / (double)EXP_TABLE, z);
    double p = fma(r, 1.0 / 120.0, 1.0 / 24.0);
    p = fma(p, r, 1.0 / 6.0);
    p = fma(p, r, 0.5);
    p = fma(p * r, r, r);
    const double v = table[n & (EXP_TABLE - 1)], w = fma(v, p, v);
    return z < -700.0 ? 0.0 : __hiloint2double(__double2hiint(w) + ((n >> 6) << 20), __double2loint(w));
}

// The threads at a row that they read as often as they need it: a warp (NT = 32), or `parts` blocks of a cluster.  Each warp has a run of the
// row's vectors.  All threads hold the same results; every sum has one order.
constexpr uint32_t TEAM_PARTS = 8;
template <int NT>
struct TeamMemory {
    static constexpr uint32_t NW = NT / 32, ALL = NT == 32 ? 1 : TEAM_PARTS * NW;
    double d[2][ALL], table[EXP_TABLE];
    uint32_t u[2][ALL][3];
};
template <int NT>
struct Team {
    static constexpr uint32_t NW = NT / 32;
    TeamMemory<NT> *mem;
    uint32_t parts, part, turn;
    __device__ __forceinline__ uint32_t lane() const { return threadIdx.x & 31; }
    __device__ __forceinline__ uint32_t warps() const { return NT == 32 ? 1 : parts * NW; }
    __device__ __forceinline__ uint32_t warp() const { return NT == 32 ? 0 : part * NW + (threadIdx.x >> 5); }
    __device__ __forceinline__ void meet()
    {
        if (NT == 32) return;
        if (parts > 1) cg::this_cluster().sync();
        else __syncthreads();
    }
    // A number of each warp's, in every block's memory.  (What is there from two calls ago has been read before the barrier of the last one.)
    template <typename V>
    __device__ __forceinline__ void tell(V *at, V v)
    {
        if (parts > 1) {
            if (lane() < parts) *cg::this_cluster().map_shared_rank(at, lane()) = v;
        } else if (lane() == 0) {
            *at = v;
        }
    }
    __device__ __forceinline__ double sum(double v)
    {
#pragma unroll
        for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
        if (NT == 32) return v;
        double *s = mem->d[turn++ & 1];
        tell(s + warp(), v);
        meet();
        v = 0.0;
        for (uint32_t w = lane(); w < warps(); w += 32) v += s[w];
#pragma unroll
        for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
        return v;
    }
    struct Three {
        uint32_t sum, least, most;
    };
    __device__ __forceinline__ static Three of_warp(Three v)
    {
        return {__reduce_add_sync(0xffffffffu, v.sum), __reduce_min_sync(0xffffffffu, v.least), __reduce_max_sync(0xffffffffu, v.most)};
    }
    __device__ __forceinline__ Three three(Three v)
    {
        v = of_warp(v);
        if (NT == 32) return v;
        auto s = mem->u[turn++ & 1];
        tell(&s[warp()][0], v.sum);
        tell(&s[warp()][1], v.least);
        tell(&s[warp()][2], v.most);
        meet();
        v = Three{0u, 0xFFFFFFFFu, 0u};
        for (uint32_t w = lane(); w < warps(); w += 32) {
            v.sum += s[w][0];
            v.least = min(v.least, s[w][1]);
            v.most = max(v.most, s[w][2]);
        }
        return of_warp(v);
    }
};

template <typename T, int NT>
__device__ __noinline__ void sample_row_64(const LogitRows &q, const SampleRules &rules, const SampleOut &o, uint64_t r, TeamMemory<NT> *mem,
                                           uint32_t parts, uint32_t part)
{
    Team<NT> team{mem, parts, part, 0};
    typedef typename Team<NT>::Three Three;
    const uint32_t lane = team.lane(), warp = team.warp(), warps = team.warps();
    const float inf = __int_as_float(0x7f800000);
    const RowVectors<T> x(static_cast<const T *>(q.x) + r * q.stride, q.V);
    const RowMask mask = row_mask(q, r);
    const bool masked = mask.any();
    const uint32_t per = (x.n + warps - 1) / warps, v0 = min(x.n, warp * per), v1 = min(x.n, v0 + per);
    auto vector = [&](uint32_t v) {  // minus infinity behind the run
        if (v >= v1) return make_uint4(MINUS_INF2<T>, MINUS_INF2<T>, MINUS_INF2<T>, MINUS_INF2<T>);
        return masked ? open_vector<T, true>(x, mask, v) : open_vector<T, false>(x, mask, v);
    };
    auto each = [&](float from, auto &&f) {  // f(entry, number) of the possible entries of vectors that have one of at least `from`
        for (uint32_t w = v0; w < v1; w += 64) {  // two at a time: the second one's load does not wait for the first one's work
            const uint4 raw[2] = {vector(w + lane), vector(w + 32 + lane)};
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                if (!(vector_max(raw[k], T{}) >= from)) continue;
                float e[EPV<T>];
                unpack(raw[k], e, T{});
#pragma unroll
                for (int i = 0; i < EPV<T>; ++i)
                    if (e[i] > -inf) f(e[i], x.first(w + 32 * k + lane) + i);
            }
        }
    };
    // the largest, how many there are, and whether something is no number
    uint32_t most = 0, bad = 0, n = 0;
    for (uint32_t w = v0; w < v1; w += 32) {
        float e[EPV<T>];
        unpack(vector(w + lane), e, T{});
#pragma unroll
        for (int i = 0; i < EPV<T>; ++i) {
            if (!(e[i] < inf)) bad = 1;
            if (e[i] > -inf) { most = max(most, ordered(e[i])); ++n; }
        }
    }
    const Three first = team.three({n, bad ? 0u : 1u, most});
    n = first.sum;
    most = first.most;
    const bool leader = part == 0 && (NT == 32 ? lane == 0 : threadIdx.x == 0);
    if (first.least == 0 || n == 0) {
        const float v = first.least == 0 ? __int_as_float(0x7fc00000) : -inf;
        if (leader) put_sample(o, r, -1, v, v, 0);
        return;
    }
    const double M = (double)from_ordered(most), scale = (double)q.scale;
    auto weight = [&](float v) {
        const double z = scale * ((double)v - M);
        return NT == 32 ? exp(z) : exp_below_1(z, mem->table);
    };

    // all of them
    double S = 0.0;
    each(-inf, [&](float v, int) { S += weight(v); });
    S = team.sum(S);

    // kept: entries whose key is above `cut`, and the first `ties` of those equal to it
    uint32_t cut = LEAST_KEY - 1, ties = 0;
    double among = S;  // sum over these
    auto halve = [&](uint32_t lo, uint32_t hi) {  // between the values, so that it comes near to where they are
        const uint32_t mid = ordered(0.5f * from_ordered(max(lo, LEAST_KEY)) + 0.5f * from_ordered(hi - 1));
        return min(max(mid, lo + 1), hi - 1);
    };
    if (rules.top_k && rules.top_k < n) {
        // the largest key that top_k entries reach: at least lo, below hi, which `above` entries reach
        uint32_t lo = LEAST_KEY - 1, hi = most + 1, above = 0;
        while (hi - lo > 1) {
            const uint32_t mid = halve(lo, hi);
            const float at_lo = from_ordered(max(lo, LEAST_KEY)), at_mid = from_ordered(mid), at_hi = from_ordered(hi - 1);
            Three t{0u, 0xFFFFFFFFu, 0u};
            each(at_lo, [&](float v, int) {
                if (v > at_hi || v < at_lo) return;
                if (v >= at_mid) { ++t.sum; t.least = min(t.least, ordered(v)); }
                else t.most = max(t.most, ordered(v));
            });
            t = team.three(t);
            if (above + t.sum >= rules.top_k) {
                lo = t.least;
            } else {
                above += t.sum;
                hi = max(t.most, lo) + 1;
            }
        }
        cut = lo;
        ties = rules.top_k - above;
        const float level = from_ordered(cut);
        double sum = 0.0;
        each(level, [&](float v, int) { if (v > level) sum += weight(v); });
        among = team.sum(sum) + (double)ties * weight(level);
    }
    if (rules.top_p < 1.0) {
        const double need = rules.top_p * among;
        uint32_t lo = cut, hi = most + 1;
        double above = 0.0;  // sum of what is above hi
        while (hi - lo > 1) {
            const uint32_t mid = halve(lo, hi);
            const float at_lo = from_ordered(lo), at_mid = from_ordered(mid), at_hi = from_ordered(hi - 1);
            Three t{0u, 0xFFFFFFFFu, 0u};
            double sum = 0.0;
            each(at_lo, [&](float v, int) {
                if (v > at_hi || v <= at_lo) return;
                if (v >= at_mid) { sum += weight(v); t.least = min(t.least, ordered(v)); }
                else t.most = max(t.most, ordered(v));
            });
            sum = above + team.sum(sum);
            t = team.three(t);
            if (sum >= need && t.least != 0xFFFFFFFFu) {
                lo = t.least;
            } else {
                above = sum;
                hi = max(t.most, lo) + 1;
            }
        }
        // (lo is an entry's key, or the cut that was there)
        const float level = from_ordered(lo);
        Three t{0u, 0u, 0u};
        if (lo != cut) each(level, [&](float v, int) { t.sum += v == level; });
        const uint32_t there = lo == cut ? ties : team.three(t).sum;
        const double w = lo < LEAST_KEY ? 0.0 : weight(level);
        const double m = w > 0.0 ? ceil((need - above) / w) : 1.0;
        ties = lo == cut && ties == 0 ? 0 : (uint32_t)min(max(m, 1.0), (double)there);
        cut = lo;
    }
    if (rules.min_p > 0.0 && (cut < LEAST_KEY || weight(from_ordered(cut)) < rules.min_p)) {
        uint32_t lo = max(cut, LEAST_KEY - 1), hi = most;  // the lowest key whose weight is enough: above lo, at most hi
        while (hi - lo > 1) {
            const uint32_t mid = lo + (hi - lo) / 2;
            if (exp(scale * ((double)from_ordered(mid) - M)) >= rules.min_p) hi = mid;
            else lo = mid;
        }
        cut = hi - 1;
        ties = 0;
    }

    // what the warps' runs hold of them; a run's ties are kept as far as there are some left
    const float level = cut < LEAST_KEY ? -inf : from_ordered(cut);
    double sum = 0.0;
    uint32_t count = 0, equal = 0;
    each(level, [&](float v, int) {
        if (v > level) { sum += weight(v); ++count; }
        equal += v == level;
    });
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    count = __reduce_add_sync(0xffffffffu, count);
    equal = __reduce_add_sync(0xffffffffu, equal);
    const double tie = ties ? weight(level) : 0.0;
    double total = sum + (double)min(equal, ties) * tie, base = 0.0;
    uint32_t before = 0, kept = count + min(equal, ties), mine = warp;
    if (NT > 32) {
        double *d = mem->d[team.turn & 1];
        auto s = mem->u[team.turn++ & 1];
        team.tell(d + warp, sum);
        team.tell(&s[warp][0], count);
        team.tell(&s[warp][1], equal);
        team.meet();
        // a lane at a run: its kept weight, with the ties in front of it
        total = 0.0;
        kept = 0;
        uint32_t front = 0;
        double at = 0.0;
        auto runs = [&](auto &&f) {  // f(weight of 32 runs' kept entries, ties in front of each)
            front = 0;
            for (uint32_t w0 = 0; w0 < warps; w0 += 32) {
                const bool there = w0 + lane < warps;
                const uint32_t e = there ? s[w0 + lane][1] : 0u;
                uint32_t up = e;
#pragma unroll
                for (int k = 1; k < 32; k *= 2) {
                    const uint32_t v = __shfl_up_sync(0xffffffffu, up, k);
                    if (lane >= (uint32_t)k) up += v;
                }
                const uint32_t b = front + up - e;
                front += __shfl_sync(0xffffffffu, up, 31);
                const double own = there ? d[w0 + lane] + (double)min(e, ties - min(ties, b)) * tie : 0.0;
                double incl = own;
#pragma unroll
                for (int k = 1; k < 32; k *= 2) {
                    const double v = __shfl_up_sync(0xffffffffu, incl, k);
                    if (lane >= (uint32_t)k) incl += v;
                }
                f(w0, own, incl, b, there ? s[w0 + lane][0] : 0u);
            }
        };
        runs([&](uint32_t, double, double incl, uint32_t, uint32_t c) {
            total += __shfl_sync(0xffffffffu, incl, 31);
            kept += __reduce_add_sync(0xffffffffu, c);
        });
        kept += min(front, ties);
        // the run that the number falls into: the first up to whose end the sum is above it, or the last with something kept
        at = (double)rules.uniform[r] * total;
        double up = 0.0;
        mine = 0xFFFFFFFFu;
        bool hit = false;
        runs([&](uint32_t w0, double own, double incl, uint32_t b, uint32_t) {
            const uint32_t some = __ballot_sync(0xffffffffu, own > 0.0), past = __ballot_sync(0xffffffffu, own > 0.0 && up + incl > at);
            if (!hit && some) {
                const uint32_t f = past ? __ffs(past) - 1 : 31 - __clz(some);
                const double in_front = __shfl_up_sync(0xffffffffu, incl, 1);
                mine = w0 + f;
                base = up + __shfl_sync(0xffffffffu, lane ? in_front : 0.0, f);
                before = __shfl_sync(0xffffffffu, b, f);
                hit = past != 0;
            }
            up += __shfl_sync(0xffffffffu, incl, 31);
        });
    }
    if (warp != mine) return;
    const double at = (double)rules.uniform[r] * total;
    uint32_t token = 0xFFFFFFFFu;
    for (uint32_t w = v0; w < v1; w += 32) {
        float e[EPV<T>];
        unpack(vector(w + lane), e, T{});
        // the lane's kept entries: ties by their number, lanes in order
        uint32_t same = 0;
#pragma unroll
        for (int i = 0; i < EPV<T>; ++i) same += e[i] == level && level > -inf;
        uint32_t incl = same;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const uint32_t v = __shfl_up_sync(0xffffffffu, incl, d);
            if (lane >= (uint32_t)d) incl += v;
        }
        uint32_t rank = before + incl - same;
        before += __shfl_sync(0xffffffffu, incl, 31);
        double own = 0.0, ws[EPV<T>];
#pragma unroll
        for (int i = 0; i < EPV<T>; ++i) {
            bool in = e[i] > level;
            if (e[i] == level && level > -inf) in = rank++ < ties;
            ws[i] = in ? weight(e[i]) : 0.0;
            own += ws[i];
        }
        double up = own;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const double v = __shfl_up_sync(0xffffffffu, up, d);
            if (lane >= (uint32_t)d) up += v;
        }
        const double prev = __shfl_up_sync(0xffffffffu, up, 1);
        const uint32_t some = __ballot_sync(0xffffffffu, own > 0.0), past = __ballot_sync(0xffffffffu, own > 0.0 && base + up > at);
        if (some) {
            // the entry in that lane's vector, or (rounding may leave the number behind the last one) the last kept one so far
            const uint32_t f = past ? __ffs(past) - 1 : 31 - __clz(some);
            uint32_t place = 0;
            double cum = base + (lane ? prev : 0.0);
            bool open = true;
#pragma unroll
            for (int i = 0; i < EPV<T>; ++i) {
                cum += ws[i];
                if (ws[i] > 0.0 && open) {
                    place = (uint32_t)(x.first(w + lane) + i);
                    open = !(cum > at);
                }
            }
            token = __shfl_sync(0xffffffffu, place, f);
        }
        base += __shfl_sync(0xffffffffu, up, 31);
        if (past) break;
    }
    if (lane == 0) {
        const double z = scale * ((double)to_f32(x.row[token]) - M);
        put_sample(o, r, token, (float)(z - log(S)), (float)(z - log(total)), kept);
    }
}

}  // namespace
