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
    double top_p, min_p, drop;  // drop: ln min_p / scale, minus infinity without min_p
    uint32_t *left;        // [n_rows] working memory: 0, or a row that one kernel leaves to another: the key of its largest logit, 1 if that is not known
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
// Whether the rows are short ones, and if so the launch.
bool vl_sample_short_f32(const LogitRows &q, const SampleRules &s, const SampleOut &o, cudaStream_t st);
bool vl_sample_short_f16(const LogitRows &q, const SampleRules &s, const SampleOut &o, cudaStream_t st);
bool vl_sample_short_bf16(const LogitRows &q, const SampleRules &s, const SampleOut &o, cudaStream_t st);

namespace {

namespace cg = cooperative_groups;

// A weight of 32 bits is within (4 + POWER_ERROR |y|) u of its value relatively, u = 2^-24, y its power of two: scale log2 e is a rounded
// product (u) with a rounded constant (0.22 u), a multiply-add makes y of it (u), and ln 2 times these 2.22 u is 1.54.
constexpr float POWER_ERROR = 1.6f;

constexpr uint32_t LEAST_KEY = 0x00800000u;  // of the lowest number; minus infinity lies below
constexpr uint32_t ZERO_KEY = 0x80000000u;   // of 0 (of both signs)

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
// row's vectors.  All threads hold the same results; every sum has one order.  A row of 131,072 bf16 logits of which 40,000 are kept takes four
// blocks 57 us, 14 without rules: ten passes of 2 to 5 us over shared memory, one of 11 with every weight in 64 bits, a barrier after each.
constexpr uint32_t TEAM_PARTS = 8, TEAM_HELD = 16;  // blocks; vectors of a thread that stay in shared memory
template <int NT>
struct TeamMemory {
    static constexpr uint32_t NW = NT / 32, ALL = NT == 32 ? 1 : TEAM_PARTS * NW;
    double d[2][ALL], second[ALL], table[EXP_TABLE];
    uint32_t u[2][ALL][3], best[NW], cut, listed;
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
                                           uint4 *held, uint32_t parts, uint32_t part, uint32_t known, uint32_t near = 0)
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
    // the first vectors of a lane are copied into its places of shared memory, if there are any, with what is closed taken out
    if (NT > 32) {
#pragma unroll 4
        for (uint32_t k = 0; k < TEAM_HELD; ++k)
            if (v0 + 32 * k < v1) held[k * NT + threadIdx.x] = vector(v0 + 32 * k + lane);
        if (threadIdx.x == 0) mem->listed = 0;
        __syncthreads();
    }
    auto each_vector = [&](auto &&f) {
#pragma unroll 1
        for (uint32_t w = v0, k = 0; w < v1; w += 32, ++k) f(NT > 32 && k < TEAM_HELD ? held[k * NT + threadIdx.x] : vector(w + lane));
    };
    auto each = [&](float from, auto &&f) {  // f(entry) of the possible entries of vectors that have one of at least `from`
        each_vector([&](const uint4 &raw) {
            if (!(vector_max(raw, T{}) >= from)) return;
            float e[EPV<T>];
            unpack(raw, e, T{});
#pragma unroll
            for (int i = 0; i < EPV<T>; ++i)
                if (e[i] > -inf) f(e[i]);
        });
    };
    // the largest and the smallest, how many there are (which is asked for with top_k), and whether something is no number (then the smallest is
    // 0); unless the largest is known, and with it that all are numbers
    uint32_t most = known, least = LEAST_KEY, n = 1;
    const bool leader = part == 0 && (NT == 32 ? lane == 0 : threadIdx.x == 0);
    if (rules.top_k || known < LEAST_KEY) {
        Three t{0u, 0xFFFFFFFFu, 0u};
        each_vector([&](const uint4 &raw) {
            float e[EPV<T>];
            unpack(raw, e, T{});
#pragma unroll
            for (int i = 0; i < EPV<T>; ++i) {
                const uint32_t key = e[i] < inf ? ordered(e[i]) : 0u;
                if (key >= LEAST_KEY) { t.most = max(t.most, key); ++t.sum; }
                if (key != LEAST_KEY - 1) t.least = min(t.least, key);
            }
        });
        t = team.three(t);
        n = t.sum;
        most = t.most;
        least = t.least;
        if (least == 0 || n == 0) {
            const float v = least == 0 ? __int_as_float(0x7fc00000) : -inf;
            if (leader) put_sample(o, r, -1, v, v, 0);
            return;
        }
    }
    const double M = (double)from_ordered(most), scale = (double)q.scale;
    auto weight = [&](float v) {
        const double z = scale * ((double)v - M);
        return NT == 32 ? exp(z) : exp_below_1(z, mem->table);
    };
    // sum over the entries that `in` takes, of vectors that have one of at least `from`
    auto add = [&](float from, auto &&in) {
        double sum = 0.0;
        each_vector([&](const uint4 &raw) {
            if (!(vector_max(raw, T{}) >= from)) return;
            float e[EPV<T>];
            unpack(raw, e, T{});
            double part[EPV<T>];
#pragma unroll
            for (int i = 0; i < EPV<T>; ++i) part[i] = weight(in(e[i]) ? e[i] : -inf);
#pragma unroll
            for (int k = EPV<T> / 2; k; k /= 2)
#pragma unroll
                for (int i = 0; i < k; ++i) part[i] += part[i + k];
            sum += part[0];
        });
        return sum;
    };

    // Sixteen sums of every thread's own, which lie behind the held vectors, over all threads: bin k, and the bins up to it, in lane k (and 0 and
    // all of them in the lanes from 16 on).  A warp of each block adds up a bin.
    auto bins_up = [&](auto type, double *v, double *up) {
        __syncthreads();
        const decltype(type) *const bin = reinterpret_cast<const decltype(type) *>(held + TEAM_HELD * NT) + (threadIdx.x >> 5) * NT + lane;
        double sum = 0.0;
#pragma unroll
        for (uint32_t k = 0; k < NT / 32; ++k) sum += (double)bin[32 * k];
#pragma unroll
        for (int k = 16; k; k >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, k);
        double *const d = mem->d[team.turn++ & 1];
        team.tell(d + warp, sum);
        team.meet();
        sum = 0.0;
        for (uint32_t p = 0; p < parts; ++p) sum += lane < 16 ? d[p * Team<NT>::NW + lane] : 0.0;
        *v = *up = sum;
#pragma unroll
        for (int k = 1; k < 32; k *= 2) {
            const double w = __shfl_up_sync(0xffffffffu, *up, k);
            if (lane >= (uint32_t)k) *up += w;
        }
    };

    // Among the keys lo .. hi: the largest whose entries, with those above up to hi and *above, have `need` of weight (or, counted, are as
    // many); lo - 1 if all of them do not.  *above becomes the weight of what is above it.  need(sum of all) is asked for once.
    auto search = [&](uint32_t lo, uint32_t hi, bool counted, double *above, auto &&need) -> uint32_t {
        const uint32_t none = lo - 1;
        double wanted = 0.0;
        if constexpr (NT == 32) {
            const double front = *above;
            auto reach = [&](uint32_t key) {  // the entries from a key on
                const float from = from_ordered(key), to = from_ordered(hi);
                if (!counted) return team.sum(add(from, [&](float v) { return v >= from && v <= to; }));
                uint32_t c = 0;
                each(from, [&](float v) { c += v >= from && v <= to; });
                return (double)__reduce_add_sync(0xffffffffu, c);
            };
            const double all = lo > hi ? 0.0 : reach(lo);
            wanted = need(all);
            if (front + all < wanted) { *above = front + all; return none; }
            uint32_t under = hi + 1;  // what its entries and those above reach is not enough
            while (under - lo > 1) {
                const uint32_t mid = lo + (under - lo) / 2;
                const double v = front + reach(mid);
                if (v >= wanted) lo = mid;
                else { under = mid; *above = v; }
            }
            return lo;
        } else {
            // sixteen runs of keys at a time, whose weights every thread adds up for its own entries, a warp of each block for all threads
            double *const own = reinterpret_cast<double *>(held + TEAM_HELD * NT) + threadIdx.x;
            bool asked = false;
            while (!asked || lo < hi) {
                const uint32_t span = hi - lo;
                const uint32_t shift = lo > hi || span < 16 ? 0 : 28 - __clz(span);
#pragma unroll
                for (uint32_t k = 0; k < 16; ++k) own[k * NT] = 0.0;
                const float from = from_ordered(lo);
                if (lo <= hi)
                    each_vector([&](const uint4 &raw) {
                        if (!(vector_max(raw, T{}) >= from)) return;
                        float e[EPV<T>];
                        unpack(raw, e, T{});
                        double w[EPV<T>];
                        uint32_t at[EPV<T>], nearest = 16;
#pragma unroll
                        for (int i = 0; i < EPV<T>; ++i) {
                            const uint32_t key = ordered(e[i]);
                            at[i] = key < lo || key > hi ? 16u : (hi - key) >> shift;
                            nearest = min(nearest, at[i]);
                        }
                        if (nearest == 16) return;
#pragma unroll
                        for (int i = 0; i < EPV<T>; ++i) w[i] = counted ? 1.0 : weight(e[i]);
#pragma unroll
                        for (int i = 0; i < EPV<T>; ++i)
                            if (at[i] < 16) own[at[i] * NT] += w[i];
                    });
                double v, up;
                bins_up(double{}, &v, &up);
                if (!asked) wanted = need(__shfl_sync(0xffffffffu, up, 31));
                const double prev = __shfl_up_sync(0xffffffffu, up, 1);
                const uint32_t past = __ballot_sync(0xffffffffu, lane < 16 && *above + up >= wanted), some = __ballot_sync(0xffffffffu, v > 0.0);
                if (!past && !asked) {
                    *above += __shfl_sync(0xffffffffu, up, 31);
                    return none;
                }
                asked = true;
                // (in a narrower run rounding may leave too little: then what is lowest in it)
                const uint32_t j = past ? __ffs(past) - 1 : 31 - __clz(some | 1u);
                *above += __shfl_sync(0xffffffffu, lane ? prev : 0.0, j);
                const uint32_t next_hi = hi - (j << shift), low = (1u << shift) - 1;
                lo = next_hi - lo > low ? next_hi - low : lo;
                hi = next_hi;
            }
            return lo;
        }
    };

    // kept: entries above the logit `level` (whose key is `cut`), and the first `ties` of those equal to it
    static_assert(NT == 32 || Team<NT>::NW == 16, "a warp for each of the sixteen runs");
    uint32_t cut = LEAST_KEY - 1, ties = 0;
    const bool all = !rules.top_k || rules.top_k >= n, shares = rules.top_p < 1.0;
    double S = 0.0, need = 0.0;  // sum over the row; what the kept entries have to reach
    if (!(all && shares) && (rules.top_k || rules.min_p > 0.0)) S = team.sum(add(-inf, [](float) { return true; }));
    if (!all) {
        double above = 0.0;
        cut = search(least, most, true, &above, [&](double) { return (double)rules.top_k; });
        ties = rules.top_k - (uint32_t)above;
    }
    const uint32_t first_cut = cut, first_ties = ties;
    // a lane's weight and entries above `upto`: what is worked out already of what is kept
    double high = 0.0;
    uint32_t high_count = 0;
    float upto = inf;
    if (shares) {
        auto needed = [&](double sum) {
            if (all) S = sum;
            else sum += (double)ties * weight(from_ordered(cut));
            return need = rules.top_p * sum;
        };
        double above = 0.0;
        if (NT == 32 && near > cut) {
            // 32 bits have found a key that the cut is at or next to: looked at as it is, and from neighbour to neighbour
            const uint32_t none = all ? LEAST_KEY - 1 : cut;
            double sum = team.sum(add(-inf, [&](float v) { return ordered(v) > none; }));
            const double wanted = needed(sum);
            uint32_t at = near;
            bool found = false;
            for (int tries = 0; tries < 8 && !found; ++tries) {
                const float here = from_ordered(at);
                double over = team.sum(add(here, [&](float v) { return v > here; })), with = over;
                Three t{0u, 0xFFFFFFFFu, 0u};  // entries equal to it, the next key above and below
                each(-inf, [&](float v) {
                    const uint32_t key = ordered(v);
                    t.sum += key == at;
                    if (key > at) t.least = min(t.least, key);
                    if (key < at && key > none) t.most = max(t.most, key);
                });
                t = team.three(t);
                with += (double)t.sum * weight(here);
                if (over >= wanted && t.least != 0xFFFFFFFFu) at = t.least;
                else if (with < wanted && t.most) at = t.most;
                else found = true;
                if (found) cut = with >= wanted ? at : none;
            }
            if (!found) cut = search(all ? least : cut + 1, most, false, &above, [&](double) { return wanted; });
        } else if (NT == 32 || !all) {
            cut = search(all ? least : cut + 1, most, false, &above, needed);
        } else {
            // Where the cut lies as far as 32 bits tell it: the logits in 2^28 steps below the largest one, sixteen runs of steps at a time.  A sum of
            // 32-bit terms is within NARROW of its value: (4 + 1.6 |y|) u of a weight, |y| up to 40 for what is not nothing, a thread's
            // additions to a bin (TEAM_HELD vectors; longer rows are not narrowed down).
            constexpr double NARROW = 2e-5;
            constexpr uint32_t LISTED = NT;  // entries that are looked at one by one
            const float M32 = from_ordered(most), c = q.scale * LOG2E;
            const float per = 0x1p28f / fmaxf(fminf(M32 - from_ordered(least), 64.0f / q.scale), 1e-30f);
            auto step_of = [&](float v) { return (uint32_t)fminf((M32 - v) * per, 0x0.ffffffp28f); };
            uint32_t lo = 0, hi = (1u << 28) - 1;
            float *const own = reinterpret_cast<float *>(held + TEAM_HELD * NT) + threadIdx.x;
            double front = 0.0, wanted = 0.0, slack = 0.0;
            for (uint32_t shift = 24; x.n <= warps * 32 * TEAM_HELD;) {
#pragma unroll
                for (uint32_t k = 0; k < 16; ++k) own[k * NT] = 0.0f;
                each_vector([&](const uint4 &raw) {
                    float e[EPV<T>];
                    unpack(raw, e, T{});
#pragma unroll
                    for (int i = 0; i < EPV<T>; ++i) {
                        const uint32_t t = step_of(e[i]), at = (t - lo) >> shift;
                        if (t >= lo && t <= hi && e[i] > -inf) own[at * NT] += ex2((e[i] - M32) * c);
                    }
                });
                double v, up;
                bins_up(float{}, &v, &up);
                if (shift == 24) {
                    const double sum = __shfl_sync(0xffffffffu, up, 31);
                    wanted = rules.top_p * sum;
                    slack = NARROW * sum;
                }
                const double prev = __shfl_up_sync(0xffffffffu, up, 1);
                const uint32_t perhaps = __ballot_sync(0xffffffffu, lane < 16 && front + up + slack >= wanted);
                const uint32_t sure = __ballot_sync(0xffffffffu, lane < 16 && front + up - slack >= wanted);
                const uint32_t a = perhaps ? __ffs(perhaps) - 1 : 15, b = sure ? __ffs(sure) - 1 : 15;
                front += __shfl_sync(0xffffffffu, lane ? prev : 0.0, a);
                hi = min(hi, lo + ((b + 1) << shift) - 1);
                lo += a << shift;
                // (four times: what is left is one logit of 16 bits, or some dozen of 32)
                if (shift <= 12 || b - a > 3) break;
                shift = 28 - __clz(hi - lo);
            }
            __syncthreads();  // (the last sums have been read)
            // in 64 bits: the whole sum, and what is above these steps; and which keys lie in them, with a list of the first ones of each block
            uint32_t *const list_keys = reinterpret_cast<uint32_t *>(held + TEAM_HELD * NT);
            static_assert(4 * LISTED * 4 + 2 * LISTED * 8 <= 16 * NT * 8, "fits the runs' sums");
            // (the order in which entries are listed is any: their weights, at most 1, are added up as whole numbers of 2^-54, LISTED of which are below
            // 2^64, so that it makes no difference; what that leaves out is below 2^-45, next to sums of 1 and more.  By their order instead, as 64-bit
            // numbers: 165 us for 157, 1,024 rows of 131,072 bf16 logits with top_p 0.95)
            unsigned long long *const list_weights = reinterpret_cast<unsigned long long *>(list_keys + 4 * LISTED);
            double sum = 0.0;
            Three t{0u, 0xFFFFFFFFu, 0u};
            each_vector([&](const uint4 &raw) {
                float e[EPV<T>];
                unpack(raw, e, T{});
                double w[EPV<T>];
#pragma unroll
                for (int i = 0; i < EPV<T>; ++i) w[i] = weight(e[i]);
#pragma unroll
                for (int i = 0; i < EPV<T>; ++i) {
                    const uint32_t at = step_of(e[i]), key = ordered(e[i]);
                    sum += w[i];
                    if (at < lo) { high += w[i]; ++high_count; }
                    if (at >= lo && at <= hi && e[i] > -inf) {
                        ++t.sum;
                        t.least = min(t.least, key);
                        t.most = max(t.most, key);
                        const uint32_t place = atomicAdd(&mem->listed, 1u);
                        if (place < LISTED) {
                            list_keys[place] = key;
                            list_weights[place] = __double2ull_rn(w[i] * 0x1p54);
                        }
                    }
                }
            });
            // (all at once: three numbers of a warp, two sums)
            double above_own = high;
#pragma unroll
            for (int k = 16; k; k >>= 1) {
                sum += __shfl_xor_sync(0xffffffffu, sum, k);
                above_own += __shfl_xor_sync(0xffffffffu, above_own, k);
            }
            t = Team<NT>::of_warp(t);
            double *const d0 = mem->d[team.turn & 1];
            uint32_t(*const u0)[3] = mem->u[team.turn++ & 1];
            team.tell(d0 + warp, sum);
            team.tell(mem->second + warp, above_own);
            team.tell(&u0[warp][0], t.sum);
            team.tell(&u0[warp][1], t.least);
            team.tell(&u0[warp][2], t.most);
            team.meet();
            t = Three{0u, 0xFFFFFFFFu, 0u};
            S = above = 0.0;
            for (uint32_t w = lane; w < warps; w += 32) {
                S += d0[w];
                above += mem->second[w];
                t.sum += u0[w][0];
                t.least = min(t.least, u0[w][1]);
                t.most = max(t.most, u0[w][2]);
            }
#pragma unroll
            for (int k = 16; k; k >>= 1) {
                S += __shfl_xor_sync(0xffffffffu, S, k);
                above += __shfl_xor_sync(0xffffffffu, above, k);
            }
            t = Team<NT>::of_warp(t);
            need = rules.top_p * S;
            auto same = [&](double) { return need; };
            cut = 0;
            if (above < need && t.most) {
                upto = from_ordered(t.most);
                if (t.least == t.most) {
                    cut = t.least;
                } else if (t.sum <= LISTED) {  // the first block looks at all of them
                    if (part == 0) {
                        uint32_t *const all_keys = list_keys + 2 * LISTED;
                        unsigned long long *const all_weights = list_weights + LISTED;
                        uint32_t front = 0;
                        for (uint32_t p = 0; p < parts; ++p) {
                            const uint32_t m = *cg::this_cluster().map_shared_rank(&mem->listed, p);
                            if (threadIdx.x < m) {
                                all_keys[front + threadIdx.x] = cg::this_cluster().map_shared_rank(list_keys, p)[threadIdx.x];
                                all_weights[front + threadIdx.x] = cg::this_cluster().map_shared_rank(list_weights, p)[threadIdx.x];
                            }
                            front += m;
                        }
                        __syncthreads();
                        uint32_t best = 0;
                        if (threadIdx.x < t.sum) {
                            const uint32_t key = all_keys[threadIdx.x];
                            unsigned long long up = 0;
                            for (uint32_t j = 0; j < t.sum; ++j) up += all_keys[j] >= key ? all_weights[j] : 0ull;
                            if (above + (double)up * 0x1p-54 >= need) best = key;
                        }
                        best = __reduce_max_sync(0xffffffffu, best);
                        if (lane == 0) mem->best[threadIdx.x >> 5] = best;
                        __syncthreads();
                        best = __reduce_max_sync(0xffffffffu, lane < Team<NT>::NW ? mem->best[lane] : 0u);
                        if (threadIdx.x < parts) *cg::this_cluster().map_shared_rank(&mem->cut, threadIdx.x) = best;
                    }
                    team.meet();
                    cut = mem->cut;
                }
                if (cut == 0) {
                    cut = search(t.least, t.most, false, &above, same);
                    if (cut < t.least) cut = t.least > least ? search(least, t.least - 1, false, &above, same) : LEAST_KEY - 1;
                }
            } else {  // (the margin makes this an error of rounding at most)
                above = 0.0;
                high = 0.0;
                high_count = 0;
                cut = search(least, most, false, &above, same);
            }
        }
        if (all && cut < least) cut = LEAST_KEY - 1;
    }

    // what the warps' runs hold above the cut and of ties; a run's ties are kept as far as there are some left
    double sum = 0.0, total = 0.0, base = 0.0, tie = 0.0;
    uint32_t count = 0, equal = 0, kept = 0, before = 0, mine = warp;
    float level = -inf;
    double *d = nullptr;
    uint32_t(*su)[3] = nullptr;
    auto runs = [&](auto &&f) {  // f(first run, kept weight of a lane's run, of the runs up to it, ties in front of it, entries above the cut)
        uint32_t front = 0;
        for (uint32_t w0 = 0; w0 < warps; w0 += 32) {
            const bool there = w0 + lane < warps;
            const uint32_t e = there ? su[w0 + lane][1] : 0u;
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
            f(w0, own, incl, b, there ? su[w0 + lane][0] : 0u);
        }
        return front;
    };
    // min_p keeps the logits from `lowest` on: where the cut is lower, these alone decide
    const uint32_t lowest = ordered(fmaxf(__double2float_ru(M + rules.drop), LOWEST));
    const bool by_min = rules.min_p > 0.0 && cut < lowest;
    if (by_min) {
        // (the key below that of 0 is the one of -0, which no entry has and which as a logit is equal to 0)
        cut = lowest - (lowest == ZERO_KEY ? 2 : 1);
        ties = 0;
        high = 0.0;
        high_count = 0;
        upto = inf;
    }
    {
        level = cut < LEAST_KEY ? -inf : from_ordered(cut);
        sum = high;
        count = high_count;
        equal = 0;
        each_vector([&](const uint4 &raw) {
            float e[EPV<T>];
            unpack(raw, e, T{});
            uint32_t in = 0;
#pragma unroll
            for (int i = 0; i < EPV<T>; ++i) {
                in += e[i] > level && e[i] <= upto;
                equal += e[i] == level && level > -inf;
            }
            count += in;
            if (!in) return;
            double part[EPV<T>];
#pragma unroll
            for (int i = 0; i < EPV<T>; ++i) part[i] = weight(e[i] > level && e[i] <= upto ? e[i] : -inf);
#pragma unroll
            for (int k = EPV<T> / 2; k; k /= 2)
#pragma unroll
                for (int i = 0; i < k; ++i) part[i] += part[i + k];
            sum += part[0];
        });
#pragma unroll
        for (int k = 16; k; k >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, k);
        count = __reduce_add_sync(0xffffffffu, count);
        equal = __reduce_add_sync(0xffffffffu, equal);
        double above = sum;
        uint32_t there = equal;
        tie = 0.0;
        if (NT > 32) {
            d = mem->d[team.turn & 1];
            su = mem->u[team.turn++ & 1];
            team.tell(d + warp, sum);
            team.tell(&su[warp][0], count);
            team.tell(&su[warp][1], equal);
            team.meet();
            above = 0.0;
            there = runs([&](uint32_t, double, double incl, uint32_t, uint32_t) { above += __shfl_sync(0xffffffffu, incl, 31); });
        }
        const double w = level > -inf ? weight(level) : 0.0;
        if (shares && level > -inf && !by_min) {
            const uint32_t most_ties = cut == first_cut ? first_ties : there;
            const double m = w > 0.0 ? ceil((need - above) / w) : 1.0;
            ties = (uint32_t)min(max(m, 1.0), (double)most_ties);
        }
        tie = ties ? w : 0.0;
    }
    if (NT == 32) {
        total = sum + (double)min(equal, ties) * tie;
        kept = count + min(equal, ties);
    } else {
        const uint32_t there = runs([&](uint32_t, double, double incl, uint32_t, uint32_t n) {
            total += __shfl_sync(0xffffffffu, incl, 31);
            kept += __reduce_add_sync(0xffffffffu, n);
        });
        kept += min(there, ties);
        // the run that the number falls into: the first up to whose end the sum is above it, or the last with something kept
        const double at = (double)rules.uniform[r] * total;
        double up = 0.0;
        mine = 0;
        bool hit = false;
        runs([&](uint32_t w0, double own, double incl, uint32_t b, uint32_t) {
            const uint32_t some = __ballot_sync(0xffffffffu, own > 0.0), past = __ballot_sync(0xffffffffu, own > 0.0 && up + incl > at);
            const double in_front = __shfl_up_sync(0xffffffffu, incl, 1);
            if (!hit && some) {
                const uint32_t f = past ? __ffs(past) - 1 : 31 - __clz(some);
                mine = w0 + f;
                base = up + __shfl_sync(0xffffffffu, lane ? in_front : 0.0, f);
                before = __shfl_sync(0xffffffffu, b, f);
                hit = past != 0;
            }
            up += __shfl_sync(0xffffffffu, incl, 31);
        });
    }
    if (!(rules.top_k || rules.top_p < 1.0 || rules.min_p > 0.0)) S = total;
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
    if (lane == 0 && token == 0xFFFFFFFFu) {  // (the largest entry is always kept: no weight at all is an error, told as what is no number)
        const float nan = __int_as_float(0x7fc00000);
        put_sample(o, r, -1, nan, nan, 0);
    } else if (lane == 0) {
        const double z = scale * ((double)to_f32(x.row[token]) - M);
        put_sample(o, r, token, (float)(z - log(S)), (float)(z - log(total)), kept);
    }
}

}  // namespace
