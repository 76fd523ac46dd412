// Log probabilities of given tokens, entropy and best alternatives of rows of logits: how likely the model behind the candidates found
// them (the factorisation of Section 3.1), under the masks of vl_occupied_masks where it decodes around occupied registers
// (Section 4.5).
//
// With z = scale x over the open entries, M = max x, d_i = x_i - M, e_i = exp(scale d_i):
//   L = ln sum e_i,   log p_i = scale d_i - L,   entropy = L - scale (sum e_i d_i) / (sum e_i)
// Both terms of the entropy are non-negative, so nothing cancels, and M apart from L keeps digits where the logits are far from zero.
// One pass: a thread holds the largest logit so far and the two sums in 32 bits, and scales the sums when the largest one rises.
//
// What bounds it: reading the logits once; per element also one exponential (16 a clock and multiprocessor: 119 us for the 5.4e8 of
// 4,096 rows of 131,072, against 164 us for their bytes in bf16) and about six more instructions, of which those on pairs of
// numbers (f32x2) and of 16-bit halves do two elements at once.
#include <cooperative_groups.h>

#include "vl_logits.cuh"

namespace {

namespace cg = cooperative_groups;
typedef unsigned long long key_t64;

constexpr float LOWEST = -3.402823466e38f;
// Stands for minus infinity in a difference: times scale >= 1e-20 its exponential is 0, and 0 times it is 0.
constexpr float FAR_BELOW = -1e30f;
constexpr uint32_t TOP_MAX = VL_MAX_ALTERNATIVES;
constexpr uint32_t MAX_PARTS = 8;  // thread blocks of a row

struct ScoreOut {
    float *logprob, *entropy, *stats;
    uint32_t top;
    int32_t *ids;
    float *lps;
};

// ---- values with their places, as keys: larger values first, lower places first among equals (zeros of both signs are equal)
__device__ __forceinline__ uint32_t ordered(float x)
{
    const uint32_t b = __float_as_uint(x + 0.0f);
    return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float from_ordered(uint32_t o) { return __uint_as_float((o & 0x80000000u) ? o & 0x7FFFFFFFu : ~o); }
__device__ __forceinline__ key_t64 rank_key(float x, uint32_t i) { return ((key_t64)ordered(x) << 32) | (0xFFFFFFFFu - i); }
__device__ __forceinline__ uint32_t key_place(key_t64 k) { return 0xFFFFFFFFu - (uint32_t)k; }
__device__ __forceinline__ float key_value(key_t64 k) { return from_ordered((uint32_t)(k >> 32)); }

__device__ __forceinline__ key_t64 exchange(key_t64 k, uint32_t d, bool larger)
{
    const key_t64 other = __shfl_xor_sync(0xffffffffu, k, d);
    return (k > other) == larger ? k : other;
}
// A warp's 32 keys, largest first.
__device__ __forceinline__ key_t64 sort32(key_t64 k, uint32_t lane)
{
#pragma unroll
    for (uint32_t n = 2; n <= 32; n *= 2)
#pragma unroll
        for (uint32_t d = n / 2; d; d /= 2) k = exchange(k, d, ((lane & d) == 0) == ((lane & n) == 0));
    return k;
}
// The first 32 of two sorted lists of 32.
__device__ __forceinline__ key_t64 merge32(key_t64 a, key_t64 b, uint32_t lane)
{
    const key_t64 r = __shfl_sync(0xffffffffu, b, 31 - lane);
    key_t64 k = a > r ? a : r;
#pragma unroll
    for (uint32_t d = 16; d; d /= 2) k = exchange(k, d, (lane & d) == 0);
    return k;
}
// NW sorted lists in shared memory; the first 32 of all of them end up in list 0.  Every warp of the block calls it.
template <int NW>
__device__ __forceinline__ void merge_lists(key_t64 (*lists)[32], uint32_t warp, uint32_t lane)
{
#pragma unroll
    for (uint32_t half = NW / 2; half; half /= 2) {
        __syncthreads();
        if (warp < half) lists[warp][lane] = merge32(lists[warp][lane], lists[warp + half][lane], lane);
    }
    __syncthreads();
}

// ---- running sums
struct Sums {
    float m, s, t;  // largest logit; sum e, sum e d relative to it
};
__device__ __forceinline__ void raise(Sums &a, float m, float c)
{
    const float d = fmaxf(a.m - m, FAR_BELOW), f = ex2(d * c);
    a.t = (a.t + a.s * d) * f;
    a.s *= f;
    a.m = m;
}
__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}
__device__ __forceinline__ void warp_join(Sums &a, float c)
{
    raise(a, from_ordered(__reduce_max_sync(0xffffffffu, ordered(a.m))), c);
    a.s = warp_sum(a.s);
    a.t = warp_sum(a.t);
}

// Two more entries; low: minus the largest one, twice; c2: scale log2 e, twice.
__device__ __forceinline__ void sum_two(float x0, float x1, f32x2 low, f32x2 c2, f32x2 &s, f32x2 &t)
{
    float d0, d1, y0, y1;
    apart(add2(both(x0, x1), low), d0, d1);
    const f32x2 d = both(max_nan(d0, FAR_BELOW), max_nan(d1, FAR_BELOW));
    apart(mul2(d, c2), y0, y1);
    const f32x2 e = both(ex2(y0), ex2(y1));
    s = add2(s, e);
    t = fma2(e, d, t);
}

// A thread's state over the vectors of its stripe.
struct Run {
    float m;
    f32x2 s, t;
    uint32_t best;  // vector in which m was met first
};
template <typename T, int N, bool TOP>
__device__ __forceinline__ void take(Run &a, const uint4 (&raw)[N], uint32_t v, uint32_t step, float c)
{
    float vm[N], m;
#pragma unroll
    for (int u = 0; u < N; ++u) vm[u] = vector_max(raw[u], T{});
    m = vm[0];
#pragma unroll
    for (int u = 1; u < N; ++u) m = fmaxf(m, vm[u]);
    if (m > a.m) {
        const float d = fmaxf(a.m - m, FAR_BELOW), f = ex2(d * c);
        a.t = mul2(fma2(a.s, both(d, d), a.t), both(f, f));
        a.s = mul2(a.s, both(f, f));
        a.m = m;
        if (TOP) {
#pragma unroll
            for (int u = N - 1; u >= 0; --u)
                if (vm[u] == m) a.best = v + u * step;
        }
    }
    const float base = fmaxf(a.m, LOWEST);  // (nothing but impossible entries so far)
    const f32x2 low = both(-base, -base), c2 = both(c, c);
#pragma unroll
    for (int u = 0; u < N; ++u) {
        float x[EPV<T>];
        unpack(raw[u], x, T{});
#pragma unroll
        for (int j = 0; j < EPV<T>; j += 2) sum_two(x[j], x[j + 1], low, c2, a.s, a.t);
    }
}

__device__ __forceinline__ void empty_row(const ScoreOut &o, uint64_t r, bool left_out, uint32_t tid, uint32_t nt)
{
    const float inf = __int_as_float(0x7f800000);
    if (tid == 0) {
        if (o.logprob) o.logprob[r] = left_out ? 0.0f : -inf;
        if (o.entropy) o.entropy[r] = 0.0f;
        if (o.stats) *reinterpret_cast<float2 *>(o.stats + 2 * r) = left_out ? make_float2(0.0f, 0.0f) : make_float2(-inf, -inf);
    }
    for (uint32_t j = tid; j < o.top; j += nt) { o.ids[r * o.top + j] = -1; o.lps[r * o.top + j] = -inf; }
}

// Keys of a vector's entries that are no smaller than `least` and no impossible ones, handed to f.
template <typename T, typename F>
__device__ __forceinline__ void each_key(const uint4 &raw, int first, key_t64 least, F &&f)
{
    const float inf = __int_as_float(0x7f800000), floor = least ? key_value(least) : -inf;
    float x[EPV<T>];
    unpack(raw, x, T{});
#pragma unroll
    for (int j = 0; j < EPV<T>; ++j)
        if (x[j] >= floor && x[j] > -inf) {
            const key_t64 k = rank_key(x[j], (uint32_t)(first + j));
            if (k >= least) f(k);
        }
}

template <typename T, bool MASKED>
__device__ __forceinline__ uint4 fetch(const RowVectors<T> &x, const RowMask &mask, uint32_t v)
{
    uint4 raw = x.whole(v) ? *x.at(v) : x.part(v);
    if (MASKED) close_entries<T>(raw, mask.closed_from(x.first(v), EPV<T>));
    return raw;
}

constexpr uint32_t CAND = 512;  // candidates for the alternatives of a part

// The alternatives one by one, each a pass over the part: for rows whose best entries are crowded into a few threads' stripes.
template <typename T, bool MASKED, int NT>
__device__ __noinline__ void alternatives_one_by_one(const T *row, uint32_t V, const RowMask &mask, uint32_t v0, uint32_t v1, uint32_t top,
                                                     key_t64 (*lists)[32])
{
    const RowVectors<T> x(row, V);
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    key_t64 last = ~0ull, mine = 0;
    for (uint32_t j = 0; j < top; ++j) {
        key_t64 best = 0;
        for (uint32_t v = v0 + threadIdx.x; v < v1; v += NT)
            each_key<T>(fetch<T, MASKED>(x, mask, v), x.first(v), best, [&](key_t64 k) { if (k < last && k > best) best = k; });
        for (int d = 16; d; d >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, d));
        __syncthreads();
        if (lane == 0) lists[0][warp] = best;
        __syncthreads();
        for (uint32_t w = 0; w < NT / 32; ++w) best = max(best, lists[0][w]);
        if (lane == j) mine = best;
        last = best;
    }
    __syncthreads();
    if (warp == 0) lists[0][lane] = mine;
    __syncthreads();
}

// A part's 32 first keys into lists[0].  The k-th of the threads' best keys bounds the k-th of all from below, and only the k threads
// at or above it can have entries that are no smaller: their stripes alone are read again (from L2).
template <typename T, bool MASKED, int NT>
__device__ __forceinline__ void alternatives(const RowVectors<T> &x, const RowMask &mask, uint32_t v0, uint32_t v1, const Run &a, uint32_t top,
                                             key_t64 (*lists)[32], key_t64 *cand, uint32_t *n_cand)
{
    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    key_t64 mine = 0;
    if (a.best < v1)
        each_key<T>(fetch<T, MASKED>(x, mask, a.best), x.first(a.best), 0ull, [&](key_t64 k) { if (k > mine) mine = k; });
    lists[warp][lane] = sort32(mine, lane);
    if (tid == 0) *n_cand = 0;
    merge_lists<NT / 32>(lists, warp, lane);
    const key_t64 least = lists[0][top - 1];
    for (uint32_t j = warp; j < top; j += NT / 32) {
        const key_t64 k = lists[0][j];
        if (!k) break;
        const uint32_t owner = ((key_place(k) + x.lead) / EPV<T> - v0) % NT;
        for (uint32_t v = v0 + owner + lane * NT; v < v1; v += 32 * NT)
            each_key<T>(fetch<T, MASKED>(x, mask, v), x.first(v), least, [&](key_t64 q) {
                const uint32_t at = atomicAdd(n_cand, 1u);
                if (at < CAND) cand[at] = q;
            });
    }
    __syncthreads();
    const uint32_t n = *n_cand;
    if (n > CAND) {
        alternatives_one_by_one<T, MASKED, NT>(x.row, x.V, mask, v0, v1, top, lists);
        return;
    }
    for (uint32_t j = warp; j < NT / 32; j += NT / 32) {
        key_t64 k = tid < n ? cand[tid] : 0;
        if (n > j * 32) k = sort32(k, lane);
        if (NT < CAND)  // (fewer threads than candidates: the rest of them)
            for (uint32_t b = tid - lane + NT; b < n; b += NT) k = merge32(k, sort32(b + lane < n ? cand[b + lane] : 0ull, lane), lane);
        lists[j][lane] = k;
    }
    if (n <= 32) __syncthreads();
    else merge_lists<NT / 32>(lists, warp, lane);
}

// Long rows: a cluster of thread blocks per row (one block if there are rows enough), each block a run of vectors, each thread every
// NT-th vector of it.
template <typename T, bool MASKED, bool TOP, int NT>
__global__ void __launch_bounds__(NT, 1024 / NT) k_score_long(const LogitRows q, const ScoreOut o, uint32_t parts)
{
    constexpr int U = 4, NW = NT / 32;
    __shared__ float s_sums[3][NW];
    __shared__ float s_part[MAX_PARTS][3];
    __shared__ key_t64 s_lists[TOP ? NW : 1][32], s_parts[TOP ? MAX_PARTS : 1][32], s_cand[TOP ? CAND : 1];
    __shared__ uint32_t s_n;
    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, part = blockIdx.x % parts;
    const float c = q.scale * 1.44269504088896341f, inf = __int_as_float(0x7f800000);
    for (uint64_t r = blockIdx.x / parts; r < q.n_rows; r += gridDim.x / parts) {
        const int64_t tok = row_token(q, r);
        if (tok < 0) {
            if (part == 0) empty_row(o, r, true, tid, NT);
            continue;
        }
        const RowVectors<T> x(static_cast<const T *>(q.x) + r * q.stride, q.V);
        const RowMask mask = row_mask(q, r);
        const uint32_t per = (x.n + parts - 1) / parts, v0 = min(x.n, part * per), v1 = min(x.n, v0 + per);
        const uint32_t f0 = max(v0, x.lead ? 1u : 0u), f1 = min(v1, (x.lead + x.V) / EPV<T>);  // whole vectors
        if (parts > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
        float x_tok = 0.0f;
        if (part == 0 && tid == 0 && o.logprob) x_tok = to_f32(x.row[tok]);

        Run a{-inf, 0ull, 0ull, 0xFFFFFFFFu};
        uint4 raw[U];
        if (f0 > v0 && tid == 0) {
            uint4 one[1] = {fetch<T, MASKED>(x, mask, v0)};
            take<T, 1, TOP>(a, one, v0, NT, c);
        }
        for (uint32_t v = v0 + tid; v < f1; v += NT * U) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const uint32_t w = v + u * NT;
                raw[u] = make_uint4(MINUS_INF2<T>, MINUS_INF2<T>, MINUS_INF2<T>, MINUS_INF2<T>);
                if (w >= f0 && w < f1) raw[u] = *x.at(w);
            }
            if (MASKED) {
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (v + u * NT < f1) close_entries<T>(raw[u], mask.closed_from(x.first(v + u * NT), EPV<T>));
            }
            take<T, U, TOP>(a, raw, v, NT, c);
        }
        if (f1 < v1 && v1 > f0 && (v1 - 1 - v0) % NT == tid) {
            uint4 one[1] = {fetch<T, MASKED>(x, mask, v1 - 1)};
            take<T, 1, TOP>(a, one, v1 - 1, NT, c);
        }

        float s0, s1, t0, t1;
        apart(a.s, s0, s1);
        apart(a.t, t0, t1);
        Sums w{a.m, s0 + s1, t0 + t1};
        warp_join(w, c);
        __syncthreads();  // (what the row in front left in shared memory has been read)
        if (lane == 0) { s_sums[0][warp] = w.m; s_sums[1][warp] = w.s; s_sums[2][warp] = w.t; }
        if (TOP) alternatives<T, MASKED, NT>(x, mask, v0, v1, a, o.top, s_lists, s_cand, &s_n);
        else __syncthreads();
        if (warp == 0) {
            w = lane < NW ? Sums{s_sums[0][lane], s_sums[1][lane], s_sums[2][lane]} : Sums{-inf, 0.0f, 0.0f};
            warp_join(w, c);
        }
        if (parts > 1) {  // to the first block of the cluster
            asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");  // (it has read the row in front, and runs)
            cg::cluster_group cluster = cg::this_cluster();
            if (warp == 0) {
                if (lane == 0) {
                    float *to = cluster.map_shared_rank(&s_part[part][0], 0);
                    to[0] = w.m; to[1] = w.s; to[2] = w.t;
                }
                if (TOP) *cluster.map_shared_rank(&s_parts[part][lane], 0) = s_lists[0][lane];
            }
            cluster.sync();
            if (part != 0) continue;
            if (warp == 0) {
                w = lane < parts ? Sums{s_part[lane][0], s_part[lane][1], s_part[lane][2]} : Sums{-inf, 0.0f, 0.0f};
                warp_join(w, c);
                if (TOP) {
                    key_t64 k = s_parts[0][lane];
                    for (uint32_t j = 1; j < parts; ++j) k = merge32(k, s_parts[j][lane], lane);
                    s_lists[0][lane] = k;
                    __syncwarp();
                }
            }
        }
        if (warp == 0) {
            if (w.s == 0.0f) {
                empty_row(o, r, false, lane, 32);
            } else {
                const float L = logf(w.s);
                if (lane == 0) {
                    if (o.logprob) o.logprob[r] = MASKED && mask.is_closed((uint32_t)tok) ? -inf : (x_tok - w.m) * q.scale - L;
                    if (o.entropy) o.entropy[r] = L - q.scale * (w.t / w.s);
                    if (o.stats) *reinterpret_cast<float2 *>(o.stats + 2 * r) = make_float2(w.m, L);
                }
                if (TOP && lane < o.top) {
                    const key_t64 k = s_lists[0][lane];
                    o.ids[r * o.top + lane] = k ? (int32_t)key_place(k) : -1;
                    o.lps[r * o.top + lane] = k ? (key_value(k) - w.m) * q.scale - L : -inf;
                }
            }
        }
    }
}

template <typename T, bool MASKED, bool TOP>
cudaError_t launch_long(const LogitRows &q, const ScoreOut &o, int device, cudaStream_t st)
{
    constexpr int NT = 512;
    const uint64_t sms = (uint64_t)vl_device_sm_count(device);
    uint32_t parts = 1;
    while (parts < MAX_PARTS && q.n_rows * parts < 2 * sms && q.V / (2 * parts) >= NT * EPV<T>) parts *= 2;
    const uint64_t rows = q.n_rows < (1ull << 27) ? q.n_rows : (1ull << 27);
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = parts;
    at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((uint32_t)(rows * parts)); cfg.blockDim = NT; cfg.stream = st;
    cfg.attrs = &at; cfg.numAttrs = 1;
    g_vl_launches.fetch_add(1);
    return cudaLaunchKernelEx(&cfg, k_score_long<T, MASKED, TOP, NT>, q, o, parts);
}

// Short rows: a group of lanes per row, every logit read once into registers.
constexpr uint32_t SHORT_WARPS = 8, SHORT_CAND = 128;

// The best entries of a row that the whole warp holds (G = 32), as in the long rows: the k-th of the lanes' best bounds the k-th of all.
template <typename T, int NV>
__device__ __forceinline__ key_t64 warp_alternatives(const uint4 (&raw)[NV], const RowVectors<T> &x, uint32_t lane, uint32_t top, key_t64 *cand,
                                                     uint32_t *n_cand)
{
    key_t64 mine = 0;
#pragma unroll
    for (int j = 0; j < NV; ++j) each_key<T>(raw[j], x.first(lane + 32 * j), mine, [&](key_t64 k) { if (k > mine) mine = k; });
    const key_t64 least = __shfl_sync(0xffffffffu, sort32(mine, lane), top - 1);
    if (lane == 0) *n_cand = 0;
    __syncwarp();
#pragma unroll
    for (int j = 0; j < NV; ++j)
        each_key<T>(raw[j], x.first(lane + 32 * j), least, [&](key_t64 k) {
            const uint32_t at = atomicAdd(n_cand, 1u);
            if (at < SHORT_CAND) cand[at] = k;
        });
    __syncwarp();
    const uint32_t n = *n_cand;
    key_t64 best = 0;
    if (n <= SHORT_CAND) {
        best = sort32(lane < n ? cand[lane] : 0ull, lane);
        for (uint32_t b = 32; b < n; b += 32) best = merge32(best, sort32(b + lane < n ? cand[b + lane] : 0ull, lane), lane);
    } else {  // one by one
        key_t64 last = ~0ull;
        for (uint32_t i = 0; i < top; ++i) {
            key_t64 b = 0;
#pragma unroll 1
            for (int j = 0; j < NV; ++j) {
                uint4 r = raw[0];
#pragma unroll
                for (int l = 1; l < NV; ++l)
                    if (j == l) r = raw[l];
                each_key<T>(r, x.first(lane + 32 * j), b, [&](key_t64 k) { if (k < last && k > b) b = k; });
            }
            for (int d = 16; d; d >>= 1) b = max(b, __shfl_xor_sync(0xffffffffu, b, d));
            if (lane == i) best = b;
            last = b;
        }
    }
    __syncwarp();
    return best;
}

template <typename T, bool MASKED, bool TOP, int G, int NV>
__global__ void __launch_bounds__(SHORT_WARPS * 32) k_score_short(const LogitRows q, const ScoreOut o, bool aligned)
{
    static_assert(NV * EPV<T> <= 32, "a lane's entries");
    static_assert(!TOP || G == 32, "alternatives take the whole warp");
    __shared__ key_t64 s_cand[TOP ? SHORT_WARPS : 1][TOP ? SHORT_CAND : 1];
    __shared__ uint32_t s_n[SHORT_WARPS];
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane % G;
    const float c = q.scale * 1.44269504088896341f, inf = __int_as_float(0x7f800000);
    const uint64_t step = (uint64_t)gridDim.x * SHORT_WARPS * (32 / G);
    for (uint64_t r0 = ((uint64_t)blockIdx.x * SHORT_WARPS + warp) * (32 / G); r0 < q.n_rows; r0 += step) {
        const uint64_t r = min(r0 + lane / G, q.n_rows - 1);
        const bool there = r0 + lane / G < q.n_rows;  // (the warp's last rows may not be: it works on the last one instead)
        const RowVectors<T> x(static_cast<const T *>(q.x) + r * q.stride, q.V);
        uint4 raw[NV];
        fetch_row<T, G, NV>(raw, x, g, aligned);
        const int64_t tok = row_token(q, r);
        uint32_t word = 0;
        if (MASKED) {
            word = row_mask(q, r).closed(g);
#pragma unroll
            for (int j = 0; j < NV; ++j) close_entries<T>(raw[j], group_closed<T, G>(word, x.first(g + G * j), aligned));
        }
        float x_tok = 0.0f;
        if (g == 0 && o.logprob && tok >= 0) x_tok = to_f32(x.row[tok]);

        float m = vector_max(raw[0], T{});
#pragma unroll
        for (int j = 1; j < NV; ++j) m = fmaxf(m, vector_max(raw[j], T{}));
#pragma unroll
        for (int d = G / 2; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
        const float base = fmaxf(m, LOWEST);
        f32x2 s2 = 0ull, t2 = 0ull;
        const f32x2 low = both(-base, -base), c2 = both(c, c);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float e[EPV<T>];
            unpack(raw[j], e, T{});
#pragma unroll
            for (int i = 0; i < EPV<T>; i += 2) sum_two(e[i], e[i + 1], low, c2, s2, t2);
        }
        float s, t, b;
        apart(s2, s, b);
        s += b;
        apart(t2, t, b);
        t += b;
#pragma unroll
        for (int d = G / 2; d; d >>= 1) {
            s += __shfl_xor_sync(0xffffffffu, s, d);
            t += __shfl_xor_sync(0xffffffffu, t, d);
        }
        const float L = logf(s);
        const bool left = tok < 0, empty = s == 0.0f;
        bool shut = false;
        if (MASKED) shut = (__shfl_sync(0xffffffffu, word, left ? 0 : (int)((uint32_t)tok >> 5) & (G - 1), G) >> (tok & 31)) & 1;
        if (g == 0 && there) {
            if (o.logprob) o.logprob[r] = left ? 0.0f : (empty || shut ? -inf : (x_tok - m) * q.scale - L);
            if (o.entropy) o.entropy[r] = left || empty ? 0.0f : L - q.scale * (t / s);
            if (o.stats)
                *reinterpret_cast<float2 *>(o.stats + 2 * r) = left ? make_float2(0.0f, 0.0f) : make_float2(empty ? -inf : m, L);
        }
        if (TOP) {
            const key_t64 k = warp_alternatives<T, NV>(raw, x, lane, o.top, s_cand[warp], &s_n[warp]);
            if (lane < o.top) {
                const bool one = k != 0 && !left;
                o.ids[r * o.top + lane] = one ? (int32_t)key_place(k) : -1;
                o.lps[r * o.top + lane] = one ? (key_value(k) - m) * q.scale - L : -inf;
            }
        }
    }
}

template <typename T, bool MASKED, bool TOP, int G, int NV>
cudaError_t run_short(const LogitRows &q, const ScoreOut &o, bool aligned, cudaStream_t st)
{
    const uint64_t blocks = (q.n_rows + SHORT_WARPS * (32 / G) - 1) / (SHORT_WARPS * (32 / G));
    k_score_short<T, MASKED, TOP, G, NV><<<(uint32_t)(blocks < (1u << 30) ? blocks : (1u << 30)), SHORT_WARPS * 32, 0, st>>>(q, o, aligned);
    g_vl_launches.fetch_add(1);
    return cudaGetLastError();
}

// Whether the rows are short, and if so the launch.
template <typename T, bool MASKED, bool TOP>
bool launch_short(const LogitRows &q, const ScoreOut &o, cudaStream_t st, cudaError_t *e)
{
    bool aligned;
    const uint32_t n = row_vectors(q, sizeof(T), &aligned);
    if constexpr (TOP) {
        if (n <= 32) *e = run_short<T, MASKED, true, 32, 1>(q, o, aligned, st);
        else if (n <= 64) *e = run_short<T, MASKED, true, 32, 2>(q, o, aligned, st);
        else if (n <= 128) *e = run_short<T, MASKED, true, 32, 4>(q, o, aligned, st);
        else if (n <= 256 && sizeof(T) == 4) *e = run_short<T, MASKED, true, 32, 32 / EPV<T>>(q, o, aligned, st);
        else return false;
    } else {
        if (n <= 4) *e = run_short<T, MASKED, false, 4, 1>(q, o, aligned, st);
        else if (n <= 16) *e = run_short<T, MASKED, false, 4, 4>(q, o, aligned, st);
        else if (n <= 32) *e = run_short<T, MASKED, false, 8, 4>(q, o, aligned, st);
        else if (n <= 64) *e = run_short<T, MASKED, false, 16, 4>(q, o, aligned, st);
        else if (n <= 128) *e = run_short<T, MASKED, false, 32, 4>(q, o, aligned, st);
        else if (n <= 256 && sizeof(T) == 4) *e = run_short<T, MASKED, false, 32, 32 / EPV<T>>(q, o, aligned, st);
        else return false;
    }
    return true;
}

template <typename T, bool MASKED, bool TOP>
cudaError_t launch(const LogitRows &q, const ScoreOut &o, int device, cudaStream_t st)
{
    cudaError_t e;
    return launch_short<T, MASKED, TOP>(q, o, st, &e) ? e : launch_long<T, MASKED, TOP>(q, o, device, st);
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
    if (!(x->scale >= 1e-20f && x->scale <= 1e20f)) return VL_ERR_INVALID_ARG;
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
    const bool masked = q.occupied || q.widths;
    return by_type(x->dtype, [&](auto type) {
        using T = decltype(type);
        cudaStream_t st = (cudaStream_t)stream;
        const cudaError_t e = masked ? (top ? launch<T, true, true>(q, o, device, st) : launch<T, true, false>(q, o, device, st))
                                     : (top ? launch<T, false, true>(q, o, device, st) : launch<T, false, false>(q, o, device, st));
        return e == cudaSuccess ? VL_OK : VL_ERR_CUDA;
    });
}
