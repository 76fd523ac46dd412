// Drawing from long rows: one pass over the row, and a second look at what matters of it.
//
// A block of four warps, a cluster of such blocks, or one warp is at a row; each warp has a run of the row's vectors and cuts it into eight segments.
// The pass keeps for every segment the sum of its weights (in 64 bits from 32 entries of a lane in 32), and for every lane of it the largest
// logit: 1,024 groups of a block, 256 of a warp alone.
//   No rules: the sums tell the segment that the number falls into, and that one is read again.
//   top_k, top_p, min_p: the groups' largest logits, counted in 128 steps below the largest one, bound the cut from below: top_k groups with
//   such a logit, or groups whose largest entries alone have weight enough, mean that the cut is no lower.  The groups that reach the bound are
//   read again, and what reaches it is gathered, put in order, and the rules are applied in 64 bits.
// A row is left to k_sample_rest where a border is nearer to what it is compared with than the 32-bit terms are known (eps, below), where more
// than CAP entries reach the bound (1,024; 256 of a warp alone), or where a logit is no number or beyond the range of the sums.
//
// eps: a weight is within (4 + 1.6 |y|) u of its value, u = 2^-24, y its power of two relative to the warp's reference, which no entry
// passes by more than 3; a lane's 32 entries go through 8 additions, and 64 bits hold what these make.  The mean of |y| relative to the largest logit
// is at most log2(V / S).  S is therefore known to eps S, eps = (16 + 1.6 (log2(V / S) + 3)) u, and a border between two parts of it as in the
// short rows.
//
// What bounds it: the pass reads the logits once (1,024 rows of 131,072 bf16: 42 us after the median of the rows, 65 after the last, for a floor of
// 42: one wave of blocks, each at a row, seven to a multiprocessor), then every row has an end of about 15 us under load, most of it waiting (barriers, the second
// look's loads, 64-bit operations one behind the other), 78 us in all; with one warp at a row, 28 ends run side by side.
#pragma once
#include "vl_sample_short.cuh"

namespace {

constexpr uint32_t LD_U = 4, LD_RING = 3, LD_SEGS = 8, LD_PARTS = 8;
constexpr uint32_t LD_STEP = 32 * LD_U;               // vectors of a warp at a time
constexpr uint32_t LD_BINS = 128, LD_GUESS = 320;
// A block of NT threads: its ring, and what lies there after the pass: up to CAP keys, then their weights, then the groups.
template <uint32_t NT>
struct Long {
    static constexpr uint32_t WARPS = NT / 32, RING_BYTES = NT * LD_U * LD_RING * 16, CAP = 8 * NT, WEIGHTS_AT = CAP * 8, GROUPS_AT = CAP * 16;
    static_assert(GROUPS_AT + LD_SEGS * NT * 2 <= RING_BYTES && CAP * 24 <= RING_BYTES && NT * 24 <= RING_BYTES - GROUPS_AT, "fits the ring");
};

__device__ __forceinline__ void ld_copy(uint32_t to, const uint4 *from)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void ld_close() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void ld_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// The smallest of several vectors' elements.
template <int N>
__device__ __forceinline__ float vectors_min(const uint4 (&r)[N], float)
{
    float m = __uint_as_float(r[0].x);
#pragma unroll
    for (int j = 0; j < N; ++j)
        m = fminf(m, fminf(fminf(__uint_as_float(r[j].x), __uint_as_float(r[j].y)), fminf(__uint_as_float(r[j].z), __uint_as_float(r[j].w))));
    return m;
}
template <typename P, int N>
__device__ __forceinline__ P halves_min(const uint4 (&r)[N])
{
    P m[4];
    memcpy(m, &r[0], 16);
#pragma unroll
    for (int j = 1; j < N; ++j) {
        P h[4];
        memcpy(h, &r[j], 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) m[i] = __hmin2(m[i], h[i]);
    }
    return __hmin2(__hmin2(m[0], m[1]), __hmin2(m[2], m[3]));
}
template <int N>
__device__ __forceinline__ float vectors_min(const uint4 (&r)[N], __half)
{
    const __half2 m = halves_min<__half2>(r);
    return fminf(__low2float(m), __high2float(m));
}
template <int N>
__device__ __forceinline__ float vectors_min(const uint4 (&r)[N], __nv_bfloat16)
{
    const __nv_bfloat162 m = halves_min<__nv_bfloat162>(r);
    return fminf(__low2float(m), __high2float(m));
}

// A vector's entries of minus infinity.
template <typename T>
__device__ __forceinline__ uint32_t impossible(const uint4 &r, T)
{
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
    uint32_t n = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (sizeof(T) == 4) n += w[j] == MINUS_INF2<T>;
        else n += (w[j] << 16 == MINUS_INF2<T> << 16) + (w[j] >> 16 == MINUS_INF2<T> >> 16);
    }
    return n;
}

// A block's n keys in falling order (n <= CAP).  Few: each to its rank; many: by halves.  (A key's rank among 256 takes about as many steps as
// the halves do.)
template <uint32_t NT>
__device__ __forceinline__ void sort_keys(key_t64 *keys, uint32_t n)
{
    const uint32_t tid = threadIdx.x;
    if (n <= 2 * NT) {
        key_t64 mine[2];
        uint32_t rank[2] = {0, 0};
        mine[0] = tid < n ? keys[tid] : 0ull;
        mine[1] = tid + NT < n ? keys[tid + NT] : 0ull;
        for (uint32_t j = 0; j < n; ++j) {
            const key_t64 other = keys[j];
            rank[0] += other > mine[0];
            rank[1] += other > mine[1];
        }
        __syncthreads();
        if (tid < n) keys[rank[0]] = mine[0];
        if (tid + NT < n) keys[rank[1]] = mine[1];
        __syncthreads();
        return;
    }
    uint32_t N = 4 * NT;
    while (N < n) N *= 2;
    for (uint32_t i = n + tid; i < N; i += NT) keys[i] = 0ull;
    __syncthreads();
    for (uint32_t k = 2; k <= N; k *= 2)
        for (uint32_t d = k / 2; d; d /= 2) {
            for (uint32_t p = tid; p < N / 2; p += NT) {
                const uint32_t i = 2 * p - (p & (d - 1)), j = i + d;
                const key_t64 a = keys[i], b = keys[j];
                if ((a < b) == ((i & k) == 0)) { keys[i] = b; keys[j] = a; }
            }
            __syncthreads();
        }
}

// In place: sums of the first i + 1 of n numbers (n <= CAP).  s: a number for each warp.
template <uint32_t NT>
__device__ __forceinline__ void sum_up(double *v, uint32_t n, double *s)
{
    const uint32_t tid = threadIdx.x, lane = tid & 31, per = (n + NT - 1) / NT, first = min(n, tid * per), end = min(n, first + per);
    double own = 0.0;
    for (uint32_t i = first; i < end; ++i) own += v[i];
    double up = own;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const double w = __shfl_up_sync(0xffffffffu, up, d);
        if (lane >= (uint32_t)d) up += w;
    }
    if (lane == 31) s[tid >> 5] = up;
    __syncthreads();
    double base = __shfl_up_sync(0xffffffffu, up, 1);
    if (lane == 0) base = 0.0;
    double front = 0.0;
    for (uint32_t w = 0; w < tid >> 5; ++w) front += s[w];
    double run = front + base;
    for (uint32_t i = first; i < end; ++i) {
        run += v[i];
        v[i] = run;
    }
    __syncthreads();
}

// The smallest of a thread's numbers over the block, in every thread; *s is 0xFFFFFFFF before, and a barrier lies between that and the call.
__device__ __forceinline__ uint32_t block_min(uint32_t v, uint32_t *s)
{
    v = __reduce_min_sync(0xffffffffu, v);
    if ((threadIdx.x & 31) == 0) atomicMin(s, v);
    __syncthreads();
    return *s;
}

// What a row's listed entries are drawn with.
struct Listed {
    const LogitRows &q;
    const SampleRules &s;
    const SampleOut &o;
    const double *table;
    uint64_t r;
    float u, M, least, L;  // least: the lowest logit that min_p keeps
    double S, eps;
    bool whole;            // nothing but the bound from top_k and top_p cut the list short
    __device__ __forceinline__ double weight(key_t64 k) const { return exp_below_1((double)q.scale * ((double)key_value(k) - (double)M), table); }
    __device__ __forceinline__ void put(key_t64 k, double total, uint32_t kept) const
    {
        const float z = log_odds(key_value(k), M, q.scale);
        put_sample(o, r, (int64_t)key_place(k), min_nan(z - L, 0.0f), min_nan(z - logf((float)total), 0.0f), kept);
    }
};

// One block, at most an entry a thread: each to its rank, sums in order, and the sums in the order of the numbers by looking at all of them.
// buffer: 24 bytes an entry.  False if that is too near to call.
template <uint32_t NT>
struct Few {
    static constexpr uint32_t NW = NT / 32;
    double sums[NW];
    uint32_t counts[NW][3], places[NW];
};
template <uint32_t NT>
__device__ __forceinline__ bool draw_few(const Listed &a, const key_t64 *keys, uint32_t n, unsigned char *buffer, Few<NT> &f)
{
    key_t64 *const sorted = reinterpret_cast<key_t64 *>(buffer);
    double *const w = reinterpret_cast<double *>(buffer + NT * 8), *const sums = w + NT;
    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    key_t64 key = tid < n ? keys[tid] : 0ull;
    double own = tid < n ? a.weight(key) : 0.0;
    if (warp * 32 < n) {
        uint32_t rank = 0;
#pragma unroll 4
        for (uint32_t j = 0; j < n; ++j) rank += keys[j] > key;
        if (tid < n) {
            sorted[rank] = key;
            w[rank] = own;
        }
    }
    __syncthreads();
    key = tid < n ? sorted[tid] : 0ull;
    own = tid < n ? w[tid] : 0.0;
    double up = own;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const double v = __shfl_up_sync(0xffffffffu, up, d);
        if (lane >= (uint32_t)d) up += v;
    }
    if (lane == 31) f.sums[warp] = up;
    __syncthreads();
    for (uint32_t k = 0; k < warp; ++k) up += f.sums[k];
    sums[tid] = up;
    __syncthreads();
    uint32_t kept = a.s.top_k ? min(n, a.s.top_k) : n;
    const bool p = a.s.top_p < 1.0;
    const double need = p ? a.s.top_p * (a.s.top_k ? sums[kept - 1] : a.S) : 0.0, lacks = a.s.top_k ? 0.0 : a.eps * need;
    // sums that do not reach what is needed, for certain and perhaps; logits that min_p keeps
    const uint32_t under = __popc(__ballot_sync(0xffffffffu, tid < kept && up < need - lacks));
    const uint32_t perhaps = __popc(__ballot_sync(0xffffffffu, tid < kept && up < need + lacks));
    const uint32_t from = __popc(__ballot_sync(0xffffffffu, tid < n && key_value(key) >= a.least));
    if (lane == 0) { f.counts[warp][0] = under; f.counts[warp][1] = perhaps; f.counts[warp][2] = from; }
    __syncthreads();
    uint32_t all[3] = {0, 0, 0};
#pragma unroll
    for (uint32_t k = 0; k < NT / 32; ++k)
#pragma unroll
        for (int j = 0; j < 3; ++j) all[j] += f.counts[k][j];
    if (p) {
        if (all[0] != all[1] || (a.whole && all[0] >= kept)) return false;
        kept = min(kept, all[0] + 1);
    }
    kept = min(kept, all[2]);
    const double total = sums[kept - 1], at = (double)a.u * total;
    const uint32_t place = tid < kept ? key_place(key) : 0xFFFFFFFFu;
    uint32_t first = 0xFFFFFFFFu;
    if (warp * 32 < kept) {
        double part[4] = {0.0, 0.0, 0.0, 0.0};  // (four additions under way)
        for (uint32_t j0 = 0; j0 < kept; j0 += 4)
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j)
                if (j0 + j < kept && key_place(sorted[j0 + j]) <= place) part[j] += w[j0 + j];
        const double sum = (part[0] + part[1]) + (part[2] + part[3]);
        first = __reduce_min_sync(0xffffffffu, sum > at ? place : 0xFFFFFFFFu);
    }
    if (lane == 0) f.places[warp] = first;
    __syncthreads();
    for (uint32_t k = 0; k < NT / 32; ++k) first = min(first, f.places[k]);
    if (place == first && tid < kept) a.put(key, total, kept);
    return first != 0xFFFFFFFFu;
}

// The same for n keys in any order (n <= CAP): sorted, summed up, cut; what is kept is sorted by its numbers and summed up again.
template <uint32_t NT>
__device__ __forceinline__ bool draw_many(const Listed &a, key_t64 *keys, uint32_t n, double *w, key_t64 *second, double *s_sums, uint32_t *s_found)
{
    const uint32_t tid = threadIdx.x;
    if (tid < 2) s_found[tid] = 0xFFFFFFFFu;
    sort_keys<NT>(keys, n);
    for (uint32_t i = tid; i < n; i += NT) w[i] = a.weight(keys[i]);
    __syncthreads();
    sum_up<NT>(w, n, s_sums);
    uint32_t kept = a.s.top_k ? min(n, a.s.top_k) : n;
    if (a.s.top_p < 1.0) {
        const double need = a.s.top_p * (a.s.top_k ? w[kept - 1] : a.S), lacks = a.s.top_k ? 0.0 : a.eps * need;
        uint32_t first = 0xFFFFFFFFu;
        for (uint32_t i = tid; i < kept && first == 0xFFFFFFFFu; i += NT)
            if (w[i] >= need) first = i;
        first = block_min(first, s_found);
        if (first != 0xFFFFFFFFu) {
            if (w[first] < need + lacks || (first && w[first - 1] >= need - lacks)) return false;
            kept = first + 1;
        } else if (a.whole || w[kept - 1] >= need - lacks) {  // (else what is listed is all that min_p leaves)
            return false;
        }
    }
    if (a.s.min_p > 0.0) {
        uint32_t first = 0xFFFFFFFFu;
        for (uint32_t i = tid; i < kept && first == 0xFFFFFFFFu; i += NT)
            if (key_value(keys[i]) < a.least) first = i;
        kept = min(kept, block_min(first, s_found + 1));
    }
    const double total = w[kept - 1], at = (double)a.u * total;
    for (uint32_t i = tid; i < kept; i += NT) second[i] = (key_t64)(0xFFFFFFFFu - key_place(keys[i])) << 32 | i;
    __syncthreads();
    sort_keys<NT>(second, kept);
    for (uint32_t i = tid; i < kept; i += NT) w[i] = a.weight(keys[(uint32_t)second[i]]);
    if (tid == 0) s_found[0] = 0xFFFFFFFFu;
    __syncthreads();
    sum_up<NT>(w, kept, s_sums);
    uint32_t first = 0xFFFFFFFFu;
    for (uint32_t i = tid; i < kept && first == 0xFFFFFFFFu; i += NT)
        if (w[i] > at) first = i;
    first = block_min(first, s_found);
    if (first == 0xFFFFFFFFu) return false;
    if (tid == 0) a.put(keys[(uint32_t)second[first]], total, kept);
    return true;
}

// An entry of a vector's word.
__device__ __forceinline__ float entry_of(uint32_t word, int, float) { return __uint_as_float(word); }
__device__ __forceinline__ float entry_of(uint32_t word, int high, __half) { return __half2float(__ushort_as_half((unsigned short)(high ? word >> 16 : word))); }
__device__ __forceinline__ float entry_of(uint32_t word, int high, __nv_bfloat16) { return __uint_as_float(high ? word & 0xFFFF0000u : word << 16); }

// A block reads the vectors from .. to - 1 of a row again, NT at a time, in the order of the numbers, for the entry up to which the sum is above
// `at`; before: the sum in front of them; back: a weight's part that its rounded reference lacks.  *found becomes 1 if no border is nearer than slack.
struct Segment {
    uint64_t r;
    uint32_t from, to, kept;
    double before, at, slack, back;
    float M, L;
};
template <typename T, bool MASKED, uint32_t NT>
__device__ __forceinline__ void find_in_segment(const LogitRows &q, const SampleOut &o, const Segment g, double *s_sums, uint32_t *found)
{
    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const RowVectors<T> x(static_cast<const T *>(q.x) + g.r * q.stride, q.V);
    const RowMask mask = row_mask(q, g.r);
    double before = g.before;
    for (uint32_t w0 = g.from; w0 < g.to; w0 += NT) {
        const uint32_t v = w0 + tid;
        uint4 raw = make_uint4(MINUS_INF2<T>, MINUS_INF2<T>, MINUS_INF2<T>, MINUS_INF2<T>);
        if (v < g.to) raw = open_vector<T, MASKED>(x, mask, v);
        float xs[EPV<T>], e[EPV<T>];
        unpack(raw, xs, T{});
        powers<T>(xs, g.M, q.scale * LOG2E, false, e);
        const double own = (double)sum_of(e) * g.back;
        double up = own;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const double t = __shfl_up_sync(0xffffffffu, up, d);
            if (lane >= (uint32_t)d) up += t;
        }
        if (lane == 31) s_sums[warp] = up;
        __syncthreads();
        double front = before;
        for (uint32_t k = 0; k < NT / 32; ++k) {
            if (k < warp) front += s_sums[k];
            before += s_sums[k];
        }
        double cum = front + (up - own);
        if (cum <= g.at && front + up > g.at) {
            const float c = q.scale * LOG2E, b = -__fmul_rn(g.M, c);
#pragma unroll 1
            for (int i = 0; i < EPV<T>; ++i) {  // (one lane, once a row: few registers)
                const int at = i / (EPV<T> / 4);
                const uint32_t word = at == 0 ? raw.x : at == 1 ? raw.y : at == 2 ? raw.z : raw.w;
                const float v = entry_of(word, i & 1, T{});
                const double next = cum + (double)ex2(__fmaf_rn(v, c, b)) * g.back;
                if (next > g.at) {
                    if (g.at >= cum + g.slack && next >= g.at + g.slack) {
                        const float lp = min_nan(log_odds(v, g.M, q.scale) - g.L, 0.0f);
                        put_sample(o, g.r, (int64_t)x.first(w0 + tid) + i, lp, lp, g.kept);
                        *found = 1;
                    }
                    break;
                }
                cum = next;
            }
        }
        __syncthreads();
        if (before > g.at) break;
    }
}

template <typename T, bool MASKED, bool RULES, bool CLUSTER, uint32_t NT>
__global__ void __launch_bounds__(NT, 1024 / NT) k_sample_long(const LogitRows q, const SampleRules s, const SampleOut o,
                                                              uint32_t log_of_parts)
{
    typedef Long<NT> K;
    constexpr uint32_t U = LD_U, RING = LD_RING, NW = K::WARPS, MAX_PARTS = CLUSTER ? LD_PARTS : 1;
    static_assert(!CLUSTER || NT == LD_BINS, "a thread for each bin");
    constexpr uint32_t RECS = RULES ? NW : NW * LD_SEGS;  // sums of a part
    const uint32_t log_parts = CLUSTER ? log_of_parts : 0, parts = 1u << log_parts, part = blockIdx.x & (parts - 1);
    extern __shared__ __align__(16) uint4 s_ring[];
    __shared__ T s_most[RULES ? LD_SEGS : 1][RULES ? NT : 1];
    __shared__ double s_sum[MAX_PARTS * RECS], s_sums[NW];
    __shared__ float s_ref[MAX_PARTS * RECS], s_max[MAX_PARTS * NW], s_min[MAX_PARTS * NW], s_bound;
    __shared__ uint32_t s_count[MAX_PARTS * NW], s_bins[RULES ? LD_BINS : 1], s_mass[RULES ? LD_BINS : 1], s_n[3], s_found[2], s_base;
    __shared__ double s_table[EXP_TABLE];
    __shared__ Few<NT> s_few;
    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint64_t step = gridDim.x >> log_parts;
    const float c = q.scale * LOG2E, inf = __int_as_float(0x7f800000), margin = 3.0f / c;
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(s_ring) + tid * 16;
    unsigned char *const buffer = reinterpret_cast<unsigned char *>(s_ring);
    cg::cluster_group cluster = cg::this_cluster();
    auto away = [&](auto *p, uint32_t b) { return CLUSTER ? cluster.map_shared_rank(p, b) : p; };  // the same place in another block
    auto meet = [&]() {
        if (CLUSTER) cluster.sync();
        else __syncthreads();
    };
    pdl_go();
    for (uint32_t i = tid; i < EXP_TABLE; i += NT) s_table[i] = exp2((double)i / EXP_TABLE);
    if (CLUSTER) cluster.sync();  // (all blocks of the cluster run)

    for (uint64_t r = blockIdx.x >> log_parts; r < q.n_rows; r += step) {
        const float u = s.uniform[r];
        if (!drawn_at_all(u)) {
            if (part == 0 && tid == 0) {
                put_sample(o, r, -1, 0.0f, 0.0f, 0);
                s.left[r] = 0;
            }
            continue;
        }
        const RowVectors<T> x(static_cast<const T *>(q.x) + r * q.stride, q.V);
        const RowMask mask = row_mask(q, r);
        // the block's part of the row, and the warp's run of that, in vectors
        const uint32_t per_part = (x.n + parts - 1) >> log_parts;
        const uint32_t p0 = min(x.n, part * per_part), p1 = min(x.n, p0 + per_part);
        const uint32_t per = ((p1 - p0 + NW - 1) / NW + 7) & ~7u;
        const uint32_t v0 = min(p1, p0 + warp * per), v1 = min(p1, v0 + per);
        const uint32_t steps = (v1 - v0 + LD_STEP - 1) / LD_STEP;
        const uint32_t seg_steps = ((per + LD_STEP - 1) / LD_STEP + LD_SEGS - 1) / LD_SEGS;  // the same in every warp of the block
        // a vector that reaches into a neighbouring row is copied whole (and not taken from there), one that may reach out of the matrix is not
        const uint32_t lo = r == 0 && x.lead ? 1u : 0u, hi = r == q.n_rows - 1 ? (x.lead + x.V) / EPV<T> : x.n;
        uint32_t in = 0, slot_in = 0, slot_out = 0;
        auto copy_step = [&]() {
            if (in < steps) {
                const uint32_t v = v0 + in * LD_STEP + lane, to = ring + slot_in * (U * NT * 16);
#pragma unroll
                for (uint32_t j = 0; j < U; ++j)
                    if (v + 32 * j < v1 && v + 32 * j >= lo && v + 32 * j < hi) ld_copy(to + j * (NT * 16), x.at(v + 32 * j));
                slot_in = slot_in + 1 == RING ? 0 : slot_in + 1;
                ++in;
            }
            ld_close();
        };
#pragma unroll 1
        for (uint32_t i = 0; i < RING - 1; ++i) copy_step();

        // the warp's reference; the lane's largest logit, the smallest of its groups', its possible entries
        float ref = -inf, limit = -inf, most = -inf, least = inf;
        double total = 0.0;
        uint32_t at_step = 0, count = 0;
#pragma unroll 1
        for (uint32_t seg = 0; seg < LD_SEGS; ++seg) {
            float group = -inf;
            const uint32_t end = min(steps, at_step + seg_steps);
#pragma unroll 1
            for (; at_step < end; ++at_step) {
                ld_wait<RING - 2>();
                const uint32_t first = v0 + at_step * LD_STEP, v = first + lane;
                const uint4 *slot = s_ring + slot_out * (U * NT) + tid;
                slot_out = slot_out + 1 == RING ? 0 : slot_out + 1;
                uint4 raw[U];
                const bool whole = first + LD_STEP <= v1 && (first > 0 || x.lead == 0) && first + LD_STEP <= (x.lead + x.V) / EPV<T>;
#pragma unroll
                for (uint32_t j = 0; j < U; ++j) {
                    const uint32_t w = v + 32 * j;
                    raw[j] = slot[j * NT];
                    if (!whole) {
                        if (w >= v1) raw[j] = make_uint4(MINUS_INF2<T>, MINUS_INF2<T>, MINUS_INF2<T>, MINUS_INF2<T>);
                        else if (!x.whole(w)) raw[j] = x.part(w);
                    }
                    if (MASKED) close_entries<T>(raw[j], w < v1 ? mask.closed_from(x.first(w), EPV<T>) : 0u);
                }
                copy_step();
                const float m = vectors_max<(int)U>(raw, T{});
                group = fmaxf(group, m);
                if (!RULES) {  // impossible entries are few: they are looked for where the smallest is one
                    count += U * EPV<T>;
                    if (vectors_min<(int)U>(raw, T{}) == -inf) {
#pragma unroll
                        for (uint32_t j = 0; j < U; ++j) count -= impossible(raw[j], T{});
                    }
                }
                if (__any_sync(0xffffffffu, m > limit)) {
                    const float top = from_ordered(__reduce_max_sync(0xffffffffu, ordered(m)));
                    limit = top + margin;
                    // twice as far below as the largest logit may lie: what has no reference there is 0 as it is, and next to any row's largest
                    if (top * c > -2.0f * FAR_OUT) {
                        total *= ref == -inf ? 0.0 : (double)ex2(__fsub_rn(__fmul_rn(ref, c), __fmul_rn(top, c)));
                        ref = top;
                    }
                }
                const float b = ref == -inf ? 0.0f : -__fmul_rn(ref, c);
                const f32x2 c2 = both(c, c), low = both(b, b);
                f32x2 acc[U];
#pragma unroll
                for (uint32_t j = 0; j < U; ++j) {
                    float e[EPV<T>];
                    unpack(raw[j], e, T{});
                    acc[j] = 0ull;
#pragma unroll
                    for (int i = 0; i < EPV<T>; i += 2) {
                        float y0, y1;
                        apart(fma2(both(e[i], e[i + 1]), c2, low), y0, y1);
                        acc[j] = add2(acc[j], both(ex2(y0), ex2(y1)));
                    }
                }
                float a0, a1;
                apart(add2(add2(acc[0], acc[1]), add2(acc[2], acc[3])), a0, a1);
                total += (double)(a0 + a1);
            }
            most = fmaxf(most, group);
            if (RULES) {
                if (group > -inf) least = fminf(least, group);
                from_f32(s_most[RULES ? seg : 0][RULES ? tid : 0], group);
            } else {
#pragma unroll
                for (int d = 16; d; d >>= 1) total += __shfl_xor_sync(0xffffffffu, total, d);
                if (lane < parts) {
                    *away(&s_sum[RULES ? 0 : part * RECS + warp * LD_SEGS + seg], lane) = total;
                    *away(&s_ref[RULES ? 0 : part * RECS + warp * LD_SEGS + seg], lane) = ref;
                }
                total = 0.0;
            }
        }
        ld_wait<0>();
        most = from_ordered(__reduce_max_sync(0xffffffffu, ordered(most)));
        if (RULES) {
            least = from_ordered(__reduce_min_sync(0xffffffffu, ordered(least)));
#pragma unroll
            for (int d = 16; d; d >>= 1) total += __shfl_xor_sync(0xffffffffu, total, d);
        } else {
            count = __reduce_add_sync(0xffffffffu, count);
        }
        if (lane < parts) {
            const uint32_t at = part * NW + warp;
            *away(&s_max[at], lane) = most;
            if (RULES) {
                *away(&s_min[at], lane) = least;
                *away(&s_sum[at], lane) = total;
                *away(&s_ref[at], lane) = ref;
            } else {
                *away(&s_count[at], lane) = count;
            }
        }
        if (RULES) {
            for (uint32_t i = tid; i < LD_BINS; i += NT) s_bins[RULES ? i : 0] = s_mass[RULES ? i : 0] = 0;
            if (tid < 3) s_n[tid] = 0;
        }
        meet();

        // M and S relative to it, the same in every thread
        const uint32_t warps = parts * NW;  // at most 32
        const float M = from_ordered(__reduce_max_sync(0xffffffffu, lane < warps ? ordered(s_max[lane]) : 0u));
        const float low = RULES ? from_ordered(__reduce_min_sync(0xffffffffu, lane < warps ? ordered(s_min[lane]) : 0xFFFFFFFFu)) : 0.0f;
        count = RULES ? 0u : __reduce_add_sync(0xffffffffu, lane < warps ? s_count[lane] : 0u);
        const double cM = (double)c * (double)M;
        auto relative = [&](uint32_t i) {  // (a warp's sums are relative to its rounded product; without one they are 0, or no number)
            return s_ref[i] == -inf ? s_sum[i] : s_sum[i] * exp_below_1(((double)__fmul_rn(s_ref[i], c) - cM) * LN2_64, s_table);
        };
        double S = 0.0;
        for (uint32_t i0 = 0; i0 < parts * RECS; i0 += 32) {
            double v = i0 + lane < parts * RECS ? relative(i0 + lane) : 0.0;
#pragma unroll
            for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
            S += v;
        }
        bool settled = false;
        const bool number = S > 0.0 && S < 1e300 && !far_out(M, c);
        if (M == -inf && S == 0.0) {
            if (part == 0 && tid == 0) put_sample(o, r, -1, -inf, -inf, 0);
            settled = true;
        } else if (number) {
            const float mean = POWER_ERROR * (__log2f((float)q.V / (float)S) + 3.1f);  // (of what a weight's power of two costs; the references add up to 3)
            const double eps = (double)((16.0f + mean) * 0x1p-24f);
            // what a border between two parts of S is known to
            const double slack = S * (double)(0x1p-24f * (8.0f * u * (1.0f - u) + mean * fmaxf(u, 1.0f - u) + 24.0f * u + 4.0f));
            const float L = max_nan(logf((float)S), 0.0f);
            if (!RULES) {
                // the segment that the number falls into, and what lies in front of it
                const double at = (double)u * S;
                double before = 0.0;
                uint32_t mine = 0xFFFFFFFFu;
                for (uint32_t i0 = 0; i0 < parts * RECS && mine == 0xFFFFFFFFu; i0 += 32) {
                    const double own = i0 + lane < parts * RECS ? relative(i0 + lane) : 0.0;
                    double up = own;
#pragma unroll
                    for (int d = 1; d < 32; d *= 2) {
                        const double v = __shfl_up_sync(0xffffffffu, up, d);
                        if (lane >= (uint32_t)d) up += v;
                    }
                    const uint32_t past = __ballot_sync(0xffffffffu, before + up > at);
                    const uint32_t f = past ? __ffs(past) - 1 : 31;
                    if (past) mine = i0 + f;
                    const double front = __shfl_sync(0xffffffffu, past ? up - own : up, f);
                    before += front;
                }
                if (mine == 0xFFFFFFFFu) mine = 0;  // (not found: nothing is found there either)
                if (mine / RECS == part) {  // its block reads it again, in the order of the numbers
                    if (tid == 0) s_found[0] = 0;
                    __syncthreads();
                    const uint32_t w = mine % RECS / LD_SEGS, a = min(p1, p0 + w * per), b = min(p1, a + per);
                    const uint32_t from = min(b, a + (mine % LD_SEGS) * seg_steps * LD_STEP), to = min(b, from + seg_steps * LD_STEP);
                    const double back = exp_below_1(((double)__fmul_rn(M, c) - cM) * LN2_64, s_table);
                    find_in_segment<T, MASKED, NT>(q, o, Segment{r, from, to, count, before, at, slack, back, M, L}, s_sums, s_found);
                    if (tid == 0) s.left[r] = s_found[0] ? 0u : ordered(M);
                }
                meet();
                continue;
            }
            // the bound
            const float range = fminf(M - low, 64.0f / q.scale), width = range * (1.0f / LD_BINS);
            const float each = width > 1e-30f ? 1.0f / width : 0.0f;
            if (s.top_k || s.top_p < 1.0) {
#pragma unroll
                for (uint32_t seg = 0; seg < LD_SEGS; ++seg) {
                    const float d = M - to_f32(s_most[RULES ? seg : 0][RULES ? tid : 0]);
                    if (d <= range) {
                        const uint32_t bin = RULES ? min(LD_BINS - 1, (uint32_t)(d * each)) : 0;
                        atomicAdd(&s_bins[bin], 1u);
                        if (!s.top_k) atomicAdd(&s_mass[bin], (uint32_t)(ex2(-d * c) * 0x1p18f));
                    }
                }
            }
            meet();
            if (CLUSTER) {  // of all the blocks (the own bins may still be asked for by others: the sums lie where the ring was)
                uint32_t n = 0, m = 0;
#pragma unroll
                for (uint32_t p = 0; p < MAX_PARTS; ++p)
                    if (p < parts) {
                        n += *away(&s_bins[RULES ? tid : 0], p);
                        m += *away(&s_mass[RULES ? tid : 0], p);
                    }
                reinterpret_cast<uint32_t *>(buffer)[tid] = n;
                reinterpret_cast<uint32_t *>(buffer)[LD_BINS + tid] = m;
                __syncthreads();
            }
            const uint32_t *const bins = CLUSTER ? reinterpret_cast<uint32_t *>(buffer) : s_bins, *const mass = CLUSTER ? bins + LD_BINS : s_mass;
            const float from = fmaxf(__double2float_ru((double)M + s.drop), LOWEST);  // of min_p
            if (warp == 0) {
                float bound = LOWEST;
                if (s.top_k || s.top_p < 1.0) {
                    constexpr uint32_t PER = LD_BINS / 32;
                    uint32_t n[PER], m[PER], n_own = 0, m_own = 0;
#pragma unroll
                    for (uint32_t i = 0; i < PER; ++i) {
                        n_own += n[i] = bins[lane * PER + i];
                        m_own += m[i] = mass[lane * PER + i];
                    }
                    uint32_t n_up = n_own, m_up = m_own;
#pragma unroll
                    for (int d = 1; d < 32; d *= 2) {
                        const uint32_t a = __shfl_up_sync(0xffffffffu, n_up, d), b = __shfl_up_sync(0xffffffffu, m_up, d);
                        if (lane >= (uint32_t)d) { n_up += a; m_up += b; }
                    }
                    n_up -= n_own;
                    m_up -= m_own;
                    const float need = (float)(s.top_p * S) * 0x1p18f;
                    // no group counted in a bin or above it has a largest logit below the bin's lower end
                    auto end_of = [&](uint32_t bin) { return M - (float)(bin + 1) * width * (1.0f + 0x1p-20f) - fabsf(M) * 0x1p-22f; };
                    const uint32_t m_all = __shfl_sync(0xffffffffu, m_up + m_own, 31);
                    float sure = -inf, guess = -inf;
#pragma unroll
                    for (uint32_t i = 0; i < PER; ++i) {
                        n_up += n[i];
                        m_up += m[i];
                        if (sure == -inf && (s.top_k ? n_up >= s.top_k : (float)m_up >= need)) sure = end_of(lane * PER + i);
                        if (guess == -inf && (m_up >= m_all - (m_all >> 6) || n_up > LD_GUESS)) guess = n_up <= LD_GUESS ? end_of(lane * PER + i) : inf;
                    }
                    // the weights of a group's other entries are not counted: where the largest ones alone are not enough, what reaches the
                    // groups that have nearly all of these may be; if they are many, the row is broad, and nothing is listed
                    uint32_t reached = __ballot_sync(0xffffffffu, sure > -inf);
                    if (!reached && !s.top_k) {
                        reached = __ballot_sync(0xffffffffu, guess > -inf);
                        sure = guess;
                    }
                    if (reached) bound = fmaxf(__shfl_sync(0xffffffffu, sure, __ffs(reached) - 1), LOWEST);
                }
                // (with both, the first top_k are listed whole: top_p is of their sum)
                if (!(s.top_k && s.top_p < 1.0)) bound = fmaxf(bound, from);
                if (lane == 0) s_bound = bound;
            }
            __syncthreads();
            const float bound = s_bound;
            const bool all = s.min_p == 0.0 || bound != from;  // (else min_p decides what is listed)
            // the groups that reach it, and of these the entries
            uint16_t *const groups = reinterpret_cast<uint16_t *>(buffer + K::GROUPS_AT);
#pragma unroll 1
            for (uint32_t seg = 0; seg < LD_SEGS; ++seg)
                if (to_f32(s_most[RULES ? seg : 0][RULES ? tid : 0]) >= bound) groups[atomicAdd(&s_n[1], 1u)] = (uint16_t)(seg * NT + tid);
            __syncthreads();
            const uint32_t vectors = seg_steps * U, items = s_n[1] * vectors;
            key_t64 *list = reinterpret_cast<key_t64 *>(buffer);
            for (uint32_t i0 = tid; i0 < items; i0 += 4 * NT) {
                uint4 raw[4];
                uint32_t at[4];
#pragma unroll
                for (uint32_t k = 0; k < 4; ++k) {
                    const uint32_t item = i0 + k * NT;
                    raw[k] = make_uint4(MINUS_INF2<T>, MINUS_INF2<T>, MINUS_INF2<T>, MINUS_INF2<T>);
                    at[k] = 0;
                    if (item < items) {
                        const uint32_t id = groups[item / vectors], of = item % vectors, seg = id / NT, t = id % NT;
                        const uint32_t a = min(p1, p0 + (t >> 5) * per), b = min(p1, a + per);
                        const uint32_t st = seg * seg_steps + of / U, v = a + st * LD_STEP + (of % U) * 32 + (t & 31);
                        if (v < b) {
                            at[k] = v;
                            raw[k] = open_vector<T, MASKED>(x, mask, v);
                        }
                    }
                }
#pragma unroll
                for (uint32_t k = 0; k < 4; ++k) {
                    if (!(vector_max(raw[k], T{}) >= bound)) continue;
                    float e[EPV<T>];
                    unpack(raw[k], e, T{});
#pragma unroll
                    for (int i = 0; i < EPV<T>; ++i)
                        if (e[i] >= bound) {
                            const uint32_t place = atomicAdd(&s_n[0], 1u);
                            if (place < K::CAP) list[place] = rank_key(e[i], (uint32_t)(x.first(at[k]) + i));
                        }
                }
            }
            __syncthreads();
            uint32_t n = s_n[0];
            if (CLUSTER) {  // to the first block
                if (tid == 0) s_base = atomicAdd(away(&s_n[2], 0), n);
                __syncthreads();
                key_t64 *const to = away(reinterpret_cast<key_t64 *>(buffer + K::WEIGHTS_AT), 0);
                for (uint32_t i = tid; i < min(n, K::CAP); i += NT)
                    if (s_base + i < K::CAP) to[s_base + i] = list[i];
                meet();
                n = s_n[2];
                list = reinterpret_cast<key_t64 *>(buffer + K::WEIGHTS_AT);
            }
            if (part == 0 && n <= K::CAP && n > 0) {
                const Listed a{q, s, o, s_table, r, u, M, from, L, S, eps, all};
                settled = n <= NT ? draw_few<NT>(a, list, n, buffer + K::GROUPS_AT, s_few)
                                  : draw_many<NT>(a, list, n, reinterpret_cast<double *>(buffer + (CLUSTER ? 0 : K::WEIGHTS_AT)),
                                              reinterpret_cast<key_t64 *>(buffer + K::GROUPS_AT), s_sums, s_found);
            }
        }
        if (part == 0 && tid == 0) s.left[r] = settled ? 0u : number ? ordered(M) : 1u;
        meet();
    }
}

// The rows that were left, each to a cluster of blocks, which works them out in 64 bits.
constexpr uint32_t RS_THREADS = 512, RS_BYTES = TEAM_HELD * RS_THREADS * 16 + 16 * RS_THREADS * 8;
template <typename T>
__global__ void __launch_bounds__(RS_THREADS) k_sample_rest(const LogitRows q, const SampleRules s, const SampleOut o, uint32_t log_parts)
{
    extern __shared__ __align__(16) uint4 s_held[];  // [TEAM_HELD][RS_THREADS], then [16][RS_THREADS] sums of 64 bits
    __shared__ TeamMemory<RS_THREADS> mem;
    __shared__ uint32_t s_warp[RS_THREADS / 32], s_row[RS_THREADS], s_known[RS_THREADS];
    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, parts = 1u << log_parts, part = blockIdx.x & (parts - 1);
    const uint32_t clusters = gridDim.x >> log_parts, me = blockIdx.x >> log_parts;
    if (tid < EXP_TABLE) mem.table[tid] = exp2((double)tid / EXP_TABLE);
    uint64_t number = 0;  // of rows left so far: cluster b takes every clusters-th from b on
    pdl_wait();
    if (parts > 1) cg::this_cluster().sync();  // (all blocks of the cluster run)
    else __syncthreads();
    for (uint64_t base = 0; base < q.n_rows; base += RS_THREADS) {
        const uint32_t known = base + tid < q.n_rows ? s.left[base + tid] : 0u;
        const bool left = known != 0;
        const uint32_t some = __ballot_sync(0xffffffffu, left);
        if (!__syncthreads_or(some)) continue;
        if (lane == 0) s_warp[warp] = __popc(some);
        __syncthreads();
        uint32_t front = __popc(some & ((1u << lane) - 1)), all = 0;
        for (uint32_t w = 0; w < RS_THREADS / 32; ++w) {
            if (w < warp) front += s_warp[w];
            all += s_warp[w];
        }
        // the first of these that is the cluster's, and how many are; in the same order in each of its blocks
        const uint32_t skip = (uint32_t)((me + clusters - number % clusters) % clusters), n = all > skip ? (all - skip - 1) / clusters + 1 : 0;
        if (left && front >= skip && (front - skip) % clusters == 0) {
            s_row[(front - skip) / clusters] = tid;
            s_known[(front - skip) / clusters] = known;
        }
        number += all;
        __syncthreads();
        for (uint32_t i = 0; i < n; ++i) {
            sample_row_64<T, RS_THREADS>(q, s, o, base + s_row[i], &mem, s_held, parts, part, s_known[i]);
            if (parts > 1) cg::this_cluster().sync();  // (the next row's first sums may go where this row's last ones are read)
            else __syncthreads();
        }
    }
}

template <typename T, bool MASKED, bool RULES, bool CLUSTER, uint32_t NT>
cudaError_t run_sample_long(const LogitRows &q, const SampleRules &s, const SampleOut &o, uint32_t log_parts, int device,
                            cudaStream_t st)
{
    constexpr auto kernel = k_sample_long<T, MASKED, RULES, CLUSTER, NT>;
    const cudaError_t e = allow_smem<kernel, (int)Long<NT>::RING_BYTES>(device);
    if (e != cudaSuccess) return e;
    const uint32_t parts = 1u << log_parts;
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = parts;
    at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.blockDim = NT; cfg.dynamicSmemBytes = Long<NT>::RING_BYTES; cfg.stream = st;
    cfg.attrs = &at; cfg.numAttrs = CLUSTER ? 1 : 0;
    const uint64_t most = (1ull << 30) >> log_parts;
    cfg.gridDim = dim3((uint32_t)((q.n_rows < most ? q.n_rows : most) * parts));
    g_vl_launches.fetch_add(1);
    return cudaLaunchKernelEx(&cfg, kernel, q, s, o, log_parts);
}

constexpr uint32_t SMALL_ROWS = 2048;  // vectors
template <typename T, bool MASKED, bool RULES>
cudaError_t launch_sample_long(const LogitRows &q, const SampleRules &s, const SampleOut &o, int device, cudaStream_t st)
{
    const uint32_t n = q.V / EPV<T>;
    uint32_t log_parts = 0;
    const uint64_t sms = (uint64_t)vl_device_sm_count(device);
    // Blocks of a row: more of them shorten the pass and cost barriers of 1 us; they pay where most multiprocessors would be idle and a block
    // keeps 4,096 vectors (2,048 for a handful of rows).  Device time in us with 1, 2, 4, 8 blocks, bf16, top_k 50 and top_p 0.9: one row of 131,072
    // 29, 26, 20, 18; 100 rows 33, 30, 26, 28; 300 rows 40, 39, 51, 69; 100 rows of 32,768 18.6, 21, 21, 24.  With 4,096 and with 2,048, top_p 0.95: one
    // row of 131,072 20.5, 18.4, eight 21.1, 19.3, 64 25.4, 25.3; one row of 32,768 14.8, 17.4.
    const uint32_t least = q.n_rows <= 8 ? 2048 : 4096;
    while ((1u << log_parts) < LD_PARTS && q.n_rows << (log_parts + 1) <= sms * 3 && n >> (log_parts + 1) >= least) ++log_parts;
    // One warp at a row where a row is short and there are rows for all the places: it has no barriers, and 28 rows are at their ends at once
    // instead of seven (5,000 rows of 8,192 bf16 logits 76 us with four warps at each, 57 with one; 4,000 of 32,768 98 and 155).  It has a quarter of
    // the groups and of the list, which a large top_k does not fit: 5,000 of 8,192 with top_k 50, 100, 150, 200, 300 59, 117, 273, 1,197, 1,211 with one,
    // 81, 130, 177, 218, 1,219 with four.
    const bool small = n <= SMALL_ROWS && q.n_rows >= 4 * sms;
    const cudaError_t e = log_parts ? run_sample_long<T, MASKED, RULES, true, 128>(q, s, o, log_parts, device, st)
                          : small   ? run_sample_long<T, MASKED, RULES, false, 32>(q, s, o, 0, device, st)
                                    : run_sample_long<T, MASKED, RULES, false, 128>(q, s, o, 0, device, st);
    if (e != cudaSuccess) return e;
    constexpr auto rest = k_sample_rest<T>;
    if (const cudaError_t f = allow_smem<rest, (int)RS_BYTES>(device); f != cudaSuccess) return f;
    // Blocks at a row: where few rows can be left, or a thread would have more than eight vectors of it.  A pass over a row takes a block 2 us and
    // more whatever the row is, and a cluster another 1: 5,000 rows of 8,192 bf16 logits of which a third is left take
    // 213 us with one block at each, 953 with four.  Few broad rows of 131,072 bf16 logits, four blocks and eight: one row 66, 55, eight 71, 55, twelve 74,
    // 59, sixteen (for which there is no room at once) 75, 92.
    const uint32_t log_rest = q.n_rows <= 8 && n >= 2048 ? 3 : n < 4096 ? 0 : n < 8192 ? 1 : 2;
    const uint64_t clusters = (uint64_t)vl_device_sm_count(device) >> log_rest;
    cudaLaunchAttribute at[2]{};
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = 1u << log_rest;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((uint32_t)(q.n_rows < clusters ? q.n_rows : clusters) << log_rest);
    cfg.blockDim = RS_THREADS; cfg.dynamicSmemBytes = RS_BYTES; cfg.stream = st;
    cfg.attrs = at; cfg.numAttrs = 2;
    g_vl_launches.fetch_add(1);
    return cudaLaunchKernelEx(&cfg, rest, q, s, o, log_rest);
}

template <typename T>
cudaError_t launch_sample_long(const LogitRows &q, const SampleRules &s, const SampleOut &o, int device, cudaStream_t st)
{
    if (!s.left) return cudaErrorInvalidValue;  // (vl_sample_work is 0 for short rows alone)
    const bool masked = q.occupied || q.widths;
    if (s.top_k || s.top_p < 1.0 || s.min_p > 0.0)
        return masked ? launch_sample_long<T, true, true>(q, s, o, device, st) : launch_sample_long<T, false, true>(q, s, o, device, st);
    return masked ? launch_sample_long<T, true, false>(q, s, o, device, st) : launch_sample_long<T, false, false>(q, s, o, device, st);
}

}  // namespace
