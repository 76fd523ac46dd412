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
// 4,096 rows of 131,072, against 164 us for their bytes in bf16) and about five more instructions, of which those on pairs of
// numbers (f32x2) and of 16-bit halves do two elements at once.
#pragma once
#include <cooperative_groups.h>

#include "vl_rank.cuh"

namespace {

namespace cg = cooperative_groups;
// The lanes' sums together, relative to the lanes' largest m.
__device__ __forceinline__ void warp_join(Sums &a, float m, float c)
{
    raise(a, from_ordered(__reduce_max_sync(0xffffffffu, ordered(m))), c);
    a.s = warp_sum(a.s);
    a.t = warp_sum(a.t);
}
// The entries of vectors into the sums relative to m.
template <typename T, int N>
__device__ __forceinline__ void add_vectors(const uint4 (&raw)[N], float m, float c, f32x2 &s, f32x2 &t)
{
    m = m == __int_as_float(0xFF800000) ? 0.0f : m;  // (nothing but impossible entries, whose powers of two are 0 relative to anything)
    if (!far_out(m, c)) {
        const float b = -__fmul_rn(m, c);
        const f32x2 c2 = both(c, c), low = both(b, b);
#pragma unroll
        for (int u = 0; u < N; ++u) {
            float x[EPV<T>];
            unpack(above<T>(raw[u]), x, T{});
#pragma unroll
            for (int j = 0; j < EPV<T>; j += 2) {
                f32x2 y = fma2(both(x[j], x[j + 1]), c2, low);
                float y0, y1;
                apart(y, y0, y1);
                if (!BOUNDED<T>) {
                    y0 = max_nan(y0, FAR_BELOW);
                    y1 = max_nan(y1, FAR_BELOW);
                    y = both(y0, y1);
                }
                const f32x2 e = both(ex2(y0), ex2(y1));
                s = add2(s, e);
                t = fma2(e, y, t);
            }
        }
    } else {
#pragma unroll
        for (int u = 0; u < N; ++u) {
            float x[EPV<T>];
            unpack(raw[u], x, T{});
#pragma unroll
            for (int j = 0; j < EPV<T>; j += 2) {
                const float y0 = max_nan((x[j] - m) * c, FAR_BELOW), y1 = max_nan((x[j + 1] - m) * c, FAR_BELOW);
                const f32x2 e = both(ex2(y0), ex2(y1));
                s = add2(s, e);
                t = fma2(e, both(y0, y1), t);
            }
        }
    }
}

// A thread's state over the vectors of its stripe.  Its sums are relative to the largest logit it had met when a logit last was more than
// 8 powers of two above the one before: nearly always to the first vectors' largest, so that the rest has nothing to scale.
struct Run {
    float ref, limit, m;  // what the sums are relative to; what a logit has to pass for another one; the largest
    f32x2 s, t;
    uint32_t best;  // vector in which m was met first
};
template <typename T, int N, bool TOP>
__device__ __forceinline__ void take(Run &a, const uint4 (&raw)[N], uint32_t v, uint32_t step, float c, float margin)
{
    const float m = vectors_max<N>(raw, T{});
    if (TOP) {
        if (m > a.m) {
#pragma unroll
            for (int u = N - 1; u >= 0; --u)
                if (vector_max(raw[u], T{}) == m) a.best = v + u * step;
        }
    }
    a.m = fmaxf(a.m, m);
    if (m > a.limit) {
        const float d = step_down(a.ref, m, c), f = ex2(d);
        a.t = mul2(fma2(a.s, both(d, d), a.t), both(f, f));
        a.s = mul2(a.s, both(f, f));
        a.ref = m;
        a.limit = m + margin;
    }
    add_vectors<T, N>(raw, a.ref, c, a.s, a.t);
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

// ---- long rows
// Clusters of thread blocks, each at a row at a time and then at the next one; a block has a run of the row's vectors, a thread every
// NT-th of it.  Each thread copies its own vectors into its own places of shared memory, RING - 1 groups of U ahead, over the end of a
// row into the next one: the loads go on while a row is summed up, and take no registers.  (What a thread copies it alone reads: no
// barrier.)  The warps' sums of a row meet in one of the cluster's blocks and are summed up there by one warp, another one for every
// row; nobody waits for it: there are two sets of places, and a cluster barrier whose two halves are a row apart.
// Small blocks, eight to a multiprocessor: what a warp does once per row weighs less with four warps at a row than with sixteen
// (bf16, 4,096 rows of 131,072 185 us and 198 with blocks of 512 threads when this was chosen, 180 now: 5.9 TB/s; 1,200 rows of 8,000 12
// and 22).  592 rows of 1,000,000 take 203 us, 5.8 TB/s.
constexpr int LONG_THREADS = 128, LONG_U = 4, LONG_RING = 3, LONG_PARTS = 8;
constexpr int long_smem(int threads) { return threads * LONG_U * LONG_RING * 16; }

__device__ __forceinline__ void copy_vector(uint32_t to, const uint4 *from)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_close() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// A block's part of a row: vectors v0 .. v1 - 1.  The first and the last vector of a row may reach into its neighbours; they are
// read whole all the same, but for the first of the first row and the last of the last one, which may reach out of the matrix.
template <typename T>
struct PartOfRow {
    RowVectors<T> x;
    uint32_t v0, v1, lo, hi;  // lo .. hi - 1 are copied
    __device__ __forceinline__ PartOfRow(const LogitRows &q, uint64_t r, uint32_t part, uint32_t log_parts)
        : x(static_cast<const T *>(q.x) + r * q.stride, q.V), v0(0), v1(x.n)
    {
        if (log_parts) {
            const uint32_t per = (x.n + (1u << log_parts) - 1) >> log_parts;
            v0 = min(x.n, part * per);
            v1 = min(x.n, v0 + per);
        }
        lo = r == 0 && x.lead ? max(v0, 1u) : v0;
        hi = r == q.n_rows - 1 ? min(v1, (x.lead + x.V) / EPV<T>) : v1;
    }
};

// The alternatives of a row: 32 groups of its threads have a best entry each, and the k-th best of these bounds the k-th best entry from
// below.  A thread whose best entry is below the bound has none of the k; the stripes of the others (about k of them) are read again
// (from L2), and what is no smaller than the bound is gathered in one block.  If that is more than fits (rows of many equal logits), the
// k-th best of what was gathered is a higher bound, and the stripes are read once more.
constexpr uint32_t CAND = 256, TOP_GROUPS = 32;
static_assert(LONG_PARTS * (LONG_THREADS / 32) <= TOP_GROUPS && VL_MAX_ALTERNATIVES <= TOP_GROUPS, "a group lies in a warp; as many groups as alternatives");

// The k-th best of the groups' keys.
__device__ __forceinline__ key_t64 bound_of(const key_t64 *keys, uint32_t top, uint32_t lane)
{
    const key_t64 mine = keys[lane];
    uint32_t rank = 0;
#pragma unroll 8
    for (uint32_t j = 0; j < 32; ++j) {
        const key_t64 other = __shfl_sync(0xffffffffu, mine, j);
        rank += other > mine || (other == mine && j < lane);
    }
    return __shfl_sync(0xffffffffu, mine, __ffs(__ballot_sync(0xffffffffu, rank == top - 1)) - 1);
}

// One warp: the k-th best of n keys (all different, n >= k).
__device__ __forceinline__ key_t64 kth_key(const key_t64 *keys, uint32_t n, uint32_t k, uint32_t lane)
{
    key_t64 found = 0;
    for (uint32_t i = lane; i < n; i += 32) {
        uint32_t rank = 0;
        for (uint32_t j = 0; j < n; ++j) rank += keys[j] > keys[i];
        if (rank == k - 1) found = keys[i];
    }
    for (int d = 16; d; d >>= 1) found = max(found, __shfl_xor_sync(0xffffffffu, found, d));
    return found;
}

template <typename T, bool MASKED, bool TOP, bool CLUSTER, int NT>
__global__ void __launch_bounds__(NT, 1024 / NT) k_score_long(const LogitRows q, const ScoreOut o, uint32_t log_of_parts)
{
    constexpr int U = LONG_U, RING = LONG_RING, NW = NT / 32, MAX_PARTS = CLUSTER ? LONG_PARTS : 1;
    const uint32_t log_parts = CLUSTER ? log_of_parts : 0;
    extern __shared__ uint4 s_ring[];  // [RING][U][NT]
    __shared__ float s_sums[2][MAX_PARTS * NW][3];
    __shared__ key_t64 s_keys[TOP ? TOP_GROUPS : 1], s_cand[TOP ? CAND : 1], s_bound;
    __shared__ uint32_t s_n[2];
    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, parts = 1u << log_parts, part = blockIdx.x & (parts - 1);
    const uint64_t step = gridDim.x >> log_parts;
    const float c = q.scale * LOG2E, inf = __int_as_float(0x7f800000);
    const float margin = 8.0f / c;
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(s_ring) + tid * 16;
    cg::cluster_group cluster = cg::this_cluster();
    auto away = [&](auto *p, uint32_t b) { return CLUSTER ? cluster.map_shared_rank(p, b) : p; };  // the same place in another block
    auto meet = [&]() {
        if (CLUSTER) { cluster_arrive(); cluster_wait(); }
        else __syncthreads();
    };
    if (CLUSTER) cluster_arrive();

    // The rows that count, in order; the token of the one behind is loaded a row early.  (The first row is taken before its token
    // is known.)
    struct Rows {
        uint64_t r;
        int64_t next;
    };
    auto move = [&](Rows &a, bool report) {
        for (;;) {
            a.r += step;
            if (a.r >= q.n_rows) return;
            const int64_t tok = a.next;
            a.next = a.r + step < q.n_rows ? row_token(q, a.r + step) : -1;
            if (tok >= 0) return;
            if (report && part == 0) empty_row(o, a.r, true, tid, NT);
        }
    };
    Rows ahead{blockIdx.x >> log_parts, 0}, now;
    ahead.next = ahead.r + step < q.n_rows ? row_token(q, ahead.r + step) : -1;
    now = ahead;
    // the copies
    const uint4 *from = nullptr;
    uint32_t v_next = 0, v_end = 0, lo = 0, hi = 0, slot_in = 0, slot_out = 0;
    auto open = [&]() {  // (a part may have no vectors)
        for (;;) {
            const PartOfRow<T> p(q, ahead.r, part, log_parts);
            from = p.x.at(0);
            v_next = p.v0; v_end = p.v1; lo = p.lo; hi = p.hi;
            if (v_next < v_end) return;
            move(ahead, true);
            if (ahead.r >= q.n_rows) return;
        }
    };
    auto copy_group = [&]() {
        if (v_next < v_end) {
            const uint32_t to = ring + slot_in * (U * NT * 16);
            const uint4 *at = from + v_next + tid;
            if (v_next >= lo && v_next + U * NT <= hi) {
#pragma unroll
                for (int u = 0; u < U; ++u) copy_vector(to + u * (NT * 16), at + u * NT);
            } else {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const uint32_t v = v_next + u * NT + tid;
                    if (v >= lo && v < hi) copy_vector(to + u * (NT * 16), at + u * NT);
                }
            }
            slot_in = slot_in + 1 == RING ? 0 : slot_in + 1;
            v_next += U * NT;
            if (v_next >= v_end) {
                move(ahead, true);
                if (ahead.r < q.n_rows) open();
            }
        }
        copies_close();
    };
    open();
#pragma unroll 1
    for (int i = 0; i < RING - 1; ++i) copy_group();

    uint32_t set = 0;
    bool waiting = true;  // for the other half of the barrier
    for (; now.r < q.n_rows; move(now, false)) {
        const uint64_t r = now.r;
        const int64_t tok = row_token(q, r);
        const PartOfRow<T> p(q, r, part, log_parts);
        const RowVectors<T> &x = p.x;
        const uint32_t groups = (p.v1 - p.v0 + U * NT - 1) / (U * NT);
        if (r < step && tok < 0) {  // the first row, after all not
            for (uint32_t g = 0; g < groups; ++g) {
                copies_wait<RING - 2>();
                slot_out = slot_out + 1 == RING ? 0 : slot_out + 1;
                copy_group();
            }
            if (part == 0) empty_row(o, r, true, tid, NT);
            continue;
        }
        const RowMask mask = row_mask(q, r);
        const uint32_t half = (set >> log_parts) & 1, block = set & (parts - 1);  // where the row is summed up, and by which warp
        const bool last = part == block && warp == ((set >> log_parts) & (NW - 1));
        float x_tok = 0.0f;
        if (last && lane == 0 && o.logprob) x_tok = to_f32(x.row[tok]);
        Run a{-inf, -inf, -inf, 0ull, 0ull, 0xFFFFFFFFu};
        const uint32_t whole0 = p.v0 == 0 && x.lead ? 1 : 0;  // groups of which every vector is whole
        const uint32_t whole1 = (min(p.v1, (x.lead + x.V) / EPV<T>) - p.v0) / (U * NT);
        for (uint32_t g = 0; g < groups; ++g) {
            copies_wait<RING - 2>();
            const uint32_t v = p.v0 + g * (U * NT) + tid;
            const uint4 *slot = s_ring + slot_out * (U * NT) + tid;
            slot_out = slot_out + 1 == RING ? 0 : slot_out + 1;
            if (g >= whole0 && g < whole1) {
                uint4 raw[U];
#pragma unroll
                for (int u = 0; u < U; ++u) raw[u] = slot[u * NT];
                copy_group();  // (into the places read a group ago)
                if (MASKED) {
#pragma unroll
                    for (int u = 0; u < U; ++u) close_entries<T>(raw[u], mask.closed_from(x.first(v + u * NT), EPV<T>));
                }
                take<T, U, TOP>(a, raw, v, NT, c, margin);
            } else {  // with the row's first or last vectors
                copy_group();
                const uint32_t rest = p.v1 - (v - tid);
#pragma unroll 1
                for (uint32_t u = 0; u < U && u * NT < rest; ++u) {
                    const uint32_t w = v + u * NT;
                    uint4 raw[1] = {make_uint4(MINUS_INF2<T>, MINUS_INF2<T>, MINUS_INF2<T>, MINUS_INF2<T>)};
                    if (w < p.v1) {
                        raw[0] = slot[u * NT];
                        if (w < p.lo || w >= p.hi) raw[0] = x.part(w);
                        uint32_t bits = MASKED ? mask.closed_from(x.first(w), EPV<T>) : 0u;
                        if (w == 0) bits |= (1u << x.lead) - 1;
                        if (w == x.n - 1) bits |= 0xFFu << (EPV<T> - (x.n * EPV<T> - x.lead - x.V));
                        if (bits) close_entries<T>(raw[0], bits & ((1u << EPV<T>) - 1));
                    }
                    take<T, 1, TOP>(a, raw, w, NT, c, margin);
                }
            }
        }

        float s0, s1, t0, t1;
        apart(a.s, s0, s1);
        apart(a.t, t0, t1);
        Sums w{a.ref, s0 + s1, t0 + t1};
        warp_join(w, a.m, c);
        if (CLUSTER && waiting) cluster_wait();  // the places have been read (at first: the blocks of the cluster run)
        if (lane == 0) {
            float *to = away(&s_sums[half][part * NW + warp][0], block);
            to[0] = w.m; to[1] = w.s; to[2] = w.t;
        }
        uint32_t n = 0;
        if (TOP) {
            // a key that the thread's best entry reaches, whatever its place in its vector; the best of each of the block's 32 / parts
            // groups, to every block
            const bool any = a.best < p.v1;
            const int in = any ? x.first(a.best) : 0;
            key_t64 k = any ? rank_key(a.m, (uint32_t)(in + EPV<T> - 1)) : 0ull;
            const uint32_t lanes = min(32u, (uint32_t)NW * parts);  // of a group within a warp
            for (uint32_t d = 1; d < lanes; d *= 2) k = max(k, __shfl_xor_sync(0xffffffffu, k, d));
            const uint32_t per_warp = 32 / lanes;
            for (uint32_t b = lane % lanes; b < parts; b += lanes)
                *away(&s_keys[TOP ? (part * NW + warp) * per_warp + lane / lanes : 0], b) = k;
            if (tid == 0) s_n[set & 1] = 0;
            meet();
            key_t64 bound = bound_of(s_keys, o.top, lane);
            uint32_t *const count = away(&s_n[set & 1], block);
            key_t64 *const cand = away(&s_cand[0], block);
            for (;;) {
                uint32_t left = __ballot_sync(0xffffffffu, any && rank_key(a.m, (uint32_t)max(in, 0)) >= bound);
                while (left) {
                    const uint32_t owner = warp * 32 + __ffs(left) - 1;
                    left &= left - 1;
                    for (uint32_t v = p.v0 + owner + lane * NT; v < p.v1; v += 32 * NT)
                        each_key<T>(fetch<T, MASKED>(x, mask, v), x.first(v), bound, [&](key_t64 e) {
                            const uint32_t at = atomicAdd(count, 1u);
                            if (at < CAND) cand[at] = e;
                        });
                }
                meet();
                n = *count;
                if (n <= CAND) break;
                meet();
                if (last) {
                    bound = kth_key(s_cand, CAND, o.top, lane);
                    if (lane == 0) s_n[set & 1] = 0;
                    if (lane < parts) *away(&s_bound, lane) = bound;
                }
                meet();
                bound = s_bound;
            }
            // the count has been read: the other half is before the next row, or at the end, where no block may leave while another
            // one reads its shared memory
            if (CLUSTER) cluster_arrive();
        } else {
            if (CLUSTER) {
                cluster_arrive();
                waiting = !last;
                if (last) cluster_wait();
            } else {
                __syncthreads();
            }
        }
        ++set;
        if (!last) continue;
        w = Sums{-inf, 0.0f, 0.0f};
        for (uint32_t i = lane; i < parts * NW; i += 32) {
            Sums b{s_sums[half][i][0], s_sums[half][i][1], s_sums[half][i][2]};
            const float m = fmaxf(w.m, b.m);
            raise(w, m, c);
            raise(b, m, c);
            w.s += b.s;
            w.t += b.t;
        }
        warp_join(w, w.m, c);
        if (w.s == 0.0f) {
            empty_row(o, r, false, lane, 32);
            continue;
        }
        float L, H;
        finish(w, c, &L, &H);
        if (lane == 0) {
            if (o.logprob) o.logprob[r] = MASKED && mask.is_closed((uint32_t)tok) ? -inf : log_odds(x_tok, w.m, q.scale) - L;
            if (o.entropy) o.entropy[r] = H;
            if (o.stats) *reinterpret_cast<float2 *>(o.stats + 2 * r) = make_float2(w.m, L);
        }
        if (TOP) {
            for (uint32_t i = lane; i < n; i += 32) {
                const key_t64 k = s_cand[i];
                uint32_t rank = 0;
                for (uint32_t j = 0; j < n; ++j) rank += s_cand[j] > k;
                if (rank < o.top) {
                    o.ids[r * o.top + rank] = (int32_t)key_place(k);
                    o.lps[r * o.top + rank] = log_odds(key_value(k), w.m, q.scale) - L;
                }
            }
            if (lane >= n && lane < o.top) { o.ids[r * o.top + lane] = -1; o.lps[r * o.top + lane] = -inf; }
        }
    }
    if (CLUSTER && waiting) cluster_wait();
}

// Clusters of 2^at blocks that run at once on the device (asked once).
template <auto kernel>
int long_clusters(int device, uint32_t at, const cudaLaunchConfig_t &cfg)
{
    static std::atomic<int> known[64][4];
    const bool keep = device >= 0 && device < 64;
    int n = keep ? known[device][at].load() : 0;
    if (n > 0) return n;
    if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess || n < 1) n = 1;
    if (keep) known[device][at].store(n);
    return n;
}

template <typename T, bool MASKED, bool TOP, bool CLUSTER, int NT>
cudaError_t run_long(const LogitRows &q, const ScoreOut &o, uint32_t log_parts, int device, cudaStream_t st)
{
    constexpr auto kernel = k_score_long<T, MASKED, TOP, CLUSTER, NT>;
    const cudaError_t e = allow_smem<kernel, long_smem(NT)>(device);
    if (e != cudaSuccess) return e;
    const uint32_t parts = 1u << log_parts;
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = parts;
    at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(parts); cfg.blockDim = NT; cfg.dynamicSmemBytes = long_smem(NT); cfg.stream = st;
    cfg.attrs = &at; cfg.numAttrs = CLUSTER ? 1 : 0;
    const uint64_t most = CLUSTER ? (uint64_t)long_clusters<kernel>(device, log_parts, cfg)
                                  : (1024 / NT) * (uint64_t)vl_device_sm_count(device);
    cfg.gridDim = dim3((uint32_t)((q.n_rows < most ? q.n_rows : most) * parts));
    g_vl_launches.fetch_add(1);
    return cudaLaunchKernelEx(&cfg, kernel, q, o, log_parts);
}

// Blocks of a row.  More of them shorten it and cost the cluster's barriers; they may not be more than run at once, and less than 2,048
// vectors (16 a thread) are worth a block only where most multiprocessors would be idle: us for 1, 2, 4, 8 blocks, bf16: one row of
// 131,072 15.4, 10.3, 7.3, 5.9; 100 rows 16.8, 13.4, 11.3, 11.4; 300 rows 23.7, 21.5, 21.5, 22.5; 100 rows of 32,000 7.5, 7.1, 6.4, 7.3;
// 300 rows 10.7, 11.3, 12.9, 15.8; 100 rows of 8,000 5.1, 5.8, 5.2, 5.9.
template <typename T, bool MASKED, bool TOP>
cudaError_t launch_long(const LogitRows &q, const ScoreOut &o, int device, cudaStream_t st)
{
    const uint64_t resident = (1024 / LONG_THREADS) * (uint64_t)vl_device_sm_count(device);
    const uint32_t n = q.V / EPV<T>;
    uint32_t log_parts = 0;
    if (n >= 2048)
        while ((1u << log_parts) < LONG_PARTS && q.n_rows << (log_parts + 1) <= (n >> (log_parts + 1) > 2048 ? resident : resident * 2 / 5))
            ++log_parts;
    if (log_parts == 1 && n < 8192) log_parts = 0;
    if (log_parts) return run_long<T, MASKED, TOP, true, LONG_THREADS>(q, o, log_parts, device, st);
    // half as many warps at a row where it is short and there are rows for all the places: us in blocks of 128 and of 64 threads, bf16: 16,000
    // rows of 5,000 65.7, 48.7; of 16,000 125, 104; of 32,000 196, 213; 1,200 rows of 9,000 11.1, 10.7; 600 rows 7.1, 7.4
    if (n <= 2048 && q.n_rows >= resident) return run_long<T, MASKED, TOP, false, LONG_THREADS / 2>(q, o, 0, device, st);
    return run_long<T, MASKED, TOP, false, LONG_THREADS>(q, o, 0, device, st);
}

// Short rows: a group of lanes per row, every logit read once into registers.

template <typename T, bool MASKED, bool TOP, bool ALIGNED, int G, int NV>
__global__ void __launch_bounds__(SHORT_WARPS * 32, short_blocks(NV)) k_score_short(const LogitRows q, const ScoreOut o)
{
    static_assert(!TOP || G == 32, "alternatives take the whole warp");
    __shared__ key_t64 s_cand[TOP ? SHORT_WARPS : 1][TOP ? SHORT_CAND : 1];
    __shared__ uint32_t s_n[SHORT_WARPS];
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane % G;
    const float c = q.scale * LOG2E, inf = __int_as_float(0x7f800000);
    const uint64_t step = (uint64_t)gridDim.x * SHORT_WARPS * (32 / G);
    for (uint64_t r0 = ((uint64_t)blockIdx.x * SHORT_WARPS + warp) * (32 / G); r0 < q.n_rows; r0 += step) {
        const uint64_t r = min(r0 + lane / G, q.n_rows - 1);
        const bool there = r0 + lane / G < q.n_rows;  // (the warp's last rows may not be: it works on the last one instead)
        const RowVectors<T> x(static_cast<const T *>(q.x) + r * q.stride, q.V);
        uint4 raw[NV];
        fetch_row<T, G, NV, ALIGNED>(raw, x, g, r != 0 && r != q.n_rows - 1);
        const int64_t tok = row_token(q, r);
        bool shut = false;
        if (MASKED) shut = close_row<T, G, NV, ALIGNED>(raw, x, row_mask(q, r), g, tok);
        float x_tok = 0.0f;
        if (g == 0 && o.logprob && tok >= 0) x_tok = to_f32(x.row[tok]);

        const float own = vectors_max<NV>(raw, T{});
        float m = own;
#pragma unroll
        for (int d = G / 2; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
        f32x2 s2 = 0ull, t2 = 0ull;
        add_vectors<T, NV>(raw, m, c, s2, t2);
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
        float L, H;
        finish(Sums{m, s, t}, c, &L, &H);
        const bool left = tok < 0, empty = s == 0.0f;
        if (g == 0 && there) {
            if (o.logprob) o.logprob[r] = left ? 0.0f : (empty || shut ? -inf : log_odds(x_tok, m, q.scale) - L);
            if (o.entropy) o.entropy[r] = left || empty ? 0.0f : H;
            if (o.stats)
                *reinterpret_cast<float2 *>(o.stats + 2 * r) = left ? make_float2(0.0f, 0.0f) : make_float2(empty ? -inf : m, L);
        }
        if (TOP) {
            const key_t64 k = warp_alternatives<T, NV>(raw, own, x, lane, o.top, s_cand[warp], &s_n[warp]);
            if (lane < o.top) {
                const bool one = k != 0 && !left;
                o.ids[r * o.top + lane] = one ? (int32_t)key_place(k) : -1;
                o.lps[r * o.top + lane] = one ? log_odds(key_value(k), m, q.scale) - L : -inf;
            }
        }
    }
}

// Whether the rows are short, and if so the launch.
template <typename T, bool MASKED, bool TOP, bool ALIGNED>
bool launch_short(const LogitRows &q, const ScoreOut &o, uint32_t n, cudaStream_t st)
{
    auto run = [&](auto g, auto v) {
        constexpr int G = decltype(g)::value, NV = decltype(v)::value;
        const uint64_t blocks = (q.n_rows + SHORT_WARPS * (32 / G) - 1) / (SHORT_WARPS * (32 / G));
        k_score_short<T, MASKED, TOP, ALIGNED, G, NV>
            <<<(uint32_t)(blocks < (1u << 30) ? blocks : (1u << 30)), SHORT_WARPS * 32, 0, st>>>(q, o);
        g_vl_launches.fetch_add(1);
    };
    if (short_shape<TOP, ALIGNED>(n, q.W, run)) return true;
    if (n > 512) return false;
    run(std::integral_constant<int, 32>{}, std::integral_constant<int, 16>{});
    return true;
}

template <typename T, bool MASKED, bool TOP>
cudaError_t launch(const LogitRows &q, const ScoreOut &o, int device, cudaStream_t st)
{
    bool aligned;
    const uint32_t n = row_vectors(q, sizeof(T), &aligned);
    if (aligned ? launch_short<T, MASKED, TOP, true>(q, o, n, st) : launch_short<T, MASKED, TOP, false>(q, o, n, st)) return cudaGetLastError();
    return launch_long<T, MASKED, TOP>(q, o, device, st);
}

template <typename T>
cudaError_t launch_scores(const LogitRows &q, const ScoreOut &o, int device, cudaStream_t st)
{
    if (q.occupied || q.widths) return o.top ? launch<T, true, true>(q, o, device, st) : launch<T, true, false>(q, o, device, st);
    return o.top ? launch<T, false, true>(q, o, device, st) : launch<T, false, false>(q, o, device, st);
}

}  // namespace
