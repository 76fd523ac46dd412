// What the kernels that score rows of logits and those that draw from them share: entries in order, sums of powers of two, the best entries
// of a row that a warp holds.
#pragma once
#include "vl_logits.cuh"

namespace {

typedef unsigned long long key_t64;

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

// ---- running sums
// In powers of two: y_i = c x_i - B with c = scale log2 e and B = c m rounded, m the largest logit so far; s = sum 2^y, t = sum 2^y y.
// One multiply-add makes y, and B being rounded makes no difference: it is the same B in every term, and what it lacks to c m (little,
// up to FAR_OUT) is put right once, at the end.  Where c m is larger, y is (x - m) c.
constexpr float FAR_BELOW = -1e30f;  // stands for minus infinity, whose 2^y y would be none: its power of two is 0 (scale >= 1e-6)
struct Sums {
    float m, s, t;
};
// What sums relative to m lack to sums relative to the larger m1, as a power of two.
__device__ __forceinline__ float step_down(float m, float m1, float c)
{
    const float B = __fmul_rn(m, c), B1 = __fmul_rn(m1, c);
    const bool far = far_out(m, c), far1 = far_out(m1, c);
    if (!far && !far1) return __fsub_rn(B, B1);
    // one of them is relative to c m itself: the other one's B lacks something to it
    const float lacks = (far ? 0.0f : __fmaf_rn(m, c, -B)) - (far1 ? 0.0f : __fmaf_rn(m1, c, -B1));
    return fmaxf((m - m1) * c - lacks, FAR_BELOW);
}
__device__ __forceinline__ void raise(Sums &a, float m, float c)
{
    const float d = step_down(a.m, m, c), f = ex2(d);
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
// L = ln sum exp(scale (x - m)), and the entropy: neither is below 0, whatever rounding makes of it (a ln p is not above 0); minus infinity
// for no entries.
__device__ __forceinline__ void finish(const Sums &a, float c, float *L, float *H)
{
    const float ln_s = logf(a.s);
    const float l = far_out(a.m, c) ? ln_s : fmaf(LN2, __fmaf_rn(-a.m, c, __fmul_rn(a.m, c)), ln_s);
    *L = a.s == 0.0f ? ln_s : max_nan(l, 0.0f);
    *H = max_nan(ln_s - LN2 * __fdividef(a.t, a.s), 0.0f);  // (s is between 1/2 and 2^31)
}

// scale (x - m); the halves' difference is a number where x - m is none, and as exact.
__device__ __forceinline__ float log_odds(float x, float m, float scale) { return (0.5f * x - 0.5f * m) * (2.0f * scale); }

constexpr uint32_t SHORT_WARPS = 8, SHORT_CAND = 128;

// The k-th largest of the lanes' values (0 if fewer lanes have one): value by value for few, sorted for many.
__device__ __forceinline__ uint32_t kth_value(uint32_t v, uint32_t k, uint32_t lane)
{
    if (k <= 8) {
        for (uint32_t found = 0;;) {
            const uint32_t most = __reduce_max_sync(0xffffffffu, v);
            found += __popc(__ballot_sync(0xffffffffu, v == most));
            if (found >= k || most == 0) return most;
            if (v == most) v = 0;
        }
    }
#pragma unroll
    for (uint32_t n = 2; n <= 32; n *= 2)
#pragma unroll
        for (uint32_t d = n / 2; d; d /= 2) {
            const uint32_t other = __shfl_xor_sync(0xffffffffu, v, d);
            v = ((lane & d) == 0) == ((lane & n) == 0) ? max(v, other) : min(v, other);
        }
    return __shfl_sync(0xffffffffu, v, k - 1);
}

// The best entries of a row that the whole warp holds (G = 32), one to a lane in order, as in the long rows: the k-th of the lanes' best bounds
// the k-th of all, what is no smaller is gathered, and if that is more than fits, the k-th of what was gathered is a higher bound.
// own: the lane's largest logit.
template <typename T, int NV>
__device__ __forceinline__ key_t64 warp_alternatives(const uint4 (&raw)[NV], float own, const RowVectors<T> &x, uint32_t lane, uint32_t top,
                                                     key_t64 *cand, uint32_t *n_cand)
{
    const float inf = __int_as_float(0x7f800000);
    key_t64 least = (key_t64)kth_value(own > -inf ? ordered(own) : 0u, top, lane) << 32;
    key_t64 best = 0;
    for (;;) {
        const float floor = fmaxf(least ? key_value(least) : -inf, LOWEST);  // (an impossible entry is none)
        if (lane == 0) *n_cand = 0;
        __syncwarp();
        if (own >= floor) {
            constexpr int AT_ONCE = 32 / EPV<T>;  // vectors whose entries are bits of a word
#pragma unroll
            for (int j0 = 0; j0 < NV; j0 += AT_ONCE) {
                uint32_t there = 0;
#pragma unroll
                for (int j = j0; j < NV && j < j0 + AT_ONCE; ++j) {
                    float e[EPV<T>];
                    unpack(raw[j], e, T{});
#pragma unroll
                    for (int i = 0; i < EPV<T>; ++i) there |= (uint32_t)(e[i] >= floor) << ((j - j0) * EPV<T> + i);
                }
                while (there) {  // one or two
                    const uint32_t b = __ffs(there) - 1, i = x.first(lane + 32 * (j0 + b / EPV<T>)) + b % EPV<T>;
                    there &= there - 1;
                    const key_t64 k = rank_key(to_f32(x.row[i]), i);  // (from L1)
                    if (k < least) continue;
                    const uint32_t at = atomicAdd(n_cand, 1u);
                    if (at < SHORT_CAND) cand[at] = k;
                }
            }
        }
        __syncwarp();
        const uint32_t n = *n_cand, kept = min(n, SHORT_CAND);
        if (n <= 32) {  // each to the lane of its rank
            const key_t64 mine = lane < n ? cand[lane] : 0ull;
            uint32_t rank = 0;
            for (uint32_t j = 0; j < n; ++j) rank += cand[j] > mine;
            if (lane < n) cand[32 + rank] = mine;
            __syncwarp();
            best = lane < n ? cand[32 + lane] : 0ull;
        } else {
            best = sort32(cand[lane], lane);
            for (uint32_t b = 32; b < kept; b += 32) best = merge32(best, sort32(b + lane < kept ? cand[b + lane] : 0ull, lane), lane);
        }
        __syncwarp();
        if (n <= SHORT_CAND) return best;
        least = __shfl_sync(0xffffffffu, best, top - 1);
    }
}

}  // namespace
