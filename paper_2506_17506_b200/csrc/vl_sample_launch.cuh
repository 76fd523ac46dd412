// Which kernel draws from which rows.
#pragma once
#include <math.h>

#include "vl_sample_long.cuh"

namespace {

template <typename T>
cudaError_t launch_sample(const LogitRows &q, const SampleRules &s, const SampleOut &o, int device, cudaStream_t st)
{
    bool aligned;
    const uint32_t n = row_vectors(q, sizeof(T), &aligned);
    ShortRules h;
    h.drop = s.min_p > 0.0 ? log(s.min_p) / (double)q.scale : -INFINITY;
    h.eps = (float)((45.0 + 1.5 * log2((double)q.V + 1.0)) / 16777216.0);
    const bool masked = q.occupied || q.widths;
    if (masked ? (aligned ? launch_sample_short<T, true, true>(q, s, o, h, n, st) : launch_sample_short<T, true, false>(q, s, o, h, n, st))
               : (aligned ? launch_sample_short<T, false, true>(q, s, o, h, n, st) : launch_sample_short<T, false, false>(q, s, o, h, n, st)))
        return cudaGetLastError();
    if (!s.left) return cudaErrorInvalidValue;  // (vl_sample_work is 0 for short rows alone)
    if (s.top_k || s.top_p < 1.0 || s.min_p > 0.0)
        return masked ? launch_sample_long<T, true, true>(q, s, o, h, device, st) : launch_sample_long<T, false, true>(q, s, o, h, device, st);
    return masked ? launch_sample_long<T, true, false>(q, s, o, h, device, st) : launch_sample_long<T, false, false>(q, s, o, h, device, st);
}

}  // namespace
