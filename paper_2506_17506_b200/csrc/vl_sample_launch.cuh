// Which kernel draws from which rows.
#pragma once
#include "vl_sample_long.cuh"

namespace {

template <typename T>
cudaError_t launch_sample(const LogitRows &q, const SampleRules &s, const SampleOut &o, int device, cudaStream_t st)
{
    bool aligned;
    const uint32_t n = row_vectors(q, sizeof(T), &aligned);
    const bool masked = q.occupied || q.widths;
    if (masked ? (aligned ? launch_sample_short<T, true, true>(q, s, o, n, st) : launch_sample_short<T, true, false>(q, s, o, n, st))
               : (aligned ? launch_sample_short<T, false, true>(q, s, o, n, st) : launch_sample_short<T, false, false>(q, s, o, n, st)))
        return cudaGetLastError();
    if (!s.left) return cudaErrorInvalidValue;  // (vl_sample_work is 0 for short rows alone)
    if (s.top_k || s.top_p < 1.0 || s.min_p > 0.0)
        return masked ? launch_sample_long<T, true, true>(q, s, o, device, st) : launch_sample_long<T, false, true>(q, s, o, device, st);
    return masked ? launch_sample_long<T, true, false>(q, s, o, device, st) : launch_sample_long<T, false, false>(q, s, o, device, st);
}

}  // namespace
