// The kernels of vl_token_sample for long rows of f32 logits (files of their own: they compile side by side).
#include "vl_sample_long.cuh"

cudaError_t vl_sample_f32(const LogitRows &q, const SampleRules &s, const SampleOut &o, int device, cudaStream_t st)
{
    return vl_sample_short_f32(q, s, o, st) ? cudaGetLastError() : launch_sample_long<float>(q, s, o, device, st);
}
