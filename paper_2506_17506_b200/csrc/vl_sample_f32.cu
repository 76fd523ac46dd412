// The kernels of vl_token_sample for f32 logits (a file per type: they compile side by side).
#include "vl_sample_launch.cuh"

cudaError_t vl_sample_f32(const LogitRows &q, const SampleRules &s, const SampleOut &o, int device, cudaStream_t st)
{
    return launch_sample<float>(q, s, o, device, st);
}
