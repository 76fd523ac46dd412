// The kernels of vl_token_sample for f16 logits (a file per type: they compile side by side).
#include "vl_sample_launch.cuh"

cudaError_t vl_sample_f16(const LogitRows &q, const SampleRules &s, const SampleOut &o, int device, cudaStream_t st)
{
    return launch_sample<__half>(q, s, o, device, st);
}
