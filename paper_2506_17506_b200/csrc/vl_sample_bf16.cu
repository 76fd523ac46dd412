// The kernels of vl_token_sample for bf16 logits (a file per type: they compile side by side).
#include "vl_sample_launch.cuh"

cudaError_t vl_sample_bf16(const LogitRows &q, const SampleRules &s, const SampleOut &o, int device, cudaStream_t st)
{
    return launch_sample<__nv_bfloat16>(q, s, o, device, st);
}
