// The kernels of vl_token_logprobs for bf16 logits (a file per type: they compile side by side).
#include "vl_logprob.cuh"

cudaError_t vl_scores_bf16(const LogitRows &q, const ScoreOut &o, int device, cudaStream_t st) { return launch_scores<__nv_bfloat16>(q, o, device, st); }
