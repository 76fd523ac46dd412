// The kernels of vl_token_logprobs for f32 logits (a file per type: they compile side by side).
#include "vl_logprob.cuh"

cudaError_t vl_scores_f32(const LogitRows &q, const ScoreOut &o, int device, cudaStream_t st) { return launch_scores<float>(q, o, device, st); }
