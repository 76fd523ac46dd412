// The kernels of vl_token_logprobs for f16 logits (a file per type: they compile side by side).
#include "vl_logprob.cuh"

cudaError_t vl_scores_f16(const LogitRows &q, const ScoreOut &o, int device, cudaStream_t st) { return launch_scores<__half>(q, o, device, st); }
