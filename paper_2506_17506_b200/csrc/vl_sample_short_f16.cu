// The kernels of vl_token_sample for short rows of f16 logits (files of their own: they compile side by side).
#include "vl_sample_short.cuh"

bool vl_sample_short_f16(const LogitRows &q, const SampleRules &s, const SampleOut &o, cudaStream_t st) { return launch_sample_short<__half>(q, s, o, st); }
