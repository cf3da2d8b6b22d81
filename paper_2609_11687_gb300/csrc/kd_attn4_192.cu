// kd_attention_4bit's kernels for heads of up to 192 channels.
#include "kd_attn4.cuh"

cudaError_t kd::attn4::launch_192(const Params& p, int gs, cudaStream_t s) { return launch<6, 1>(p, gs, s); }
