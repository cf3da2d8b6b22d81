// kd_attention_4bit's kernels for heads of up to 256 channels.
#include "kd_attn4.cuh"

cudaError_t kd::attn4::launch_256(const Params& p, int gs, cudaStream_t s) { return launch<8, 1>(p, gs, s); }
