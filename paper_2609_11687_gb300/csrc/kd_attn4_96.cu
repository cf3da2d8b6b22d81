// kd_attention_4bit's kernels for heads of up to 96 channels.
#include "kd_attn4.cuh"

cudaError_t kd::attn4::launch_96(const Params& p, int gs, int nt, int grid, cudaStream_t s) {
  return nt == 1 ? launch<3, 1>(p, gs, grid, s) : launch<3, 2>(p, gs, grid, s);
}
