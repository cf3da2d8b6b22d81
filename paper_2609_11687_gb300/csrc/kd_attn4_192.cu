// kd_attention_4bit's kernels for heads of 129 to 192 channels.
#include "kd_attn4.cuh"

cudaError_t kd::attn4::launch_192(const Params& p, int nc, int gs, int grid, cudaStream_t s) {
  return nc == 5 ? launch<5, 1>(p, gs, grid, s) : launch<6, 1>(p, gs, grid, s);
}
