// kd_attention_4bit's kernels for heads of 193 to 256 channels.
#include "kd_attn4.cuh"

cudaError_t kd::attn4::launch_256(const Params& p, int nc, int gs, int grid, cudaStream_t s) {
  return nc == 7 ? launch<7, 1>(p, gs, grid, s) : launch<8, 1>(p, gs, grid, s);
}
