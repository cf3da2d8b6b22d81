// kd_attention_4bit's kernels for heads of up to 128 channels.
#include "kd_attn4.cuh"

cudaError_t kd::attn4::launch_128(const Params& p, int gs, int nt, int grid, cudaStream_t s) {
  return nt == 1 ? launch<4, 1>(p, gs, grid, s) : launch<4, 2>(p, gs, grid, s);
}
