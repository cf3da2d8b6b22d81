// kd_attention_4bit's kernels for heads of up to 64 channels.
#include "kd_attn4.cuh"

cudaError_t kd::attn4::launch_small(const Params& p, int nc, int gs, int nt, int grid, cudaStream_t s) {
  if (nc == 1) return nt == 1 ? launch<1, 1>(p, gs, grid, s) : launch<1, 2>(p, gs, grid, s);
  return nt == 1 ? launch<2, 1>(p, gs, grid, s) : launch<2, 2>(p, gs, grid, s);
}
