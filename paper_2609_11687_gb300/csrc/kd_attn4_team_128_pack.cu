// kd_attention_4bit's kernels for heads of up to 128 channels, an item to a cluster, blocks of four rows.
#include "kd_attn4.cuh"

cudaError_t kd::attn4::launch_team_128_pack(const Params& p, int nc, int gs, int grid, cudaStream_t s) {
  return nc == 1   ? launch<1, true, true>(p, gs, grid, s)
         : nc == 2 ? launch<2, true, true>(p, gs, grid, s)
         : nc == 3 ? launch<3, true, true>(p, gs, grid, s)
                   : launch<4, true, true>(p, gs, grid, s);
}
