// kd_attention_4bit's kernels for heads of 129 to 256 channels, an item to a cluster, blocks of eight rows.
#include "kd_attn4.cuh"

cudaError_t kd::attn4::launch_team_256(const Params& p, int nc, int gs, int grid, cudaStream_t s) {
  return nc == 5   ? launch<5, true, false>(p, gs, grid, s)
         : nc == 6 ? launch<6, true, false>(p, gs, grid, s)
         : nc == 7 ? launch<7, true, false>(p, gs, grid, s)
                   : launch<8, true, false>(p, gs, grid, s);
}
