// kd_attention_4bit's kernels for heads of up to 128 channels, in equal shares, blocks of four rows.
#include "kd_attn4.cuh"

cudaError_t kd::attn4::launch_shares_128_pack(const Params& p, int nc, int gs, int grid, cudaStream_t s) {
  return nc == 1   ? launch<1, false, true>(p, gs, grid, s)
         : nc == 2 ? launch<2, false, true>(p, gs, grid, s)
         : nc == 3 ? launch<3, false, true>(p, gs, grid, s)
                   : launch<4, false, true>(p, gs, grid, s);
}
