// kd_matmul_4bit's kernels for groups of 128 inputs.
#include "kd_mat4_wide.cuh"

cudaError_t kd::mat4::launch_group128(const Params& p, bool bf, int nt, int clusters, cudaStream_t s) {
  if (!nt) return bf ? launch_wide<true, 4>(p, s) : launch_wide<false, 4>(p, s);
  return bf ? launch<true, 4>(p, nt, clusters, s) : launch<false, 4>(p, nt, clusters, s);
}
