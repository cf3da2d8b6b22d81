// kd_matmul_4bit's kernels for groups of 32 inputs.
#include "kd_mat4_wide.cuh"

cudaError_t kd::mat4::launch_group32(const Params& p, bool bf, int nt, int clusters, cudaStream_t s) {
  if (!nt) return bf ? launch_wide<true, 1>(p, s) : launch_wide<false, 1>(p, s);
  return bf ? launch<true, 1>(p, nt, clusters, s) : launch<false, 1>(p, nt, clusters, s);
}
