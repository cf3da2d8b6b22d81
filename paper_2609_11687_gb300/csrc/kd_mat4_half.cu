// kd_matmul_4bit's kernels for half activations.
#include "kd_mat4.cuh"

cudaError_t kd::mat4::launch_half(const Params& p, int gs, cudaStream_t s) { return launch<kHalf>(p, gs, s); }
