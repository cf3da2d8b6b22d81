// kd_matmul_4bit's kernels for e4m3 activations.
#include "kd_mat4.cuh"

cudaError_t kd::mat4::launch_e4m3(const Params& p, int gs, cudaStream_t s) { return launch<kE4M3>(p, gs, s); }
