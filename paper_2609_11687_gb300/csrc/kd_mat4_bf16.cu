// kd_matmul_4bit's kernels for bf16 activations.
#include "kd_mat4.cuh"

cudaError_t kd::mat4::launch_bf16(const Params& p, int gs, cudaStream_t s) { return launch<kBf16>(p, gs, s); }
