// kd_matmul_4bit: argument checks and the choice of the launch (kernels: kd_mat4.cuh).
#include "kd_mat4.cuh"

namespace kd {
namespace mat4 {
namespace {

constexpr int kPassRows = 32;

// CTAs that share a tile's inputs: enough CTAs for two on each of 152 SMs, as long as
// every warp keeps at least one chunk.
int split_of(int m, int chunks) {
  const int tiles = (m + kTile - 1) / kTile;
  int s = 1;
  while (s < 8 && tiles * s < 304 && chunks >= 2 * s * kWarps) s *= 2;
  return s;
}

}  // namespace
}  // namespace mat4
}  // namespace kd

extern "C" kd_status kd_matmul_4bit(const kd_weight4* w, const void* x, kd_dtype x_dtype, const float* x_scale,
                                    int64_t rows, int64_t ldx, void* y, kd_dtype y_dtype, int64_t ldy,
                                    void* stream) {
  using namespace kd;
  using namespace kd::mat4;
  if (!weight4_sizes_ok(w) || rows < 0 || (x_dtype != KD_F16 && x_dtype != KD_BF16 && x_dtype != KD_E4M3) ||
      !float_type(y_dtype) || ldx < w->n || ldy < w->m)
    return KD_ERR_INVALID_ARG;
  if (w->m == 0 || rows == 0) return KD_OK;
  const int64_t xb = type_bytes(x_dtype), yb = type_bytes(y_dtype);
  if (!x || !y || !weight4_pointers_ok(w) || !aligned(x, (size_t)xb) || !aligned(y, (size_t)yb) ||
      !aligned(x_scale, 4))
    return KD_ERR_INVALID_ARG;
  Params p{};
  p.codes = w->codes;
  p.scales = static_cast<const uint16_t*>(w->scales);
  p.zeros = w->zeros;
  p.ldx = ldx;
  p.ldy = ldy;
  p.n = (int)w->n;
  p.m = (int)w->m;
  p.groups = (int)((w->n + w->group - 1) / w->group);
  p.pieces = (int)((w->n + 31) / 32);
  p.chunks = (int)((w->n + kChunk - 1) / kChunk);
  p.split = split_of(p.m, p.chunks);
  p.per = (p.chunks + p.split - 1) / p.split;
  p.scale_bf16 = w->scale_dtype == KD_BF16;
  p.ydtype = (int)y_dtype;
  const size_t wide = x_dtype == KD_E4M3 ? 8 : 16;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  for (int64_t r0 = 0; r0 < rows; r0 += kPassRows) {
    p.rows = (int)(rows - r0 < kPassRows ? rows - r0 : kPassRows);
    p.x = static_cast<const uint8_t*>(x) + r0 * ldx * xb;
    p.xs = x_scale ? x_scale + r0 : nullptr;
    p.y = static_cast<uint8_t*>(y) + r0 * ldy * yb;
    p.xvec = aligned(p.x, wide) && (p.rows == 1 || ldx * xb % (int64_t)wide == 0);
    const int gs = w->group / 32;
    const cudaError_t e = x_dtype == KD_F16   ? launch_half(p, gs, s)
                          : x_dtype == KD_BF16 ? launch_bf16(p, gs, s)
                                               : launch_e4m3(p, gs, s);
    if (e != cudaSuccess || cudaGetLastError() != cudaSuccess) return KD_ERR_CUDA;
  }
  return KD_OK;
}
