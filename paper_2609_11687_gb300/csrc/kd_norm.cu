// Root-mean-square norm of rows with the residual's addition and 8-bit output:
//
//     h = x + r                                   (32 bits)
//     r' = round(h)                               (the new residual, optional)
//     y = h rsqrt(mean(h^2) + eps) w              (optional output, rounded to its type)
//     s = max|y| / 448,  q = e4m3(y / s)          (optional outputs; s = 1 where max|y| < 2^-100)
//
// One pass over the row: a thread keeps its elements of h and w in registers, and one
// reduction over the row yields both sum(h^2) and max|h w| (max|y| is that times the
// row's positive factor), so x and r are read once and nothing is read again.
#include <cuda_fp8.h>

#include "kd_serve.cuh"

namespace kd {
namespace {

using namespace serve;

constexpr int64_t kNormMaxN = 16384;
constexpr float kE4M3Max = 448.f;

struct NormParams {
  const void* x;
  const void* w;
  const void* r;
  void* r_out;
  uint8_t* q;
  float* scale;
  void* y;
  int64_t n, rows, ldx, ldr, ldro, ldq, ldy;
  float eps;
  int wdtype, ydtype;
};

__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
  const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
  const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
  return lo | (hi << 16);
}

// blockDim = (threads of one row, rows of one CTA); C: 8-element pieces a thread holds.
// VEC: rows start on 16-byte boundaries and n is a multiple of 8, a piece is 8 consecutive
// elements; else the 8 elements of a piece lie blockDim.x apart (coalesced element loads).
template <int DT, int C, bool VEC>
__global__ void __launch_bounds__(512) norm_kernel(const __grid_constant__ NormParams p) {
  __shared__ float red[2][16];
  const int tid = threadIdx.x, T = blockDim.x;
  const int64_t row_at = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
  const bool live = row_at < p.rows;
  const int64_t row = live ? row_at : p.rows - 1;
  const int n = (int)p.n;
  auto index = [&](int c, int e) { return VEC ? 8 * (c * T + tid) + e : (8 * c + e) * T + tid; };

  depend_on_last();
  float h[C][8], w[C][8];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    if constexpr (VEC) {
      const int i = index(c, 0);
      if (i < n) {
        load8<DT>(p.x, row * p.ldx + i, h[c]);
        if (p.wdtype == DT) load8<DT>(p.w, i, w[c]);
        else load8<KD_F32>(p.w, i, w[c]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) h[c][e] = w[c][e] = 0.f;
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int i = index(c, e);
        h[c][e] = i < n ? load1<DT>(p.x, row * p.ldx + i) : 0.f;
        w[c][e] = i >= n ? 0.f : p.wdtype == DT ? load1<DT>(p.w, i) : load1<KD_F32>(p.w, i);
      }
    }
  }
  if (p.r) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if constexpr (VEC) {
        const int i = index(c, 0);
        if (i < n) {
          float v[8];
          load8<DT>(p.r, row * p.ldr + i, v);
#pragma unroll
          for (int e = 0; e < 8; ++e) h[c][e] += v[e];
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int i = index(c, e);
          if (i < n) h[c][e] += load1<DT>(p.r, row * p.ldr + i);
        }
      }
    }
  }

  float ss = 0.f, big = 0.f;
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      ss = __fmaf_rn(h[c][e], h[c][e], ss);
      big = max_nan(big, fabsf(h[c][e] * w[c][e]));
    }
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    ss += __shfl_xor_sync(~0u, ss, o);
    big = max_nan(big, __shfl_xor_sync(~0u, big, o));
  }
  if (T > 32) {
    // the warps of a row are consecutive: slots of one row stay together
    const int warp = (threadIdx.y * T + tid) >> 5, per = T >> 5;
    if ((tid & 31) == 0) { red[0][warp] = ss; red[1][warp] = big; }
    __syncthreads();
    ss = big = 0.f;
    for (int k = 0; k < per; ++k) {
      ss += red[0][threadIdx.y * per + k];
      big = max_nan(big, red[1][threadIdx.y * per + k]);
    }
  }
  if (!live) return;

  const float nan = __int_as_float(0x7FC00000);
  // a row whose sum of squares is no finite number has no norm: NaN, not zeros
  const float rstd = isfinite(ss) ? 1.f / sqrtf(ss / (float)n + p.eps) : nan;
  const float amax = big * rstd;
  const float scale = amax < 0x1p-100f ? 1.f : amax / kE4M3Max;
  const float inv = 1.f / scale;
  if (p.scale && tid == 0) p.scale[row] = scale;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    if constexpr (VEC) {
      const int i = index(c, 0);
      if (i >= n) break;
      if (p.r_out) store8<DT>(p.r_out, row * p.ldro + i, h[c]);
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = h[c][e] * rstd * w[c][e];
      if (p.y) {
        if (p.ydtype == KD_F32) store8<KD_F32>(p.y, row * p.ldy + i, y);
        else if (p.ydtype == KD_F16) store8<KD_F16>(p.y, row * p.ldy + i, y);
        else store8<KD_BF16>(p.y, row * p.ldy + i, y);
      }
      if (p.q)
        *reinterpret_cast<uint2*>(p.q + row * p.ldq + i) =
            make_uint2(e4m3x4(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv),
                       e4m3x4(y[4] * inv, y[5] * inv, y[6] * inv, y[7] * inv));
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int i = index(c, e);
        if (i >= n) break;
        if (p.r_out) store1<DT>(p.r_out, row * p.ldro + i, h[c][e]);
        const float y = h[c][e] * rstd * w[c][e];
        if (p.y) store1_any(p.y, p.ydtype, row * p.ldy + i, y);
        if (p.q) p.q[row * p.ldq + i] = __nv_cvt_float_to_fp8(y * inv, __NV_SATFINITE, __NV_E4M3);
      }
    }
  }
}

template <int DT, bool VEC>
cudaError_t launch(const NormParams& p, cudaStream_t s) {
  const int64_t pieces = (p.n + 7) / 8;
  const int C = pieces <= 512 ? 1 : pieces <= 1024 ? 2 : 4;
  const int T = (int)(((pieces + C - 1) / C + 31) / 32 * 32);
  const int R = T <= 128 ? 256 / T : 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((p.rows + R - 1) / R));
  cfg.blockDim = dim3(T, R);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  launch_early(attr[0]);
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return C == 1   ? cudaLaunchKernelEx(&cfg, norm_kernel<DT, 1, VEC>, p)
         : C == 2 ? cudaLaunchKernelEx(&cfg, norm_kernel<DT, 2, VEC>, p)
                  : cudaLaunchKernelEx(&cfg, norm_kernel<DT, 4, VEC>, p);
}

}  // namespace
}  // namespace kd

extern "C" kd_status kd_rmsnorm(const void* x, kd_dtype dtype, int64_t n, int64_t rows, int64_t ldx,
                                const void* weight, kd_dtype weight_dtype, float eps, const void* residual,
                                int64_t ld_residual, void* new_residual, int64_t ld_new_residual, uint8_t* q,
                                int64_t ldq, float* scale, void* y, kd_dtype y_dtype, int64_t ldy, void* stream) {
  using namespace kd;
  if (n < 1 || n > kNormMaxN) return KD_ERR_UNSUPPORTED_N;
  if (rows < 0 || rows > INT32_MAX || !float_type(dtype) || (weight_dtype != dtype && weight_dtype != KD_F32) ||
      !(eps >= 0.f) || ldx < n || (residual && ld_residual < n) || (new_residual && (!residual || ld_new_residual < n)) ||
      (q && ldq < n) || (!q) != (!scale) || (y && (ldy < n || !float_type(y_dtype))))
    return KD_ERR_INVALID_ARG;
  if (rows == 0) return KD_OK;
  if (!x || !weight || (!q && !y)) return KD_ERR_INVALID_ARG;
  const size_t eb = (size_t)type_bytes(dtype);
  if (!aligned(x, eb) || !aligned(weight, (size_t)type_bytes(weight_dtype)) || !aligned(residual, eb) ||
      !aligned(new_residual, eb) || !aligned(scale, 4) || (y && !aligned(y, (size_t)type_bytes(y_dtype))))
    return KD_ERR_INVALID_ARG;
  NormParams p{x, weight, residual, new_residual, q, scale, y, n, rows, ldx, ld_residual, ld_new_residual, ldq, ldy,
               eps, (int)weight_dtype, (int)y_dtype};
  const bool vec = n % 8 == 0 && rows_aligned16(x, ldx, rows, dtype) && aligned(weight, 16) &&
                   (!residual || rows_aligned16(residual, ld_residual, rows, dtype)) &&
                   (!new_residual || rows_aligned16(new_residual, ld_new_residual, rows, dtype)) &&
                   (!q || (aligned(q, 8) && (rows == 1 || ldq % 8 == 0))) &&
                   (!y || rows_aligned16(y, ldy, rows, y_dtype));
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = dtype == KD_F32   ? (vec ? launch<KD_F32, true>(p, s) : launch<KD_F32, false>(p, s))
                        : dtype == KD_F16 ? (vec ? launch<KD_F16, true>(p, s) : launch<KD_F16, false>(p, s))
                                          : (vec ? launch<KD_BF16, true>(p, s) : launch<KD_BF16, false>(p, s));
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? KD_OK : KD_ERR_CUDA;
}
