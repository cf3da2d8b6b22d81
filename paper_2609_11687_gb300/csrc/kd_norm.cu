// Root-mean-square norm of rows with the residual's addition and 8-bit output:
//
//     h = x + r                                   (32 bits)
//     r' = round(h)                               (the new residual, optional)
//     y = h rsqrt(mean(h^2) + eps) w              (optional output, rounded to its type)
//     s = max|y| / 448,  q = e4m3(y / s)          (optional outputs; s = 1 where max|y| < 2^-100)
//
// One pass over the row: a thread keeps its elements of h and w in registers; a reduction
// over the row yields sum(h^2), another one the largest of |y| as it is rounded (the factor
// max|h w| from the first pass would save it, but its products overflow where y does not, and
// its scale is not y's in the last place), so x and r are read once and nothing is read again.
// q is the rounded quotient's own rounding; see Quotient for why few are divided.
//
// Bound by HBM for many rows, by latency for few.  A CTA walks rows: it keeps w, and loads
// its next row before it reduces this one, so that loads are in flight all the time (a CTA
// a row reached half of the bandwidth: most of its life is the reductions).  2048 x 4096 bf16 with
// a residual, e4m3 and bf16 rows: 15.2 us, 73 % of the measured copy rate (one IEEE division an
// element: 17.2); one row 2.3 us, 333 unaligned rows of 5003 6.6 us.  64 registers are what
// 1024 threads, the longest rows, leave each: instances of two pieces a thread spill 28 to 48 bytes
// (fp16 rows and weight none, fp32 112), unaligned ones 64 to 188 and of one piece 16 to 24.
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
  int ydtype;
};

__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
  const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
  const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
  return lo | (hi << 16);
}

// e4m3(v / scale) without a division for most: the reciprocal, 2^-21 to either side of which
// the products lie below and above the quotient (they round three times, 3 2^-24, the
// quotient once).  Where both round to the same byte so does all between them.
struct Quotient {
  float scale, below, above;
  __device__ __forceinline__ explicit Quotient(float s) : scale(s) {
    const float inv = 1.f / s;
    below = inv * (1.f - 0x1p-21f);
    above = inv * (1.f + 0x1p-21f);
  }
  __device__ __forceinline__ uint32_t four(float a, float b, float c, float d) const {
    const uint32_t lo = e4m3x4(a * below, b * below, c * below, d * below);
    const uint32_t hi = e4m3x4(a * above, b * above, c * above, d * above);
    if (lo == hi) return lo;
    return e4m3x4(a / scale, b / scale, c / scale, d / scale);
  }
};

// eight elements as they come: 16 bytes of a 16-bit type, 32 of fp32; without VEC one by one
template <int DT, bool VEC>
struct Piece {
  uint4 v[DT == KD_F32 ? 2 : 1];
  // element e is at index + e (VEC) or index + e * stride; nothing past n
  __device__ __forceinline__ void load(const void* base, int64_t row, int index, int stride, int n) {
    if constexpr (VEC) {
      if (index < n) {
        const uint4* p = reinterpret_cast<const uint4*>(static_cast<const char*>(base) + (row + index) * (DT == KD_F32 ? 4 : 2));
        v[0] = p[0];
        if constexpr (DT == KD_F32) v[1] = p[1];
        return;
      }
    }
    uint32_t u[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if constexpr (!VEC) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int i = index + e * stride;
        if (i < n) {
          if constexpr (DT == KD_F32) u[e] = static_cast<const uint32_t*>(base)[row + i];
          else u[e / 2] |= (uint32_t) static_cast<const uint16_t*>(base)[row + i] << (16 * (e % 2));
        }
      }
    }
    v[0] = make_uint4(u[0], u[1], u[2], u[3]);
    if constexpr (DT == KD_F32) v[1] = make_uint4(u[4], u[5], u[6], u[7]);
  }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    if constexpr (DT == KD_F32) {
      f[0] = __uint_as_float(v[0].x); f[1] = __uint_as_float(v[0].y);
      f[2] = __uint_as_float(v[0].z); f[3] = __uint_as_float(v[0].w);
      f[4] = __uint_as_float(v[1].x); f[5] = __uint_as_float(v[1].y);
      f[6] = __uint_as_float(v[1].z); f[7] = __uint_as_float(v[1].w);
    } else {
      const float2 a = unpack2<DT>(v[0].x), b = unpack2<DT>(v[0].y), c = unpack2<DT>(v[0].z), d = unpack2<DT>(v[0].w);
      f[0] = a.x; f[1] = a.y; f[2] = b.x; f[3] = b.y;
      f[4] = c.x; f[5] = c.y; f[6] = d.x; f[7] = d.y;
    }
  }
};

constexpr int kNormThreads = 1024;  // of a CTA at most: two pieces each cover the longest row

// blockDim = (threads of one row, rows of one CTA); C: 8-element pieces a thread holds.
// VEC: rows start on 16-byte boundaries and n is a multiple of 8, a piece is 8 consecutive
// elements; else the 8 elements of a piece lie blockDim.x apart (coalesced element loads).
template <int DT, int WT, int C, bool VEC>
__global__ void __launch_bounds__(kNormThreads) norm_kernel(const __grid_constant__ NormParams p) {
  __shared__ float sums[2][kNormThreads / 32];
  __shared__ uint32_t tops[kNormThreads / 32];
  const int tid = threadIdx.x, T = blockDim.x, n = (int)p.n;
  const int64_t step = (int64_t)gridDim.x * blockDim.y;
  auto index = [&](int c) { return VEC ? 8 * (c * T + tid) : 8 * c * T + tid; };
  depend_on_last();

  Piece<WT, VEC> w[C];
#pragma unroll
  for (int c = 0; c < C; ++c) w[c].load(p.w, 0, index(c), T, n);
  Piece<DT, VEC> x[C], r[C];
  auto fetch = [&](int64_t row) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      x[c].load(p.x, row * p.ldx, index(c), T, n);
      if (p.r) r[c].load(p.r, row * p.ldr, index(c), T, n);
    }
  };
  const int64_t first = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
  if (first < p.rows) fetch(first);
  int parity = 0;
  // the rows of a CTA take turns together: one past the last takes part in the barrier only
  for (int64_t row = first; row - threadIdx.y < p.rows; row += step, parity ^= 1) {
    const bool live = row < p.rows;
    float h[C][8];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      x[c].get(h[c]);
      if (p.r) {
        float v[8];
        r[c].get(v);
#pragma unroll
        for (int e = 0; e < 8; ++e) h[c][e] += v[e];
      }
    }
    if (row + step < p.rows) fetch(row + step);
    // the sum goes out here, not with y: there are stores in flight during the reductions
    if (p.r_out && live) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        if constexpr (VEC) {
          if (index(c) < n) store8<DT>(p.r_out, row * p.ldro + index(c), h[c]);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (index(c) + e * T < n) store1<DT>(p.r_out, row * p.ldro + index(c) + e * T, h[c][e]);
        }
      }
    }
    float ss = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) ss = __fmaf_rn(h[c][e], h[c][e], ss);
#pragma unroll
    for (int o = 16; o; o >>= 1) ss += __shfl_xor_sync(~0u, ss, o);
    // the warps of a row are consecutive: slots of one row stay together
    const int per = T >> 5, at = threadIdx.y * per;
    if (T > 32) {
      if ((tid & 31) == 0) sums[parity][at + (tid >> 5)] = ss;
      __syncthreads();
      ss = 0.f;
      for (int k = 0; k < per; ++k) ss += sums[parity][at + k];
    }
    const float nan = __int_as_float(0x7FC00000);
    // a row whose sum of squares is no finite number has no norm: NaN, not zeros
    const float rstd = isfinite(ss) ? 1.f / sqrtf(ss / (float)n + p.eps) : nan;
    uint32_t top = 0;  // the largest |y| as bits, whose order is the values' with NaN above all
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float v[8];
      w[c].get(v);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        h[c][e] = h[c][e] * rstd * v[e];
        top = max(top, __float_as_uint(h[c][e]) & 0x7FFFFFFFu);
      }
    }
    float scale = 1.f;
    if (p.q) {
      top = __reduce_max_sync(~0u, top);
      if (T > 32) {
        if ((tid & 31) == 0) tops[at + (tid >> 5)] = top;
        __syncthreads();
        top = __reduce_max_sync(~0u, (tid & 31) < per ? tops[at + (tid & 31)] : 0u);
      }
      const float amax = __uint_as_float(top);
      scale = amax < 0x1p-100f ? 1.f : amax / kE4M3Max;
    }
    if (!live) continue;

    if (p.scale && tid == 0) p.scale[row] = scale;
    const Quotient quotient(scale);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const float(&y)[8] = h[c];
      if constexpr (VEC) {
        const int i = index(c);
        if (i >= n) break;
        if (p.y) {
          if (p.ydtype == KD_F32) store8<KD_F32>(p.y, row * p.ldy + i, y);
          else if (p.ydtype == KD_F16) store8<KD_F16>(p.y, row * p.ldy + i, y);
          else store8<KD_BF16>(p.y, row * p.ldy + i, y);
        }
        if (p.q)
          *reinterpret_cast<uint2*>(p.q + row * p.ldq + i) =
              make_uint2(quotient.four(y[0], y[1], y[2], y[3]), quotient.four(y[4], y[5], y[6], y[7]));
      } else {
        uint32_t q[2];
        if (p.q) {
          q[0] = quotient.four(y[0], y[1], y[2], y[3]);
          q[1] = quotient.four(y[4], y[5], y[6], y[7]);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int i = index(c) + e * T;
          if (i >= n) break;
          if (p.y) store1_any(p.y, p.ydtype, row * p.ldy + i, y[e]);
          if (p.q) p.q[row * p.ldq + i] = (uint8_t)(q[e / 4] >> (8 * (e % 4)));
        }
      }
    }
  }
}

template <int DT, int WT, bool VEC>
cudaError_t launch(const NormParams& p, cudaStream_t s) {
  const int64_t pieces = (p.n + 7) / 8;
  // two pieces a thread once the rows fill the GPU; for few rows more threads are sooner done
  const bool many = p.rows > 4 * 152;
  const int C = pieces <= (many ? 32 : 512) ? 1 : 2;
  const int T = (int)(((pieces + C - 1) / C + 31) / 32 * 32);
  const int R = T <= 128 ? 256 / T : 1;
  const int64_t groups = (p.rows + R - 1) / R;
  const int64_t at_once = 152 * (int64_t)(1024 / (T * R));  // about 64 registers a thread
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(groups < at_once ? groups : at_once));
  cfg.blockDim = dim3(T, R);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  launch_early(attr[0]);
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return C == 1 ? cudaLaunchKernelEx(&cfg, norm_kernel<DT, WT, 1, VEC>, p)
                : cudaLaunchKernelEx(&cfg, norm_kernel<DT, WT, 2, VEC>, p);
}

template <int DT>
cudaError_t launch(const NormParams& p, int wt, bool vec, cudaStream_t s) {
  if (wt == DT) return vec ? launch<DT, DT, true>(p, s) : launch<DT, DT, false>(p, s);
  return vec ? launch<DT, KD_F32, true>(p, s) : launch<DT, KD_F32, false>(p, s);
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
               eps, (int)y_dtype};
  const bool vec = n % 8 == 0 && rows_aligned16(x, ldx, rows, dtype) && aligned(weight, 16) &&
                   (!residual || rows_aligned16(residual, ld_residual, rows, dtype)) &&
                   (!new_residual || rows_aligned16(new_residual, ld_new_residual, rows, dtype)) &&
                   (!q || (aligned(q, 8) && (rows == 1 || ldq % 8 == 0))) &&
                   (!y || rows_aligned16(y, ldy, rows, y_dtype));
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = dtype == KD_F32   ? launch<KD_F32>(p, weight_dtype, vec, s)
                        : dtype == KD_F16 ? launch<KD_F16>(p, weight_dtype, vec, s)
                                          : launch<KD_BF16>(p, weight_dtype, vec, s);
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? KD_OK : KD_ERR_CUDA;
}
