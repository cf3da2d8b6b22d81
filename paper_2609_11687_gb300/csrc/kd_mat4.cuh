// Products of few activation rows with 4-bit weights and group scales (kd_matmul_4bit):
//
//     y[r][j] = xs[r] sum_g s[j][g] sum_{i in g} (c[j][i] - z[j][g]) x[r][i]
//
// on the tensor cores with the weights as the mma's A operand (16 channels) and the
// activation rows as B (8 rows), so that 8 rows fill a tile.
//
// Mapping.  A CTA owns 32 channels; its eight warps, and the CTAs of a cluster, split the
// inputs into chunks of 128 and add their partial sums in a fixed order.  Per chunk a warp
// copies its 32 x 64 bytes of codes and its rows' inputs to its own ring of stages in
// shared memory (cp.async), so that several chunks are in flight and no barrier of the
// CTA stands in the loop.
//
// K order.  The product is a sum over inputs, so A and B may enumerate them in any common
// order.  Step q of a chunk covers inputs 32q .. 32q + 31; the lanes with t = lane % 4
// take code word 4q + t of their channel (inputs 32q + 8t .. + 7) and the same eight
// inputs of their row.
//
// Codes to operands.  16-bit inputs: a mask and a shift bring codes i and i + 4 of a word
// to the low bits of two halves, an OR makes them 1024 + c (fp16) or 128 + c (bf16), and
// one packed subtraction makes c - z: every step is exact.  e4m3 inputs: the byte c in
// 0..15 read as e4m3 is exactly c 2^-9 (subnormals and the first binade are evenly
// spaced), so a mask suffices; the byte 0x80 | z is -z 2^-9, and a second mma with it as A
// subtracts the zero point.
#pragma once
#include <cooperative_groups.h>

#include "kd_weight4.cuh"

namespace kd {
namespace mat4 {

using namespace serve;

constexpr int kWarps = 8;
constexpr int kThreads = 32 * kWarps;
constexpr int kTile = 32;    // output channels of a CTA: two m16 tiles
constexpr int kChunk = 128;  // inputs of a chunk

enum { kHalf = 0, kBf16 = 1, kE4M3 = 2 };

struct Params {
  const uint32_t* codes;
  const uint16_t* scales;
  const uint8_t* zeros;
  const uint8_t* x;
  const float* xs;
  void* y;
  int64_t ldx, ldy;
  int n, m, rows;
  int groups, pieces, chunks;  // per row: scales, 16-byte pieces of codes; chunks of 128 inputs
  int per;                     // chunks of one CTA of a cluster
  int split;                   // CTAs of a cluster
  int xvec, scale_bf16, ydtype;
};

template <int XK>
constexpr int x_bytes = XK == kE4M3 ? 1 : 2;
// 16-byte units of one stage of one warp: codes, then inputs
template <int XK, int NT>
constexpr int stage_units = 128 + NT * 64 * x_bytes<XK>;
template <int XK, int NT>
constexpr int stages = NT == 1 ? (XK == kE4M3 ? 4 : 3) : NT == 2 ? (XK == kE4M3 ? 3 : 2) : 2;
template <int XK, int NT>
constexpr size_t smem_bytes = (size_t)kWarps * stages<XK, NT> * stage_units<XK, NT> * 16;

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
// `bytes` of N from src, the rest of the N zero
template <int N>
__device__ __forceinline__ void copy_async(void* dst, const void* src, int bytes) {
  if constexpr (N == 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_addr(dst)), "l"(src), "r"(bytes) : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(smem_addr(dst)), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void wait_group() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

template <int XK>
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                    uint32_t b1) {
  if constexpr (XK == kHalf)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%0, %1, %2, %3};\n"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else if constexpr (XK == kBf16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%0, %1, %2, %3};\n"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%0, %1, %2, %3};\n"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// the zero point as the decode wants it: packed 1024 + z or 128 + z, or four bytes -z 2^-9
template <int XK>
__device__ __forceinline__ uint32_t zero_word(uint32_t z) {
  if constexpr (XK == kHalf) return (0x6400u + z) * 0x10001u;
  else if constexpr (XK == kBf16) return (0x4300u + z) * 0x10001u;
  else return (0x80u | z) * 0x01010101u;
}
// codes i and i + 4 of a word, less the zero point, as two 16-bit values
template <int XK>
__device__ __forceinline__ uint32_t code_pair(uint32_t w, int i, uint32_t zw) {
  if constexpr (XK == kHalf) {
    const uint32_t v = ((w >> (4 * i)) & 0x000F000Fu) | 0x64006400u;
    const __half2 d = __hsub2(*reinterpret_cast<const __half2*>(&v), *reinterpret_cast<const __half2*>(&zw));
    return *reinterpret_cast<const uint32_t*>(&d);
  } else {
    const uint32_t v = ((w >> (4 * i)) & 0x000F000Fu) | 0x43004300u;
    const __nv_bfloat162 d =
        __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&v), *reinterpret_cast<const __nv_bfloat162*>(&zw));
    return *reinterpret_cast<const uint32_t*>(&d);
  }
}

// GS: 32-input steps of a group (1, 2, 4); NT: 8-row tiles of one pass
template <int XK, int GS, int NT>
__global__ void __launch_bounds__(kThreads) mat4_kernel(const __grid_constant__ Params p) {
  constexpr int kStages = stages<XK, NT>, kUnits = stage_units<XK, NT>, kGroups = 4 / GS;
  constexpr int XB = x_bytes<XK>;
  extern __shared__ uint4 smem[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const int rank = p.split > 1 ? (int)(blockIdx.x % p.split) : 0;
  const int j0 = (int)(blockIdx.x / p.split) * kTile;
  const int c_end = min(p.chunks, (rank + 1) * p.per);
  uint4* ring = smem + warp * kStages * kUnits;

  // inputs of rows past the batch stay zero in every stage
  for (int st = 0; st < kStages; ++st)
#pragma unroll
    for (int j = 0; j < NT; ++j)
      if (8 * j + g >= p.rows)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          if constexpr (XB == 2) ring[st * kUnits + 128 + (j * 4 + q) * 32 + lane] = make_uint4(0, 0, 0, 0);
          else reinterpret_cast<uint2*>(ring + st * kUnits + 128)[(j * 4 + q) * 32 + lane] = make_uint2(0, 0);
        }

  auto issue = [&](int c, int st) {
    uint4* to = ring + st * kUnits;
    const int piece = 4 * c + t;  // of the row's codes
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = g + 8 * i, row = j0 + r;
      const bool in = row < p.m && piece < p.pieces;
      copy_async<16>(to + r * 4 + (t ^ ((r >> 1) & 3)),
                     p.codes + (in ? ((int64_t)row * p.pieces + piece) * 4 : 0), in ? 16 : 0);
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const int r = 8 * j + g;
      if (r < p.rows) {
        const uint8_t* xr = p.x + (int64_t)r * p.ldx * XB;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int k = c * kChunk + 32 * q + 8 * t;
          const int have = min(8, max(0, p.n - k));
          if constexpr (XB == 2) {
            uint4* slot = to + 128 + (j * 4 + q) * 32 + lane;
            if (p.xvec) {
              copy_async<16>(slot, xr + (have ? (int64_t)k * 2 : 0), 2 * have);
            } else {
              uint16_t v[8];
#pragma unroll
              for (int e = 0; e < 8; ++e) v[e] = e < have ? reinterpret_cast<const uint16_t*>(xr)[k + e] : (uint16_t)0;
              *slot = make_uint4(v[0] | (uint32_t)v[1] << 16, v[2] | (uint32_t)v[3] << 16,
                                 v[4] | (uint32_t)v[5] << 16, v[6] | (uint32_t)v[7] << 16);
            }
          } else {
            uint2* slot = reinterpret_cast<uint2*>(to + 128) + (j * 4 + q) * 32 + lane;
            if (p.xvec) {
              copy_async<8>(slot, xr + (have ? k : 0), have);
            } else {
              uint32_t v[2] = {0, 0};
#pragma unroll
              for (int e = 0; e < 8; ++e)
                if (e < have) v[e / 4] |= (uint32_t)xr[k + e] << (8 * (e % 4));
              *slot = make_uint2(v[0], v[1]);
            }
          }
        }
      }
    }
  };

  // this lane's four channels: scales and zero points of a chunk's groups
  int at[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) at[i] = min(j0 + g + 8 * i, p.m - 1);
  uint32_t sraw[4][kGroups], zraw[4][kGroups];
  auto fetch_scales = [&](int c) {
#pragma unroll
    for (int k = 0; k < kGroups; ++k) {
      const int gi = min(c * kGroups + k, p.groups - 1);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t o = (int64_t)at[i] * p.groups + gi;
        sraw[i][k] = p.scales[o];
        zraw[i][k] = p.zeros ? p.zeros[o] : 8u;
      }
    }
  };

  float acc[2][NT][4];
#pragma unroll
  for (int mt = 0; mt < 2; ++mt)
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[mt][j][e] = 0.f;

  int c = rank * p.per + warp;  // this warp's chunks: c, c + kWarps, ...
#pragma unroll
  for (int st = 0; st < kStages - 1; ++st) {
    if (c + st * kWarps < c_end) issue(c + st * kWarps, st);
    commit();
  }
  if (c < c_end) fetch_scales(c);

  for (int it = 0; c < c_end; ++it, c += kWarps) {
    const int ahead = c + (kStages - 1) * kWarps;
    if (ahead < c_end) issue(ahead, (it + kStages - 1) % kStages);
    commit();
    float sc[4][kGroups];
    uint32_t zw[4][kGroups];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int k = 0; k < kGroups; ++k) {
        sc[i][k] = p.scale_bf16 ? __uint_as_float(sraw[i][k] << 16) : __half2float(__ushort_as_half((unsigned short)sraw[i][k]));
        zw[i][k] = zero_word<XK>(zraw[i][k]);
      }
    if (c + kWarps < c_end) fetch_scales(c + kWarps);
    wait_group<kStages - 1>();
    __syncwarp();
    const uint4* from = ring + (it % kStages) * kUnits;
    const uint32_t* words = reinterpret_cast<const uint32_t*>(from);
    float part[2][NT][4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int k = q / GS;
      if (q % GS == 0) {
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
          for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) part[mt][j][e] = 0.f;
      }
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = g + 8 * i;
        w[i] = words[(r * 4 + (q ^ ((r >> 1) & 3))) * 4 + t];
      }
      if constexpr (XB == 2) {
        uint32_t b[NT][4];
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          const uint4 v = from[128 + (j * 4 + q) * 32 + lane];
          b[j][0] = __byte_perm(v.x, v.z, 0x5410);
          b[j][1] = __byte_perm(v.x, v.z, 0x7632);
          b[j][2] = __byte_perm(v.y, v.w, 0x5410);
          b[j][3] = __byte_perm(v.y, v.w, 0x7632);
        }
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t a0 = code_pair<XK>(w[2 * mt], 2 * h, zw[2 * mt][k]);
            const uint32_t a1 = code_pair<XK>(w[2 * mt + 1], 2 * h, zw[2 * mt + 1][k]);
            const uint32_t a2 = code_pair<XK>(w[2 * mt], 2 * h + 1, zw[2 * mt][k]);
            const uint32_t a3 = code_pair<XK>(w[2 * mt + 1], 2 * h + 1, zw[2 * mt + 1][k]);
#pragma unroll
            for (int j = 0; j < NT; ++j) mma<XK>(part[mt][j], a0, a1, a2, a3, b[j][2 * h], b[j][2 * h + 1]);
          }
      } else {
        uint32_t b[NT][2];
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          const uint2 v = reinterpret_cast<const uint2*>(from + 128)[(j * 4 + q) * 32 + lane];
          b[j][0] = __byte_perm(v.x, v.y, 0x6420);
          b[j][1] = __byte_perm(v.x, v.y, 0x7531);
        }
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
          const uint32_t a0 = w[2 * mt] & 0x0F0F0F0Fu, a1 = w[2 * mt + 1] & 0x0F0F0F0Fu;
          const uint32_t a2 = (w[2 * mt] >> 4) & 0x0F0F0F0Fu, a3 = (w[2 * mt + 1] >> 4) & 0x0F0F0F0Fu;
          const uint32_t z0 = zw[2 * mt][k], z1 = zw[2 * mt + 1][k];
#pragma unroll
          for (int j = 0; j < NT; ++j) {
            mma<XK>(part[mt][j], z0, z1, z0, z1, b[j][0], b[j][1]);
            mma<XK>(part[mt][j], a0, a1, a2, a3, b[j][0], b[j][1]);
          }
        }
      }
      if (q % GS == GS - 1) {
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
          for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              acc[mt][j][e] = __fmaf_rn(sc[2 * mt + e / 2][k], part[mt][j][e], acc[mt][j][e]);
      }
    }
    __syncwarp();  // every lane has read the stage before it is filled again
  }

  // the warps' sums, added in warp order; then the CTAs' of the cluster, in rank order
  wait_group<0>();
  __syncthreads();
  float* red = reinterpret_cast<float*>(smem);
  constexpr int kCols = 8 * NT, kStride = kTile + 1, kOut = kTile * kCols;
#pragma unroll
  for (int mt = 0; mt < 2; ++mt)
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        red[(warp * kCols + 8 * j + 2 * t + (e & 1)) * kStride + 16 * mt + g + 8 * (e >> 1)] = acc[mt][j][e];
  __syncthreads();
  float* sum = red;  // warp 0's part receives the CTA's sums
  for (int o = threadIdx.x; o < kOut; o += kThreads) {
    const int at0 = (o / kTile) * kStride + o % kTile;
    float s = red[at0];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) s += red[w * kCols * kStride + at0];
    sum[at0] = s;
  }
  auto finish = [&](int o, float s) {
    const int r = o / kTile, j = j0 + o % kTile;
    if (r >= p.rows || j >= p.m) return;
    if constexpr (XK == kE4M3) s *= 512.f;
    if (p.xs) s *= p.xs[r];
    store1_any(p.y, p.ydtype, (int64_t)r * p.ldy + j, s);
  };
  if (p.split == 1) {
    for (int o = threadIdx.x; o < kOut; o += kThreads) finish(o, sum[(o / kTile) * kStride + o % kTile]);
  } else {
    namespace cg = cooperative_groups;
    cg::cluster_group cl = cg::this_cluster();
    cl.sync();
    for (int o = rank * kThreads + threadIdx.x; o < kOut; o += p.split * kThreads) {
      const int at0 = (o / kTile) * kStride + o % kTile;
      float s = 0.f;
      for (int k = 0; k < p.split; ++k) s += cl.map_shared_rank(sum, k)[at0];
      finish(o, s);
    }
    cl.sync();  // no CTA leaves while its sums are read
  }
}

// the launch of one pass (at most 32 rows)
template <int XK, int GS, int NT>
cudaError_t launch_one(const Params& p, cudaStream_t s) {
  auto kernel = mat4_kernel<XK, GS, NT>;
  constexpr size_t bytes = smem_bytes<XK, NT>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((p.m + kTile - 1) / kTile * p.split));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = bytes;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)p.split;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, p);
}

template <int XK>
cudaError_t launch(const Params& p, int gs, cudaStream_t s) {
  const int nt = p.rows <= 8 ? 1 : p.rows <= 16 ? 2 : 4;
#define KD_MAT4(G, N) \
  if (gs == G && nt == N) return launch_one<XK, G, N>(p, s);
  KD_MAT4(1, 1) KD_MAT4(1, 2) KD_MAT4(1, 4) KD_MAT4(2, 1) KD_MAT4(2, 2) KD_MAT4(2, 4) KD_MAT4(4, 1) KD_MAT4(4, 2)
  KD_MAT4(4, 4)
#undef KD_MAT4
  return cudaErrorInvalidValue;
}

cudaError_t launch_half(const Params& p, int gs, cudaStream_t s);
cudaError_t launch_bf16(const Params& p, int gs, cudaStream_t s);
cudaError_t launch_e4m3(const Params& p, int gs, cudaStream_t s);

}  // namespace mat4
}  // namespace kd
