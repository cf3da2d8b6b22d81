// Helpers shared by the serving operators (kd_norm.cu, kd_weight4.cu, kd_mat4*.cu,
// kd_logprob.cu): typed loads and stores, NaN-keeping maxima, argument checks.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "kashin.h"

namespace kd {
namespace serve {

inline bool float_type(int d) { return d == KD_F32 || d == KD_F16 || d == KD_BF16; }
inline int64_t type_bytes(int d) { return d == KD_F32 ? 4 : d == KD_E4M3 ? 1 : 2; }
inline bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
// every row of `ld` elements of type d starts on a 16-byte boundary
inline bool rows_aligned16(const void* p, int64_t ld, int64_t rows, int d) {
  return aligned(p, 16) && (rows <= 1 || ld * type_bytes(d) % 16 == 0);
}

// Programmatic dependent launch: a kernel launched with launch_early may be set up while the
// one before it in the stream still runs; depend_on_last, before its first access to
// global memory, waits for that one's end and results, and lets the next be set up in turn.
// What a kernel takes of its SM but its launch (tensor memory) it takes between the two
// (wait_for_last, let_next_start): taken earlier it may be what the kernel before still wants, taken
// later the next one's CTAs may hold it.
inline void launch_early(cudaLaunchAttribute& a) {
  a.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  a.val.programmaticStreamSerializationAllowed = 1;
}
__device__ __forceinline__ void wait_for_last() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void depend_on_last() {
  wait_for_last();
  let_next_start();
}

// this CTA's rank in its cluster, the cluster's index, the launch's clusters (CTAs without one
// are clusters of their own)
enum { kRank, kCluster, kClusters };
template <int WHAT>
__device__ __forceinline__ int special() {
  int r;
  if constexpr (WHAT == kRank) asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  else if constexpr (WHAT == kCluster) asm("mov.u32 %0, %%clusterid.x;" : "=r"(r));
  else asm("mov.u32 %0, %%nclusterid.x;" : "=r"(r));
  return r;
}

__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

template <int DT>
struct Elem;
template <>
struct Elem<KD_F32> {
  using type = float;
  static __device__ __forceinline__ float get(float v) { return v; }
  static __device__ __forceinline__ float put(float v) { return v; }
};
template <>
struct Elem<KD_F16> {
  using type = __half;
  static __device__ __forceinline__ float get(__half v) { return __half2float(v); }
  static __device__ __forceinline__ __half put(float v) { return __float2half_rn(v); }
};
template <>
struct Elem<KD_BF16> {
  using type = __nv_bfloat16;
  static __device__ __forceinline__ float get(__nv_bfloat16 v) { return __bfloat162float(v); }
  static __device__ __forceinline__ __nv_bfloat16 put(float v) { return __float2bfloat16_rn(v); }
};

// two 16-bit values of one word as floats
template <int DT>
__device__ __forceinline__ float2 unpack2(uint32_t w) {
  if constexpr (DT == KD_F16) return __half22float2(*reinterpret_cast<const __half2*>(&w));
  else return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
template <int DT>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  if constexpr (DT == KD_F16) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  } else {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
}

// eight consecutive elements to a 16-byte boundary
template <int DT>
__device__ __forceinline__ void store8(void* base, int64_t at, const float (&v)[8]) {
  if constexpr (DT == KD_F32) {
    float4* p = reinterpret_cast<float4*>(static_cast<float*>(base) + at);
    p[0] = make_float4(v[0], v[1], v[2], v[3]);
    p[1] = make_float4(v[4], v[5], v[6], v[7]);
  } else {
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(base) + at) =
        make_uint4(pack2<DT>(v[0], v[1]), pack2<DT>(v[2], v[3]), pack2<DT>(v[4], v[5]), pack2<DT>(v[6], v[7]));
  }
}
template <int DT>
__device__ __forceinline__ float load1(const void* base, int64_t at) {
  return Elem<DT>::get(static_cast<const typename Elem<DT>::type*>(base)[at]);
}
template <int DT>
__device__ __forceinline__ void store1(void* base, int64_t at, float v) {
  static_cast<typename Elem<DT>::type*>(base)[at] = Elem<DT>::put(v);
}
__device__ __forceinline__ float load1_any(const void* base, int dt, int64_t at) {
  return dt == KD_F32 ? load1<KD_F32>(base, at) : dt == KD_F16 ? load1<KD_F16>(base, at) : load1<KD_BF16>(base, at);
}
__device__ __forceinline__ void store1_any(void* base, int dt, int64_t at, float v) {
  if (dt == KD_F32) store1<KD_F32>(base, at, v);
  else if (dt == KD_F16) store1<KD_F16>(base, at, v);
  else store1<KD_BF16>(base, at, v);
}

}  // namespace serve
}  // namespace kd
