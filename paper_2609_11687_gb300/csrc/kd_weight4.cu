// 4-bit weights with group scales at load time: kd_quantise_4bit makes them,
// kd_dequantise_4bit expands them.  32000 x 4096 takes 0.40 ms to quantise from fp16 (0.8 TB/s,
// floor 0.049) and 0.10 to 0.11 ms to expand to 16 bits or fp32 (3.2 and 5.6 TB/s).  Both are bound
// by instructions: 407 for a warp's 128 weights (84 % of the issue slots used, the integer pipe
// 66 % busy; six of a lane's steps are IEEE divisions, which reproducible codes want) and 195 for a
// warp's 256 (79 % and 59 %: a scale is looked up for each word).
//
// Quantisation: one warp takes 128 consecutive inputs of a channel, four per lane, so a
// group of 32, 64 or 128 is 8, 16 or 32 lanes: its extremes come from that many lanes'
// shuffles, and two lanes' codes make a word.  Every step is an IEEE operation in the
// order that kashin.h states, so codes and scales are reproducible bit for bit.
#include "kd_weight4.cuh"

namespace kd {
namespace {

using namespace serve;

struct QuantParams {
  const void* w;
  uint32_t* codes;
  void* scales;
  uint8_t* zeros;
  int64_t n, m, ld, words, chunks;
  int dtype, scale_dtype, group_log, vec;
};

// a / b, in 32 bits where both fit (with the groups by shifts: 0.41 ms instead of 0.44)
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
  return (a | b) >> 32 ? a / b : (int64_t)((uint32_t)a / (uint32_t)b);
}

__global__ void __launch_bounds__(256) quantise4_kernel(const __grid_constant__ QuantParams p) {
  const int lane = threadIdx.x & 31;
  const int64_t units = p.m * p.chunks;
  for (int64_t u = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); u < units; u += (int64_t)gridDim.x * 8) {
    const int64_t j = quotient(u, p.chunks);
    const int64_t i0 = (u - j * p.chunks) * 128 + 4 * lane;
    float v[4];
    float lo = __int_as_float(0x7F800000), hi = -lo;
    bool bad = false;
    const int64_t at0 = j * p.ld + i0;
    if (p.vec && i0 + 4 <= p.n) {
      if (p.dtype == KD_F32) {
        const float4 f = *reinterpret_cast<const float4*>(static_cast<const float*>(p.w) + at0);
        v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w;
      } else {
        const uint2 h = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(p.w) + at0);
        const float2 a = p.dtype == KD_F16 ? unpack2<KD_F16>(h.x) : unpack2<KD_BF16>(h.x);
        const float2 b = p.dtype == KD_F16 ? unpack2<KD_F16>(h.y) : unpack2<KD_BF16>(h.y);
        v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y;
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = i0 + e < p.n ? load1_any(p.w, p.dtype, at0 + e) : 0.f;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (i0 + e < p.n) {
        lo = fminf(lo, v[e]);
        hi = fmaxf(hi, v[e]);
        bad = bad || !isfinite(v[e]);
      }
    }
    const int lanes = 1 << (p.group_log - 2);
    for (int o = 1; o < lanes; o <<= 1) {
      lo = fminf(lo, __shfl_xor_sync(~0u, lo, o));
      hi = fmaxf(hi, __shfl_xor_sync(~0u, hi, o));
      bad = __shfl_xor_sync(~0u, (int)bad, o) || bad;
    }
    float s;
    if (p.zeros) {
      lo = fminf(lo, 0.f);
      hi = fmaxf(hi, 0.f);
      s = (hi - lo) / 15.f;
    } else {
      s = fmaxf(hi / 7.f, -lo / 8.f);
    }
    if (bad) s = __int_as_float(0x7FC00000);
    // The scale as it is stored is the scale that the codes are for.  It is rounded up: a scale
    // rounded down leaves the group wider than its 15 steps, and the ends that the codes' range
    // then cuts are off by up to 15 * 2^-8 of a step (bf16) more than the half step of all others.
    s = p.scale_dtype == KD_F16 ? __half2float(__float2half_ru(s)) : __bfloat162float(__float2bfloat16_ru(s));
    const bool usable = isfinite(s) && s > 0.f;
    float z = p.zeros ? 0.f : 8.f;
    if (p.zeros && usable) z = fminf(15.f, fmaxf(0.f, rintf(-lo / s)));
    uint32_t c = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float q = usable ? fminf(15.f, fmaxf(0.f, rintf(v[e] / s) + z)) : z;
      c |= (i0 + e < p.n ? (uint32_t)q : 0u) << (4 * e);
    }
    const uint32_t up = __shfl_down_sync(~0u, c, 1);
    const int64_t word = i0 / 8;
    if (!(lane & 1) && word < p.words) p.codes[j * p.words + word] = c | (up << 16);
    if ((lane & (lanes - 1)) == 0 && i0 < p.n) {
      const int64_t at = (i0 >> p.group_log) * p.m + j;
      store1_any(p.scales, p.scale_dtype, at, s);
      if (p.zeros) p.zeros[at] = (uint8_t)z;
    }
  }
}

struct DequantParams {
  const uint32_t* codes;
  const void* scales;
  const uint8_t* zeros;
  void* out;
  int64_t n, m, ld, words;
  int dtype, scale_dtype, group_log, vec;
};

// one thread a code word: eight outputs
__global__ void __launch_bounds__(256) dequantise4_kernel(const __grid_constant__ DequantParams p) {
  const int64_t total = p.m * p.words;
  for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < total; u += (int64_t)gridDim.x * 256) {
    const int64_t j = quotient(u, p.words);
    const int64_t i0 = (u - j * p.words) * 8;
    if (i0 >= p.n) continue;
    const uint32_t c = p.codes[u];
    const int64_t at = (i0 >> p.group_log) * p.m + j;
    const float s = load1_any(p.scales, p.scale_dtype, at);
    const float z = p.zeros ? (float)p.zeros[at] : 8.f;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = s * ((float)((c >> (4 * e)) & 15u) - z);
    const int64_t o = j * p.ld + i0;
    if (p.vec && i0 + 8 <= p.n) {
      if (p.dtype == KD_F32) store8<KD_F32>(p.out, o, v);
      else if (p.dtype == KD_F16) store8<KD_F16>(p.out, o, v);
      else store8<KD_BF16>(p.out, o, v);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (i0 + e < p.n) store1_any(p.out, p.dtype, o + e, v[e]);
    }
  }
}

int log_of(int group) { return group == 32 ? 5 : group == 64 ? 6 : 7; }
unsigned grid_for(int64_t ctas) { return (unsigned)(ctas < (1 << 20) ? ctas : 1 << 20); }

}  // namespace
}  // namespace kd

extern "C" kd_status kd_quantise_4bit(const void* w, kd_dtype dtype, int64_t ld, const kd_weight4* out,
                                      void* stream) {
  using namespace kd;
  if (!weight4_sizes_ok(out) || !float_type(dtype) || ld < out->n) return KD_ERR_INVALID_ARG;
  if (out->m == 0) return KD_OK;
  if (!w || !aligned(w, (size_t)type_bytes(dtype)) || !weight4_pointers_ok(out)) return KD_ERR_INVALID_ARG;
  QuantParams p{w, const_cast<uint32_t*>(out->codes), const_cast<void*>(out->scales),
                const_cast<uint8_t*>(out->zeros), out->n, out->m, ld, weight4_words(out->n),
                (out->n + 127) / 128, (int)dtype, out->scale_dtype, log_of(out->group),
                rows_aligned16(w, ld, out->m, dtype)};
  quantise4_kernel<<<grid_for((p.m * p.chunks + 7) / 8), 256, 0, static_cast<cudaStream_t>(stream)>>>(p);
  return cudaGetLastError() == cudaSuccess ? KD_OK : KD_ERR_CUDA;
}

extern "C" kd_status kd_dequantise_4bit(const kd_weight4* w, kd_dtype out_dtype, void* out, int64_t ld,
                                        void* stream) {
  using namespace kd;
  if (!weight4_sizes_ok(w) || !float_type(out_dtype) || ld < w->n) return KD_ERR_INVALID_ARG;
  if (w->m == 0) return KD_OK;
  if (!out || !aligned(out, (size_t)type_bytes(out_dtype)) || !weight4_pointers_ok(w)) return KD_ERR_INVALID_ARG;
  DequantParams p{w->codes, w->scales, w->zeros, out, w->n, w->m, ld, weight4_words(w->n),
                  (int)out_dtype, w->scale_dtype, log_of(w->group),
                  rows_aligned16(out, ld, w->m, out_dtype)};
  dequantise4_kernel<<<grid_for((p.m * p.words + 255) / 256), 256, 0, static_cast<cudaStream_t>(stream)>>>(p);
  return cudaGetLastError() == cudaSuccess ? KD_OK : KD_ERR_CUDA;
}
