// Head norm and rotary positions of queries and keys in one pass (kd_rope):
//
//     h = x rsqrt(mean(x^2) + eps) w                            (with a weight)
//     y_a = A (h_a cos - h_b sin),  y_b = A (h_b cos + h_a sin)   for the pairs (a, b)
//
// Angles.  A pair's frequency is a 64-bit fraction of a turn, and position times frequency
// modulo 2^64 is one integer product that drops whole turns exactly: position 10^6 is
// as exact as position 1, without 64-bit floating point and without a reduction.  The upper 32
// bits, rounded, go to sincospif as half-turns of 24 bits (off by 2^-26 + 2^-33 turns at most).
//
// Mapping.  A lane owns one slot of a head, the two 16-byte vectors whose channels turn
// together (or two that pass through), so that partners meet in registers; 8 lanes hold a head
// of 128 16-bit channels and a warp four heads.  The slot is the lane's own for all heads
// that it visits: the warp makes the token's sines and cosines once, in shared memory, and each lane
// keeps its own in registers.  A warp takes several heads of a token where there are many tokens,
// and one round of heads where there are few, so that one token's heads are spread over the GPU.
// Heads that do not start on 16-byte boundaries, or whose parts are no whole vectors, go pair by
// pair, a warp a head, and are read twice (the second time from L1).
//
// Bound by instructions: 2048 tokens of 32 + 8 heads of 128 bf16 channels, normed, take 10.5 us (42 MB, 4.0 TB/s; a
// plain copy of as much runs at 5.9), issue slots 63 % busy, 345 instructions for a warp's four heads.  One token's heads take 1.8 us,
// 333 tokens of 10 + 2 heads of 80 channels 1.9: latency.  Pair by pair the 2048 tokens take 41 us (one element further in
// memory; 32 without norms) or 48 (100 of 128 channels turned), 333 of them 9.4 and 11: an element a lane, each read twice.
#include <cmath>

#include "kd_serve.cuh"

namespace kd {
namespace {

using namespace serve;

constexpr int64_t kRopeMaxD = 1024, kRopeMaxHeads = 65535;
constexpr int kRopeWarps = 4;  // of a CTA

struct RopeSide {
  const void* x;
  void* y;
  const void* w;
  int64_t x_token, x_head, y_token, y_head;
  int heads, wt;
};
struct RopeParams {
  RopeSide side[2];
  const int64_t* positions;
  const uint64_t* turns;
  int tasks, parts, per;  // warps' worth of work: rounds of heads, `per` of them a part, `parts` a token
  int d, rot, half;       // half: pairs lie rot/2 apart
  int lanes_log;          // lanes of a head
  float amplitude, eps, inv_d;
};

// sine and cosine of pair i, times the amplitude
__device__ __forceinline__ float2 turn_of(const RopeParams& p, int64_t position, int i) {
  const uint64_t t = (uint64_t)position * p.turns[i];
  const int32_t top = (int32_t)(uint32_t)((t + 0x80000000ull) >> 32);
  float s, c;
  sincospif((float)top * 0x1p-31f, &s, &c);
  return make_float2(s * p.amplitude, c * p.amplitude);
}

template <int DT>
struct Vec16 {  // 16 bytes as they come, as P pairs of floats
  static constexpr int V = DT == KD_F32 ? 4 : 8, P = V / 2;
  static __device__ __forceinline__ void get(uint4 u, float2 (&f)[P]) {
    if constexpr (DT == KD_F32) {
      f[0] = make_float2(__uint_as_float(u.x), __uint_as_float(u.y));
      f[1] = make_float2(__uint_as_float(u.z), __uint_as_float(u.w));
    } else {
      f[0] = unpack2<DT>(u.x);
      f[1] = unpack2<DT>(u.y);
      f[2] = unpack2<DT>(u.z);
      f[3] = unpack2<DT>(u.w);
    }
  }
  static __device__ __forceinline__ uint4 put(const float2 (&f)[P]) {
    if constexpr (DT == KD_F32)
      return make_uint4(__float_as_uint(f[0].x), __float_as_uint(f[0].y), __float_as_uint(f[1].x), __float_as_uint(f[1].y));
    else return make_uint4(pack2<DT>(f[0].x, f[0].y), pack2<DT>(f[1].x, f[1].y), pack2<DT>(f[2].x, f[2].y), pack2<DT>(f[3].x, f[3].y));
  }
};

// consecutive weights from channel c on
template <int DT, int P>
__device__ __forceinline__ void load_weights(const RopeSide& s, int c, float2 (&w)[P]) {
  if (s.wt == KD_F32) {
#pragma unroll
    for (int e = 0; e < P; e += 2) {
      const float4 f = *reinterpret_cast<const float4*>(static_cast<const float*>(s.w) + c + 2 * e);
      w[e] = make_float2(f.x, f.y);
      w[e + 1] = make_float2(f.z, f.w);
    }
  } else {
    Vec16<DT>::get(*reinterpret_cast<const uint4*>(static_cast<const typename Elem<DT>::type*>(s.w) + c), w);
  }
}

// a root and a quotient, as kd_rmsnorm's (rsqrtf is off by two units in the last place, and saves 0.4 of a prompt's 10.5 us)
__device__ __forceinline__ float inverse_root(float sum, const RopeParams& p) {
  return isfinite(sum) ? 1.f / sqrtf(sum * p.inv_d + p.eps) : __int_as_float(0x7FC00000);
}

template <int DT>
__global__ void __launch_bounds__(32 * kRopeWarps) rope_kernel(const __grid_constant__ RopeParams p) {
  constexpr int V = Vec16<DT>::V, P = V / 2;
  using T = typename Elem<DT>::type;
  extern __shared__ float2 turns_of_warp[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int task = blockIdx.x * kRopeWarps + warp;
  depend_on_last();
  if (task >= p.tasks) return;
  const int token = task / p.parts, part = task - token * p.parts;
  const int slot = lane & ((1 << p.lanes_log) - 1), nth = lane >> p.lanes_log, heads_log = 5 - p.lanes_log;
  const int rotated = p.rot / (2 * V);
  // the channels of the slot's two vectors
  const int a = slot < rotated ? (p.half ? V * slot : 2 * V * slot) : p.rot + 2 * V * (slot - rotated);
  const int b = slot < rotated && p.half ? a + p.rot / 2 : a + V;
  const bool has_a = a < p.d, has_b = b < p.d;
  const int heads = p.side[0].heads + p.side[1].heads;

  uint4 va, vb;
  auto fetch = [&](int round) {
    const int h = (round << heads_log) + nth;
    va = vb = make_uint4(0, 0, 0, 0);
    if (h >= heads) return;
    const RopeSide& s = p.side[h >= p.side[0].heads];
    const T* x = static_cast<const T*>(s.x) + token * s.x_token + (h >= p.side[0].heads ? h - p.side[0].heads : h) * s.x_head;
    if (has_a) va = *reinterpret_cast<const uint4*>(x + a);
    if (has_b) vb = *reinterpret_cast<const uint4*>(x + b);
  };
  const int first = part * p.per, last = min(first + p.per, (heads + (1 << heads_log) - 1) >> heads_log);
  fetch(first);

  float2* table = turns_of_warp + warp * (p.rot / 2);
  const int64_t position = p.positions[token];
  for (int i = lane; i < p.rot / 2; i += 32) table[i] = turn_of(p, position, i);
  __syncwarp();
  // of the slot's pairs, two at a time
  float2 sine[P], cosine[P], minus_sine[P];
  if (slot < rotated) {
#pragma unroll
    for (int e = 0; e < P; ++e) {
      const float2 u = table[V * slot + 2 * e], v = table[V * slot + 2 * e + 1];
      sine[e] = make_float2(u.x, v.x);
      minus_sine[e] = make_float2(-u.x, -v.x);
      cosine[e] = make_float2(u.y, v.y);
    }
  }

  for (int round = first; round < last; ++round) {
    float2 fa[P], fb[P];
    Vec16<DT>::get(va, fa);
    Vec16<DT>::get(vb, fb);
    if (round + 1 < last) fetch(round + 1);
    const int h = (round << heads_log) + nth;
    const RopeSide& s = p.side[h >= p.side[0].heads];
    if (p.side[0].w || p.side[1].w) {
      float2 sums = make_float2(0.f, 0.f);
#pragma unroll
      for (int e = 0; e < P; ++e) sums = fma2(fa[e], fa[e], fma2(fb[e], fb[e], sums));
      float ss = sums.x + sums.y;
      for (int o = 1 << p.lanes_log >> 1; o; o >>= 1) ss += __shfl_xor_sync(~0u, ss, o);
      if (h < heads && s.w) {
        const float r = inverse_root(ss, p);
        const float2 rr = make_float2(r, r);
        float2 w[P];
        if (has_a) {
          load_weights<DT, P>(s, a, w);
#pragma unroll
          for (int e = 0; e < P; ++e) fa[e] = mul2(mul2(fa[e], rr), w[e]);
        }
        if (has_b) {
          load_weights<DT, P>(s, b, w);
#pragma unroll
          for (int e = 0; e < P; ++e) fb[e] = mul2(mul2(fb[e], rr), w[e]);
        }
      }
    }
    if (slot < rotated) {
      if (p.half) {
#pragma unroll
        for (int e = 0; e < P; ++e) {
          const float2 x = fa[e], y = fb[e];
          fa[e] = fma2(y, minus_sine[e], mul2(x, cosine[e]));
          fb[e] = fma2(x, sine[e], mul2(y, cosine[e]));
        }
      } else {  // pair i of the slot is its i-th float2; its turn is half of turn pair i / 2
        auto turn = [&](float2 v, int i) {
          const float sn = i % 2 ? sine[i / 2].y : sine[i / 2].x, cs = i % 2 ? cosine[i / 2].y : cosine[i / 2].x;
          return make_float2(__fmaf_rn(v.y, -sn, v.x * cs), __fmaf_rn(v.x, sn, v.y * cs));
        };
#pragma unroll
        for (int e = 0; e < P; ++e) {
          fa[e] = turn(fa[e], e);
          fb[e] = turn(fb[e], P + e);
        }
      }
    }
    if (h < heads) {
      T* y = static_cast<T*>(s.y) + token * s.y_token + (h >= p.side[0].heads ? h - p.side[0].heads : h) * s.y_head;
      if (has_a) *reinterpret_cast<uint4*>(y + a) = Vec16<DT>::put(fa);
      if (has_b) *reinterpret_cast<uint4*>(y + b) = Vec16<DT>::put(fb);
    }
  }
}

// pair by pair: any strides, sizes and alignment
template <int DT>
__global__ void __launch_bounds__(32 * kRopeWarps) rope_pairs_kernel(const __grid_constant__ RopeParams p) {
  using T = typename Elem<DT>::type;
  extern __shared__ float2 turns_of_warp[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int task = blockIdx.x * kRopeWarps + warp;
  depend_on_last();
  if (task >= p.tasks) return;
  const int token = task / p.parts, part = task - token * p.parts;
  float2* table = turns_of_warp + warp * (p.rot / 2);
  const int64_t position = p.positions[token];
  for (int i = lane; i < p.rot / 2; i += 32) table[i] = turn_of(p, position, i);
  __syncwarp();
  const int heads = p.side[0].heads + p.side[1].heads, pairs = p.rot / 2, items = pairs + p.d - p.rot;
  const int last = min((part + 1) * p.per, heads);
  for (int h = part * p.per; h < last; ++h) {
    const RopeSide& s = p.side[h >= p.side[0].heads];
    const int in = h >= p.side[0].heads ? h - p.side[0].heads : h;
    const T* x = static_cast<const T*>(s.x) + token * s.x_token + in * s.x_head;
    T* y = static_cast<T*>(s.y) + token * s.y_token + in * s.y_head;
    float r = 1.f;
    if (s.w) {
      float ss = 0.f;
      for (int i = lane; i < p.d; i += 32) {
        const float v = Elem<DT>::get(x[i]);
        ss = __fmaf_rn(v, v, ss);
      }
#pragma unroll
      for (int o = 16; o; o >>= 1) ss += __shfl_xor_sync(~0u, ss, o);
      r = inverse_root(ss, p);
    }
    auto value = [&](int c) {
      const float v = Elem<DT>::get(x[c]);
      return s.w ? v * r * (s.wt == KD_F32 ? static_cast<const float*>(s.w)[c] : load1<DT>(s.w, c)) : v;
    };
#pragma unroll 4
    for (int i = lane; i < items; i += 32) {  // the pairs, then the channels that pass through
      if (i < pairs) {
        const int a = p.half ? i : 2 * i, b = p.half ? i + pairs : 2 * i + 1;
        const float2 t = table[i];
        const float u = value(a), v = value(b);
        y[a] = Elem<DT>::put(__fmaf_rn(u, t.y, -(v * t.x)));
        y[b] = Elem<DT>::put(__fmaf_rn(v, t.y, u * t.x));
      } else {
        const int c = i + pairs;
        y[c] = Elem<DT>::put(value(c));
      }
    }
  }
}

template <int DT>
cudaError_t launch(RopeParams p, int64_t tokens, bool vec, cudaStream_t s) {
  const int heads = p.side[0].heads + p.side[1].heads;
  constexpr int V = Vec16<DT>::V;
  const int slots = p.rot / (2 * V) + (p.d - p.rot + 2 * V - 1) / (2 * V);
  p.lanes_log = 0;
  while (vec && (1 << p.lanes_log) < slots) ++p.lanes_log;
  const int rounds = vec ? (heads + (32 >> p.lanes_log) - 1) >> (5 - p.lanes_log) : heads;
  // as many parts of a token's rounds as all fit the GPU at a time (28 warps an SM), at least one: 2048 tokens of
  // ten rounds take 10.5 us in two parts, 13 in one, three or more
  const int64_t share = 152 * 28 / tokens;
  p.parts = (int)(share < 1 ? 1 : share > rounds ? rounds : share);
  p.per = (rounds + p.parts - 1) / p.parts;
  p.parts = (rounds + p.per - 1) / p.per;
  p.tasks = (int)(tokens * p.parts);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((p.tasks + (int64_t)kRopeWarps - 1) / kRopeWarps));
  cfg.blockDim = dim3(32 * kRopeWarps);
  cfg.dynamicSmemBytes = (size_t)kRopeWarps * (p.rot / 2) * sizeof(float2);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  launch_early(attr[0]);
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return vec ? cudaLaunchKernelEx(&cfg, rope_kernel<DT>, p) : cudaLaunchKernelEx(&cfg, rope_pairs_kernel<DT>, p);
}

// no two heads of y overlap
bool apart(const kd_heads* h, int64_t tokens, int64_t d) {
  const bool by_head = (h->heads == 1 || h->y_head >= d) &&
                       (tokens == 1 || (h->y_token >= d && h->y_token - d >= (h->heads - 1) * (h->heads == 1 ? 0 : h->y_head)));
  const bool by_token = (tokens == 1 || h->y_token >= d) &&
                        (h->heads == 1 || (h->y_head >= d && h->y_head - d >= (tokens - 1) * (tokens == 1 ? 0 : h->y_token)));
  return by_head || by_token;
}

}  // namespace
}  // namespace kd

extern "C" kd_status kd_rope_turns(const double* frequencies, int64_t count, uint64_t* turns_host) {
  if (count < 0 || (count > 0 && (!frequencies || !turns_host))) return KD_ERR_INVALID_ARG;
  for (int64_t i = 0; i < count; ++i)
    if (!std::isfinite(frequencies[i])) return KD_ERR_INVALID_ARG;
  for (int64_t i = 0; i < count; ++i) {
    // the quotient's 53 bits as an integer and a power of two; what lies above 2^64 is whole turns
    int e = 0;
    const int64_t bits = (int64_t)std::ldexp(std::frexp(frequencies[i] / 6.283185307179586, &e), 53);
    const int shift = e - 53 + 64;
    const uint64_t size = (uint64_t)(bits < 0 ? -bits : bits);
    const uint64_t turns = shift >= 64 || shift <= -64 ? 0 : shift >= 0 ? size << shift : (size + (((uint64_t)1 << -shift) >> 1)) >> -shift;
    turns_host[i] = bits < 0 ? (uint64_t)0 - turns : turns;
  }
  return KD_OK;
}

extern "C" kd_status kd_rope(const kd_heads* q, const kd_heads* k, kd_dtype dtype, int64_t tokens, int64_t d,
                             const int64_t* positions, const uint64_t* turns, int64_t rot, kd_rope_layout layout,
                             float amplitude, float eps, void* stream) {
  using namespace kd;
  if (d < 1 || d > kRopeMaxD) return KD_ERR_UNSUPPORTED_N;
  if (!q || tokens < 0 || tokens > INT32_MAX || !float_type(dtype) || rot < 2 || rot > d || rot % 2 != 0 ||
      (layout != KD_ROPE_HALF && layout != KD_ROPE_INTERLEAVED) || !(eps >= 0.f) || !std::isfinite(amplitude))
    return KD_ERR_INVALID_ARG;
  const kd_heads none{};
  const kd_heads* sides[2] = {q, k ? k : &none};
  int64_t heads = 0;
  for (const kd_heads* h : sides) {
    if (h->heads < 0 || h->heads > kRopeMaxHeads || h->x_token < 0 || h->x_head < 0 || h->y_token < 0 || h->y_head < 0 ||
        (h->weight && h->weight_dtype != dtype && h->weight_dtype != KD_F32))
      return KD_ERR_INVALID_ARG;
    heads += h->heads;
  }
  if (tokens * heads > INT32_MAX) return KD_ERR_INVALID_ARG;
  if (tokens == 0 || heads == 0) return KD_OK;
  const int64_t eb = type_bytes(dtype), V = 16 / eb;
  bool vec = rot % (2 * V) == 0 && d % V == 0 && (rot + (d - rot + 2 * V - 1) / (2 * V) * (2 * V)) / (2 * V) <= 32;
  if (!positions || !turns || !aligned(positions, 8) || !aligned(turns, 8)) return KD_ERR_INVALID_ARG;
  RopeParams p{};
  for (int i = 0; i < 2; ++i) {
    const kd_heads* h = sides[i];
    if (h->heads == 0) continue;
    if (!h->x || !h->y || !aligned(h->x, (size_t)eb) || !aligned(h->y, (size_t)eb) || !apart(h, tokens, d) ||
        (h->weight && !aligned(h->weight, (size_t)type_bytes((int)h->weight_dtype))))
      return KD_ERR_INVALID_ARG;
    const bool one = tokens == 1, single = h->heads == 1;
    vec = vec && aligned(h->x, 16) && aligned(h->y, 16) && (!h->weight || aligned(h->weight, 16)) &&
          (one || (h->x_token % V == 0 && h->y_token % V == 0)) && (single || (h->x_head % V == 0 && h->y_head % V == 0));
    p.side[i] = RopeSide{h->x, h->y, h->weight, one ? 0 : h->x_token, single ? 0 : h->x_head, one ? 0 : h->y_token,
                         single ? 0 : h->y_head, (int)h->heads, (int)h->weight_dtype};
  }
  p.positions = positions;
  p.turns = turns;
  p.d = (int)d;
  p.rot = (int)rot;
  p.half = layout == KD_ROPE_HALF;
  p.amplitude = amplitude;
  p.eps = eps;
  p.inv_d = 1.f / (float)d;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = dtype == KD_F32   ? launch<KD_F32>(p, tokens, vec, s)
                        : dtype == KD_F16 ? launch<KD_F16>(p, tokens, vec, s)
                                          : launch<KD_BF16>(p, tokens, vec, s);
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? KD_OK : KD_ERR_CUDA;
}
