// Keys and values into and out of a paged cache of 4-bit codes (kd_cache_write_4bit,
// kd_cache_read_4bit).  For each group of a row (32, 64 or 128 channels), lo and hi its extremes:
//
//     low = lo rounded down to fp16,  step = (hi - low) / 15 rounded up to fp16,
//     code = rint((x - low) / step),  value = low + step * code
//
// Rounding the two outwards keeps every code within 0..15 without clamping and every element within
// half a step of its value.  Codes are those of IEEE divisions, reproducible bit for bit: the product with the
// reciprocal is off by less than 2^-18 (three roundings of at most 15.5), so only where it lies that close to a
// half does the division itself decide.
//
// Mapping.  A lane has eight channels: one word of codes.  4, 8, 16 or 32 lanes have a row (of a
// token, a head, and of keys or values), and reduce the extremes of a group among its 4 to 16 lanes
// by shuffles.  A warp finds its token's sequence and place once and takes several rounds of the token's rows
// where there are many tokens, one round where there are few.
//
// Writing 1361 tokens of four sequences (8 heads of 128, bf16) takes 9.6 us, 8 tokens and their way back 4.6 in two
// launches: a chain of loads (starts, lengths, table) stands before a row's place, and the row's own are issued before it.
// Reading 19,500 tokens into bf16 takes 27 us for 22 MB of codes and 80 MB of rows, of which 27 MB reach HBM meanwhile.  Writes
// alone run at 3.7 to 4.0 TB/s, also to memory that stays in L2 (a fill of 84 MB 21.8 us): the way to L2 is what bounds
// them, with issue slots 72 % busy the other half of it (a quarter fewer instructions left the 27 as they were).  (CTAs that look up a batch of tokens' places once and then share its
// rows took 14.8 and 27.8 us.)
#include "kd_cache4.cuh"

namespace kd {
namespace {

using namespace cache4;

constexpr int kCacheWarps = 4;  // of a CTA

struct RowParams {
  Pages c;
  const void* in[2];
  void* out[2];
  int64_t token[2], head[2];
  int tokens, tasks, parts, per, rounds;
  int sides;      // 2, or 1: what in[0] or out[0] is goes by first_side
  int first_side; // 0: keys, 1: values
  int lanes_log;  // lanes of a row
};

// eight consecutive elements from channel c on; VEC: they start on a 16-byte boundary and
// none lies past the row's end
template <int DT, bool VEC>
__device__ __forceinline__ void load8(const void* base, int64_t at, int c, int d, float (&v)[8]) {
  if constexpr (VEC) {
    if constexpr (DT == KD_F32) {
      const float4* f = reinterpret_cast<const float4*>(static_cast<const float*>(base) + at + c);
      const float4 a = f[0], b = f[1];
      v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
      v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
      const uint4 u = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(base) + at + c);
      const float2 a = unpack2<DT>(u.x), b = unpack2<DT>(u.y), e = unpack2<DT>(u.z), f = unpack2<DT>(u.w);
      v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y;
      v[4] = e.x; v[5] = e.y; v[6] = f.x; v[7] = f.y;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = c + e < d ? load1<DT>(base, at + c + e) : 0.f;
  }
}

struct Share {  // a warp's token and its rounds of the token's rows
  int token, first, last;
};
__device__ __forceinline__ bool share_of(const RowParams& p, Share& w) {
  const int task = blockIdx.x * kCacheWarps + (threadIdx.x >> 5);
  w.token = task / p.parts;
  w.first = (task - w.token * p.parts) * p.per;
  w.last = min(w.first + p.per, p.rounds);
  return task < p.tasks;
}
// The token's place: its position (below 0: none) and the first head's row there (-1 on a bad page); false where
// it is of no sequence.
__device__ __forceinline__ bool place_of(const RowParams& p, int token, int64_t& position, int64_t& row) {
  int before;
  const int s = sequence_of(p.c, token, before);
  if (s < 0) return false;
  position = (int64_t)p.c.lengths[s] - before;
  row = position < 0 ? -1 : row_of(p.c, s, (int)position);  // positions are less than a length
  return true;
}

template <int DT, bool VEC>
__global__ void __launch_bounds__(32 * kCacheWarps) cache_write_kernel(const __grid_constant__ RowParams p) {
  depend_on_last();
  Share w;
  if (!share_of(p, w)) return;
  const int lane = threadIdx.x & 31, word = lane & ((1 << p.lanes_log) - 1), nth = lane >> p.lanes_log;
  const int d = p.c.d, of_group = p.c.group / 8;
  constexpr int kAhead = DT == KD_F32 ? 1 : 2;  // rounds whose loads are in flight together
  float ahead[kAhead][8];
  auto fetch = [&](int first) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int item = ((first + i) << (5 - p.lanes_log)) + nth, side = item >= p.c.heads, h = item - side * p.c.heads;
#pragma unroll
      for (int e = 0; e < 8; ++e) ahead[i][e] = 0.f;
      if (first + i < w.last && item < 2 * p.c.heads && 8 * word < d)
        load8<DT, VEC>(p.in[side], w.token * p.token[side] + h * p.head[side], 8 * word, d, ahead[i]);
    }
  };
  fetch(w.first);  // while the place is looked for
  int64_t position, place;
  if (!place_of(p, w.token, position, place) || place < 0) return;
  for (int first = w.first; first < w.last; first += kAhead) {
    if (first != w.first) fetch(first);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (first + i >= w.last) break;
      const int item = ((first + i) << (5 - p.lanes_log)) + nth;
      const bool live = item < 2 * p.c.heads;
      const int side = live && item >= p.c.heads, h = live ? item - side * p.c.heads : 0;
      const int have = live ? d - 8 * word : 0;  // elements from the lane's first on
      const float(&v)[8] = ahead[i];
      const float inf = __int_as_float(0x7F800000);
      float lo = inf, hi = -inf;
      if (have > 0) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (VEC || e < have) {
            lo = min_nan(lo, v[e]);
            hi = max_nan(hi, v[e]);
          }
      }
      for (int o = min(of_group, 1 << p.lanes_log) >> 1; o; o >>= 1) {
        lo = min_nan(lo, __shfl_xor_sync(~0u, lo, o));
        hi = max_nan(hi, __shfl_xor_sync(~0u, hi, o));
      }
      __half low = __float2half_rd(lo), step = __float2half_ru((hi - __half2float(low)) / 15.f);
      const float flow = __half2float(low), fstep = __half2float(step);
      const bool fine = isfinite(flow) && isfinite(fstep);
      if (!fine) low = step = __ushort_as_half(0x7FFF);
      uint32_t codes = 0;
      if (fine && fstep > 0.f) {
        const float inverse = 1.f / fstep;
        // rounded by adding 1.5 2^23, whose last digit is 1; the code is then in the low bits
        constexpr float kRound = 12582912.f;
        uint32_t c[8];
        float off = 0.f;  // the reciprocal is 2^24 at most: a step is no smaller than 2^-24
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          const float2 q = mul2(add2(make_float2(v[e], v[e + 1]), make_float2(-flow, -flow)), make_float2(inverse, inverse));
          const float2 r = add2(q, make_float2(kRound, kRound));
          const float2 from = add2(q, make_float2(kRound - r.x, kRound - r.y));
          c[e] = __float_as_uint(r.x) & 15u;
          c[e + 1] = __float_as_uint(r.y) & 15u;
          off = fmaxf(off, fmaxf(fabsf(from.x), fabsf(from.y)));
        }
        if (off > 0.5f - 0x1p-17f) {
#pragma unroll
          for (int e = 0; e < 8; ++e) c[e] = (uint32_t)__float2int_rn((v[e] - flow) / fstep) & 15u;
        }
#pragma unroll
        for (int e = 7; e >= 0; --e) codes = codes * 16u + c[e];
        if (have < (VEC ? 1 : 8)) codes &= have <= 0 ? 0u : (1u << (4 * have)) - 1u;
      }
      if (!live) continue;
      const int64_t row = place + (int64_t)h * p.c.page;
      if (word < 4 * p.c.chunks) p.c.codes[side][row * (4 * p.c.chunks) + word] = codes;
      if (have > 0 && word % of_group == 0)
        p.c.scales[side][row * p.c.groups + word / of_group] =
            (uint32_t)__half_as_ushort(step) | (uint32_t)__half_as_ushort(low) << 16;
    }
  }
}

template <int DT, bool VEC>
__global__ void __launch_bounds__(32 * kCacheWarps) cache_read_kernel(const __grid_constant__ RowParams p) {
  depend_on_last();
  Share w;
  int64_t position, place;
  if (!share_of(p, w) || !place_of(p, w.token, position, place)) return;
  const int lane = threadIdx.x & 31, word = lane & ((1 << p.lanes_log) - 1), nth = lane >> p.lanes_log;
  const int c = 8 * word, of_group = p.c.group / 8;
  if (c >= p.c.d) return;
  const int heads = p.c.heads, items = p.sides * heads;
  const int64_t code_at = place * (4 * p.c.chunks) + word, scale_at = place * p.c.groups + word / of_group;
  constexpr int kAhead = 4;  // rounds whose loads are in flight together
  for (int first = w.first; first < w.last; first += kAhead) {
    uint32_t codes[kAhead], scale[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int item = ((first + i) << (5 - p.lanes_log)) + nth;
      if (first + i >= w.last || item >= items || place < 0) continue;
      const int which = item >= heads, side = p.first_side + which;
      const int64_t rows = (int64_t)(item - which * heads) * p.c.page;
      codes[i] = p.c.codes[side][code_at + rows * (4 * p.c.chunks)];
      scale[i] = p.c.scales[side][scale_at + rows * p.c.groups];
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int item = ((first + i) << (5 - p.lanes_log)) + nth;
      if (first + i >= w.last || item >= items) break;
      const int which = item >= heads, h = item - which * heads;
      float v[8];
      if (place < 0) {  // no place: 0; a bad page: NaN
        const float fill = position < 0 ? 0.f : __int_as_float(0x7FC00000);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = fill;
      } else {
        // codes e and e + 4 as halves 1024 + c (in the low bits) or 64 + c (four bits higher), less that
        const float step = __half2float(__ushort_as_half((unsigned short)scale[i]));
        const float low = __half2float(__ushort_as_half((unsigned short)(scale[i] >> 16)));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t u = codes[i] >> (e & 2 ? 8 : 0);
          const uint32_t bits = e & 1 ? (u & 0x00F000F0u) | 0x54005400u : (u & 0x000F000Fu) | 0x64006400u;
          const uint32_t less = e & 1 ? 0x54005400u : 0x64006400u;
          const float2 c2 = __half22float2(__hsub2(*reinterpret_cast<const __half2*>(&bits), *reinterpret_cast<const __half2*>(&less)));
          const float2 of = fma2(make_float2(step, step), c2, make_float2(low, low));  // exact products: one rounding
          v[e] = of.x;
          v[e + 4] = of.y;
        }
      }
      const int64_t at = w.token * p.token[which] + h * p.head[which] + c;
      if constexpr (VEC) {
        store8<DT>(p.out[which], at, v);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (c + e < p.c.d) store1<DT>(p.out[which], at + e, v[e]);
      }
    }
  }
}

// how the rounds of rows are shared out, and the launch
template <class Kernel>
cudaError_t launch(Kernel kernel, RowParams& p, cudaStream_t s) {
  p.lanes_log = 2;
  while ((1 << p.lanes_log) < 4 * p.c.chunks) ++p.lanes_log;
  const int of_warp = 32 >> p.lanes_log;
  p.rounds = (p.sides * p.c.heads + of_warp - 1) / of_warp;
  // as many parts of a token's rounds as all fit the GPU in two turns (64 warps an SM), at least one: the warps of
  // one token each look for its place
  const int64_t share = 152 * 64 / p.tokens;
  p.parts = (int)(share < 1 ? 1 : share > p.rounds ? p.rounds : share);
  p.per = (p.rounds + p.parts - 1) / p.parts;
  p.parts = (p.rounds + p.per - 1) / p.per;
  p.tasks = (int)((int64_t)p.tokens * p.parts);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((p.tasks + (int64_t)kCacheWarps - 1) / kCacheWarps));
  cfg.blockDim = dim3(32 * kCacheWarps);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  launch_early(attr[0]);
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, p);
}

kd_status check(const kd_cache4* cache, const kd_sequences* seqs, int64_t tokens, int dtype, int64_t k_token,
                int64_t k_head, int64_t v_token, int64_t v_head) {
  if (!cache_sizes_ok(cache) || !sequences_sizes_ok(seqs) || tokens < 0 || !float_type(dtype) || k_token < 0 || k_head < 0 ||
      v_token < 0 || v_head < 0 || tokens > INT32_MAX || tokens * 2 * cache->heads > INT32_MAX)
    return KD_ERR_INVALID_ARG;
  if (cache->d < 1 || cache->d > kMaxD) return KD_ERR_UNSUPPORTED_N;
  return KD_OK;
}

}  // namespace
}  // namespace kd

extern "C" kd_status kd_cache_write_4bit(const kd_cache4* cache, const kd_sequences* seqs, int64_t tokens, const void* k,
                                         int64_t k_token, int64_t k_head, const void* v, int64_t v_token,
                                         int64_t v_head, kd_dtype dtype, void* stream) {
  using namespace kd;
  const kd_status st = check(cache, seqs, tokens, dtype, k_token, k_head, v_token, v_head);
  if (st != KD_OK || tokens == 0 || seqs->seqs == 0 || seqs->most == 0) return st;
  const int64_t eb = type_bytes(dtype), V = 16 / eb;
  if (!cache_pointers_ok(cache) || !sequences_pointers_ok(seqs) || !k || !v || !aligned(k, (size_t)eb) || !aligned(v, (size_t)eb))
    return KD_ERR_INVALID_ARG;
  RowParams p{};
  p.c = pages_of(cache, seqs);
  p.in[0] = k;
  p.in[1] = v;
  p.token[0] = k_token;
  p.token[1] = v_token;
  p.head[0] = k_head;
  p.head[1] = v_head;
  p.tokens = (int)tokens;
  p.sides = 2;
  const bool one = tokens == 1, single = cache->heads == 1;
  const bool vec = cache->d % 8 == 0 && aligned(k, 16) && aligned(v, 16) &&
                   (one || (k_token % V == 0 && v_token % V == 0)) && (single || (k_head % V == 0 && v_head % V == 0));
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (dtype == KD_F32) e = vec ? launch(cache_write_kernel<KD_F32, true>, p, s) : launch(cache_write_kernel<KD_F32, false>, p, s);
  else if (dtype == KD_F16) e = vec ? launch(cache_write_kernel<KD_F16, true>, p, s) : launch(cache_write_kernel<KD_F16, false>, p, s);
  else e = vec ? launch(cache_write_kernel<KD_BF16, true>, p, s) : launch(cache_write_kernel<KD_BF16, false>, p, s);
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? KD_OK : KD_ERR_CUDA;
}

extern "C" kd_status kd_cache_read_4bit(const kd_cache4* cache, const kd_sequences* seqs, int64_t tokens, void* k,
                                        int64_t k_token, int64_t k_head, void* v, int64_t v_token, int64_t v_head,
                                        kd_dtype dtype, void* stream) {
  using namespace kd;
  const kd_status st = check(cache, seqs, tokens, dtype, k_token, k_head, v_token, v_head);
  if (st != KD_OK || tokens == 0 || seqs->seqs == 0 || seqs->most == 0) return st;
  const int64_t eb = type_bytes(dtype), V = 16 / eb;
  if (!cache_pointers_ok(cache) || !sequences_pointers_ok(seqs) || (!k && !v) || !aligned(k, (size_t)eb) || !aligned(v, (size_t)eb) ||
      (k && !rows_apart(tokens, cache->heads, cache->d, k_token, k_head)) ||
      (v && !rows_apart(tokens, cache->heads, cache->d, v_token, v_head)))
    return KD_ERR_INVALID_ARG;
  RowParams p{};
  p.c = pages_of(cache, seqs);
  p.tokens = (int)tokens;
  p.first_side = k ? 0 : 1;
  for (int side = 0; side < 2; ++side)
    if (side ? v : k) {
      p.out[p.sides] = side ? v : k;
      p.token[p.sides] = side ? v_token : k_token;
      p.head[p.sides] = side ? v_head : k_head;
      ++p.sides;
    }
  bool vec = cache->d % 8 == 0;
  for (int i = 0; i < p.sides; ++i)
    vec = vec && aligned(p.out[i], 16) && (tokens == 1 || p.token[i] % V == 0) && (cache->heads == 1 || p.head[i] % V == 0);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (dtype == KD_F32) e = vec ? launch(cache_read_kernel<KD_F32, true>, p, s) : launch(cache_read_kernel<KD_F32, false>, p, s);
  else if (dtype == KD_F16) e = vec ? launch(cache_read_kernel<KD_F16, true>, p, s) : launch(cache_read_kernel<KD_F16, false>, p, s);
  else e = vec ? launch(cache_read_kernel<KD_BF16, true>, p, s) : launch(cache_read_kernel<KD_BF16, false>, p, s);
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? KD_OK : KD_ERR_CUDA;
}
