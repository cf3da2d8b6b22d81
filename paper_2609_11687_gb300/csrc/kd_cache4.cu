// Keys and values into and out of a paged cache of 4-bit codes (kd_cache_write_4bit,
// kd_cache_read_4bit).  For each group of a row (32, 64 or 128 channels), lo and hi its extremes:
//
//     low = lo rounded down to fp16,  step = (hi - low) / 15 rounded up to fp16,
//     code = rint((x - low) / step),  value = low + step * code
//
// Rounding the two outwards keeps every code within 0..15 without clamping and every element within
// half a step of its value.  All divisions are IEEE's: codes are reproducible bit for bit.
//
// Mapping.  A lane has eight channels: one word of codes.  4, 8, 16 or 32 lanes have a row (of a
// token, a head, and of keys or values), and reduce the extremes of a group among its 4 to 16 lanes
// by shuffles.  A warp finds its token's sequence and place once and takes several rounds of the token's rows
// where there are many tokens, one round where there are few.
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

struct Place {  // a warp's token
  int token, first, last;  // its rounds
  int64_t position, row;   // below 0: none; a bad page
};
__device__ __forceinline__ bool place_of(const RowParams& p, Place& w) {
  const int task = blockIdx.x * kCacheWarps + (threadIdx.x >> 5);
  if (task >= p.tasks) return false;
  w.token = task / p.parts;
  w.first = (task - w.token * p.parts) * p.per;
  w.last = min(w.first + p.per, p.rounds);
  int before;
  const int s = sequence_of(p.c, w.token, before);
  if (s < 0) return false;
  w.position = (int64_t)p.c.lengths[s] - before;
  w.row = w.position < 0 ? -1 : row_of(p.c, s, w.position);
  return true;
}

template <int DT, bool VEC>
__global__ void __launch_bounds__(32 * kCacheWarps) cache_write_kernel(const __grid_constant__ RowParams p) {
  depend_on_last();
  Place w;
  if (!place_of(p, w) || w.row < 0) return;
  const int lane = threadIdx.x & 31, word = lane & ((1 << p.lanes_log) - 1), nth = lane >> p.lanes_log;
  const int d = p.c.d, of_group = p.c.group / 8;
  for (int round = w.first; round < w.last; ++round) {
    const int item = (round << (5 - p.lanes_log)) + nth;
    const bool live = item < 2 * p.c.heads;
    const int side = live && item >= p.c.heads, h = live ? item - side * p.c.heads : 0;
    const int have = live ? d - 8 * word : 0;  // elements from the lane's first on
    float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (have > 0) load8<DT, VEC>(p.in[side], w.token * p.token[side] + h * p.head[side], 8 * word, d, v);
    const float inf = __int_as_float(0x7F800000);
    float lo = inf, minus_hi = inf;  // of -x: one kind of maximum does for both
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < have) {
        lo = -max_nan(-lo, -v[e]);
        minus_hi = -max_nan(-minus_hi, v[e]);
      }
    for (int o = min(of_group, 1 << p.lanes_log) >> 1; o; o >>= 1) {
      lo = -max_nan(-lo, -__shfl_xor_sync(~0u, lo, o));
      minus_hi = -max_nan(-minus_hi, -__shfl_xor_sync(~0u, minus_hi, o));
    }
    __half low = __float2half_rd(lo), step = __float2half_ru((-minus_hi - __half2float(low)) / 15.f);
    float flow = __half2float(low), fstep = __half2float(step);
    const bool fine = isfinite(flow) && isfinite(fstep);
    if (!fine) low = step = __ushort_as_half(0x7FFF);
    uint32_t codes = 0;
    if (fine && fstep > 0.f) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < have) codes |= (uint32_t)min(__float2int_rn((v[e] - flow) / fstep), 15) << (4 * e);
    }
    if (!live) continue;
    const int64_t row = w.row + (int64_t)h * p.c.page;
    if (word < 4 * p.c.chunks) p.c.codes[side][row * (4 * p.c.chunks) + word] = codes;
    if (have > 0 && word % of_group == 0)
      p.c.scales[side][row * p.c.groups + word / of_group] =
          (uint32_t)__half_as_ushort(step) | (uint32_t)__half_as_ushort(low) << 16;
  }
}

template <int DT, bool VEC>
__global__ void __launch_bounds__(32 * kCacheWarps) cache_read_kernel(const __grid_constant__ RowParams p) {
  depend_on_last();
  Place w;
  if (!place_of(p, w)) return;
  const int lane = threadIdx.x & 31, word = lane & ((1 << p.lanes_log) - 1), nth = lane >> p.lanes_log;
  const int c = 8 * word, of_group = p.c.group / 8;
  if (c >= p.c.d) return;
#pragma unroll 2
  for (int round = w.first; round < w.last; ++round) {
    const int item = (round << (5 - p.lanes_log)) + nth;
    if (item >= p.sides * p.c.heads) break;
    const int which = item >= p.c.heads, h = item - which * p.c.heads, side = p.first_side + which;
    float v[8];
    if (w.row < 0) {  // no place: 0; a bad page: NaN
      const float fill = w.position < 0 ? 0.f : __int_as_float(0x7FC00000);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = fill;
    } else {
      const int64_t row = w.row + (int64_t)h * p.c.page;
      const uint32_t codes = p.c.codes[side][row * (4 * p.c.chunks) + word];
      const uint32_t scale = p.c.scales[side][row * p.c.groups + word / of_group];
      const float step = __half2float(__ushort_as_half((unsigned short)scale));
      const float low = __half2float(__ushort_as_half((unsigned short)(scale >> 16)));
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = low + step * (float)(codes >> (4 * e) & 15);  // the product is exact
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

// how the rounds of rows are shared out, and the launch
template <class Kernel>
cudaError_t launch(Kernel kernel, RowParams& p, cudaStream_t s) {
  p.lanes_log = 2;
  while ((1 << p.lanes_log) < 4 * p.c.chunks) ++p.lanes_log;
  const int of_warp = 32 >> p.lanes_log;
  p.rounds = (p.sides * p.c.heads + of_warp - 1) / of_warp;
  // few tokens: a warp for each round of rows; many: several rounds share the search for their place
  const int64_t share = (int64_t)p.tokens * p.rounds / (152 * 32);
  p.per = (int)(share < 1 ? 1 : share > p.rounds ? p.rounds : share);
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

// rows of `heads` x `tokens` vectors of d elements do not overlap
bool rows_apart(int64_t tokens, int64_t heads, int64_t d, int64_t token, int64_t head) {
  if (tokens > 1 && heads > 1)
    return (head >= d && token >= d && (token - d) / head >= heads - 1) ||
           (token >= d && head >= d && (head - d) / token >= tokens - 1);
  return (tokens <= 1 || token >= d) && (heads <= 1 || head >= d);
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
