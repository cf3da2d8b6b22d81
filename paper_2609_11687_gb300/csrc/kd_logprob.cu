// Log probabilities of given tokens, entropy and the largest alternatives of logit rows:
//
//     m = max x,  S = sum e^(x - m),  lse = m + ln S,  logprob(v) = (x_v - m) - ln S
//     entropy = ln S - sum e^(x - m) (x - m) / S
//
// One pass over a row: a thread walks 16-byte pieces of it, strided by the CTA, and keeps
// a running maximum m with the two sums relative to it (rescaled when m grows).
// For the alternatives it remembers where its maximum came from.  An entry's key is its
// value's order above its index' complement, so that keys are distinct and equal values
// rank by lowest index.  The k-th largest of the threads' largest keys bounds the k-th
// largest key of the row from below, and only the (at most k) threads whose largest key
// reaches it hold entries that do: they alone walk their pieces again (L2), and the
// handful of entries found is ranked by counting.
//
// Few rows: a cluster of CTAs shares a row, and its first CTA joins their sums and their
// lists of alternatives.
#include <cooperative_groups.h>

#include "kd_serve.cuh"

namespace kd {
namespace {

using namespace serve;
namespace cg = cooperative_groups;

constexpr int kT = 512;
constexpr int kWarps = kT / 32;
constexpr int kUnroll = 4;    // pieces a thread loads before it uses them
constexpr int kCap = 1024;    // alternatives found in one go
constexpr float kLog2e = 1.4426950408889634f;

struct LogpParams {
  const void* x;
  const int64_t* ids;
  float* logprobs;
  float* lse;
  float* entropy;
  int64_t* top_ids;
  float* top_logprobs;
  int64_t rows, ld, tokens;
  int vocab, top, split;
};

__device__ __forceinline__ float ex2(float v) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}

// running maximum m with s = sum e^(x - m) and t = sum e^(x - m) (x - m)
struct Run {
  float m, s, t;
};
// v - m, held above the exponents whose power is 0 anyway: entries of -infinity (also
// where m is, -inf - -inf) then count 0 in both sums.  The difference comes before the
// factor log2 e, which the type's lowest value would overflow.
__device__ __forceinline__ float under(float v, float m) { return fmaxf(v - m, -1000.f); }
__device__ __forceinline__ float power(float d) { return ex2(d * kLog2e); }
__device__ __forceinline__ Run join(Run a, Run b) {
  const float m = max_nan(a.m, b.m);
  const float da = under(a.m, m), db = under(b.m, m);
  const float fa = power(da), fb = power(db);
  Run r;
  r.m = m;
  r.s = a.s * fa + b.s * fb;
  r.t = fa * __fmaf_rn(da, a.s, a.t) + fb * __fmaf_rn(db, b.s, b.t);
  return r;
}

__device__ __forceinline__ uint32_t order_of(float v) {
  const uint32_t u = __float_as_uint(v + 0.f);  // -0 as +0
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) {
  return __uint_as_float((o & 0x80000000u) ? o & 0x7FFFFFFFu : ~o);
}
__device__ __forceinline__ unsigned long long key_of(float v, int i) {
  return (unsigned long long)order_of(v) << 32 | (0xFFFFFFFFu - (uint32_t)i);
}

template <int DT>
constexpr int kPiece = DT == KD_F32 ? 4 : 8;  // elements of 16 bytes

template <int DT>
__device__ __forceinline__ void unpack(uint4 a, float (&v)[kPiece<DT>]) {
  if constexpr (DT == KD_F32) {
    v[0] = __uint_as_float(a.x); v[1] = __uint_as_float(a.y);
    v[2] = __uint_as_float(a.z); v[3] = __uint_as_float(a.w);
  } else {
    const float2 p0 = unpack2<DT>(a.x), p1 = unpack2<DT>(a.y), p2 = unpack2<DT>(a.z), p3 = unpack2<DT>(a.w);
    v[0] = p0.x; v[1] = p0.y; v[2] = p1.x; v[3] = p1.y;
    v[4] = p2.x; v[5] = p2.y; v[6] = p3.x; v[7] = p3.y;
  }
}
template <int DT>
__device__ __forceinline__ uint4 lowest_piece() {  // a piece of -infinities
  const uint32_t w = DT == KD_F32 ? 0xFF800000u : DT == KD_F16 ? 0xFC00FC00u : 0xFF80FF80u;
  return make_uint4(w, w, w, w);
}

// A row as pieces of 16 bytes.  Piece c holds elements [first(c), first(c) + kPiece) of
// the row; the first piece may begin before the row and the last may end after it.
template <int DT>
struct Row {
  const typename Elem<DT>::type* x;
  int vocab, before, pieces;  // before: elements of piece 0 that precede the row
  __device__ __forceinline__ Row(const LogpParams& p, int64_t row) {
    x = static_cast<const typename Elem<DT>::type*>(p.x) + row * p.ld;
    vocab = p.vocab;
    before = (int)((reinterpret_cast<uintptr_t>(x) & 15u) / sizeof(*x));
    pieces = (int)(((int64_t)before + vocab + kPiece<DT> - 1) / kPiece<DT>);
  }
  __device__ __forceinline__ int first(int c) const { return c * kPiece<DT> - before; }
  __device__ __forceinline__ uint4 load(int c) const {
    const int i0 = first(c);
    if (i0 >= 0 && i0 <= vocab - kPiece<DT>) return *reinterpret_cast<const uint4*>(x + i0);
    uint32_t w[4];
    if constexpr (DT == KD_F32) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        w[e] = i0 + e >= 0 && i0 + e < vocab ? __float_as_uint(x[i0 + e]) : 0xFF800000u;
    } else {
      const uint16_t* u = reinterpret_cast<const uint16_t*>(x);
      const uint32_t low = DT == KD_F16 ? 0xFC00u : 0xFF80u;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int a = i0 + 2 * e, b = a + 1;
        w[e] = (a >= 0 && a < vocab ? (uint32_t)u[a] : low) | (b >= 0 && b < vocab ? (uint32_t)u[b] : low) << 16;
      }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};

// the largest of a piece, NaN if it holds one
template <int DT>
__device__ __forceinline__ uint4 max_piece(uint4 a, uint4 b) {
  if constexpr (DT == KD_F32) {
    return make_uint4(__float_as_uint(max_nan(__uint_as_float(a.x), __uint_as_float(b.x))),
                      __float_as_uint(max_nan(__uint_as_float(a.y), __uint_as_float(b.y))),
                      __float_as_uint(max_nan(__uint_as_float(a.z), __uint_as_float(b.z))),
                      __float_as_uint(max_nan(__uint_as_float(a.w), __uint_as_float(b.w))));
  } else {
    auto mx = [](uint32_t p, uint32_t q) {
      uint32_t r;
      if constexpr (DT == KD_F16) asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(p), "r"(q));
      else asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(p), "r"(q));
      return r;
    };
    return make_uint4(mx(a.x, b.x), mx(a.y, b.y), mx(a.z, b.z), mx(a.w, b.w));
  }
}
template <int DT>
__device__ __forceinline__ float max_of(uint4 a) {
  if constexpr (DT == KD_F32) {
    return max_nan(max_nan(__uint_as_float(a.x), __uint_as_float(a.y)),
                   max_nan(__uint_as_float(a.z), __uint_as_float(a.w)));
  } else {
    const float2 p0 = unpack2<DT>(a.x), p1 = unpack2<DT>(a.y), p2 = unpack2<DT>(a.z), p3 = unpack2<DT>(a.w);
    return max_nan(max_nan(max_nan(p0.x, p0.y), max_nan(p1.x, p1.y)), max_nan(max_nan(p2.x, p2.y), max_nan(p3.x, p3.y)));
  }
}

using Key = unsigned long long;

// a warp's 32 keys, largest first
__device__ __forceinline__ Key sort_warp(Key v, int lane) {
#pragma unroll
  for (int size = 2; size <= 32; size <<= 1)
#pragma unroll
    for (int o = size >> 1; o; o >>= 1) {
      const Key u = __shfl_xor_sync(~0u, v, o);
      const bool keep_max = ((lane & o) == 0) == ((lane & size) == 0);
      v = keep_max == (u > v) ? u : v;
    }
  return v;
}
// the 32 largest of two sorted lists (a, and b of which lane l holds entry 31 - l), sorted
__device__ __forceinline__ Key merge_warp(Key a, Key b_reversed, int lane) {
  Key v = a > b_reversed ? a : b_reversed;
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    const Key u = __shfl_xor_sync(~0u, v, o);
    v = ((lane & o) == 0) == (u > v) ? u : v;
  }
  return v;
}

struct Shared {
  Key list[kWarps][32];
  Key found[kCap];
  Key best[KD_MAX_TOP];                // the CTA's alternatives, largest first
  Key joined[8 * KD_MAX_TOP];
  Run run[kWarps];
  Run total;
  int count;
};

// the largest key of each thread of the CTA below `below`, over all threads
__device__ __forceinline__ Key max_key(Shared& sh, Key v) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    const Key u = __shfl_xor_sync(~0u, v, o);
    v = u > v ? u : v;
  }
  __syncthreads();
  if (lane == 0) sh.list[warp][0] = v;
  __syncthreads();
  v = sh.list[0][0];
  for (int w = 1; w < kWarps; ++w) v = sh.list[w][0] > v ? sh.list[w][0] : v;
  return v;
}

template <int DT>
__global__ void __launch_bounds__(kT) logprob_kernel(const __grid_constant__ LogpParams p) {
  __shared__ Shared sh;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = p.split > 1 ? (int)(blockIdx.x % p.split) : 0;
  const int64_t step = gridDim.x / p.split;

  for (int64_t row = blockIdx.x / p.split; row < p.rows; row += step) {
    const Row<DT> r(p, row);
    // this CTA's pieces [c0, c1); this thread's: c0 + tid, c0 + tid + kT, ...
    const int per = (r.pieces + p.split - 1) / p.split;
    const int c0 = min(r.pieces, rank * per), c1 = min(r.pieces, c0 + per);

    const float low = __int_as_float(0xFF800000);
    Run run{low, 0.f, 0.f};
    int where = -1;  // the first piece of the batch of kUnroll that holds this thread's maximum
    for (int c = c0 + tid; c < c1; c += kUnroll * kT) {
      uint4 a[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) a[u] = c + u * kT < c1 ? r.load(c + u * kT) : lowest_piece<DT>();
      uint4 am = a[0];
#pragma unroll
      for (int u = 1; u < kUnroll; ++u) am = max_piece<DT>(am, a[u]);
      const float bm = max_of<DT>(am);
      if (where < 0 || !(bm <= run.m)) {
        const float m = max_nan(run.m, bm);
        const float d = under(run.m, m), f = power(d);
        run.t = f * __fmaf_rn(d, run.s, run.t);
        run.s *= f;
        run.m = m;
        where = c;
      }
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        float v[kPiece<DT>];
        unpack<DT>(a[u], v);
#pragma unroll
        for (int e = 0; e < kPiece<DT>; ++e) {
          const float d = under(v[e], run.m), x = power(d);
          run.s += x;
          run.t = __fmaf_rn(x, d, run.t);
        }
      }
    }

    // the CTA's sums
    Run tot = run;
#pragma unroll
    for (int o = 16; o; o >>= 1) {
      Run b;
      b.m = __shfl_xor_sync(~0u, tot.m, o);
      b.s = __shfl_xor_sync(~0u, tot.s, o);
      b.t = __shfl_xor_sync(~0u, tot.t, o);
      // both partners join in the same order: the lower lane's first
      tot = (lane & o) ? join(b, tot) : join(tot, b);
    }
    __syncthreads();  // the last row's shared values have been read
    if (lane == 0) sh.run[warp] = tot;
    if (tid == 0) sh.count = 0;

    if (p.top > 0) {
      // this thread's largest key
      Key mine = 0;
      if (where >= 0 && !isnan(run.m)) {
        for (int u = 0; u < kUnroll; ++u) {
          const int c = where + u * kT;
          if (c >= c1) break;
          float v[kPiece<DT>];
          unpack<DT>(r.load(c), v);
          const int i0 = r.first(c);
#pragma unroll
          for (int e = 0; e < kPiece<DT>; ++e)
            if (i0 + e >= 0 && i0 + e < r.vocab) {
              const Key k = key_of(v[e], i0 + e);
              mine = k > mine ? k : mine;
            }
        }
      }
      // the k-th largest of the threads' keys: warps sort theirs, then merge pairwise
      Key v = sort_warp(mine, lane);
      sh.list[warp][lane] = v;
#pragma unroll
      for (int w = 1; w < kWarps; w <<= 1) {
        __syncthreads();
        if (warp % (2 * w) == 0) {
          v = merge_warp(v, sh.list[warp + w][31 - lane], lane);
          sh.list[warp][lane] = v;
        }
      }
      __syncthreads();
      const Key bar = sh.list[0][p.top - 1];
      // entries that reach it
      if (mine && mine >= bar)
        for (int c = c0 + tid; c < c1; c += kT) {
          float w[kPiece<DT>];
          unpack<DT>(r.load(c), w);
          const int i0 = r.first(c);
#pragma unroll
          for (int e = 0; e < kPiece<DT>; ++e)
            if (i0 + e >= 0 && i0 + e < r.vocab) {
              const Key k = key_of(w[e], i0 + e);
              if (k >= bar) {
                const int at = atomicAdd(&sh.count, 1);
                if (at < kCap) sh.found[at] = k;
              }
            }
        }
      if (tid < KD_MAX_TOP) sh.best[tid] = 0;
      __syncthreads();
      const int count = sh.count;
      if (count <= kCap) {
        for (int i = tid; i < count; i += kT) {
          const Key k = sh.found[i];
          int above = 0;
          for (int j = 0; j < count; ++j) above += sh.found[j] > k;
          if (above < p.top) sh.best[above] = k;
        }
      } else {
        // the row's largest entries crowd in a few threads' pieces: one at a time
        Key last = ~(Key)0;
        for (int n = 0; n < p.top; ++n) {
          Key next = 0;
          for (int c = c0 + tid; c < c1; c += kT) {
            float w[kPiece<DT>];
            unpack<DT>(r.load(c), w);
            const int i0 = r.first(c);
#pragma unroll
            for (int e = 0; e < kPiece<DT>; ++e)
              if (i0 + e >= 0 && i0 + e < r.vocab) {
                const Key k = key_of(w[e], i0 + e);
                if (k < last && k > next) next = k;
              }
          }
          last = max_key(sh, next);
          if (tid == 0) sh.best[n] = last;
        }
      }
    }
    __syncthreads();
    if (tid == 0) {
      Run a = sh.run[0];
      for (int w = 1; w < kWarps; ++w) a = join(a, sh.run[w]);
      sh.total = a;
    }
    __syncthreads();

    Run all = sh.total;
    const Key* best = sh.best;
    if (p.split > 1) {
      cg::cluster_group cl = cg::this_cluster();
      cl.sync();
      if (rank == 0) {
        for (int k = 1; k < p.split; ++k) all = join(all, cl.map_shared_rank(&sh, k)->total);
        const int n = p.split * p.top;
        for (int i = tid; i < n; i += kT) sh.joined[i] = cl.map_shared_rank(&sh, i / p.top)->best[i % p.top];
        __syncthreads();
        Key k = 0;
        int above = KD_MAX_TOP;
        if (tid < n) {
          k = sh.joined[tid];
          above = 0;
          for (int j = 0; j < n; ++j) above += sh.joined[j] > k;
        }
        if (k && above < p.top) sh.best[above] = k;
        __syncthreads();
      }
      cl.sync();  // no CTA goes on while its lists are read
      if (rank != 0) continue;
    }

    const float nan = __int_as_float(0x7FC00000), inf = __int_as_float(0x7F800000);
    const bool none = all.m == -inf, over = all.m == inf;
    const float log_s = logf(all.s);
    const float lse = none || over || isnan(all.m) ? all.m : all.m + log_s;
    // (v - m) - ln S, not v - lse: beside a large m the logarithm would be rounded off
    auto logprob = [&](float v) { return none ? -inf : over ? nan : (v - all.m) - log_s; };
    if (tid == 0) {
      if (p.lse) p.lse[row] = lse;
      if (p.entropy) p.entropy[row] = none ? 0.f : over ? nan : log_s - all.t / all.s + (all.m - all.m);
    }
    for (int64_t i = tid; i < p.tokens; i += kT) {
      const int64_t id = p.ids[row * p.tokens + i];
      p.logprobs[row * p.tokens + i] =
          id < 0 ? 0.f : id >= p.vocab ? nan : logprob(Elem<DT>::get(r.x[id]));
    }
    if (tid < p.top) {
      const Key k = best[tid];
      const bool ok = !isnan(all.m);
      p.top_ids[row * p.top + tid] = ok ? (int64_t)(0xFFFFFFFFu - (uint32_t)k) : -1;
      p.top_logprobs[row * p.top + tid] = ok ? logprob(value_of((uint32_t)(k >> 32))) : nan;
    }
  }
}

template <int DT>
cudaError_t launch(const LogpParams& p, cudaStream_t s) {
  const int64_t rows = p.rows < (1 << 20) ? p.rows : 1 << 20;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(rows * p.split));
  cfg.blockDim = dim3(kT);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)p.split;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, logprob_kernel<DT>, p);
}

}  // namespace
}  // namespace kd

extern "C" kd_status kd_token_logprobs(const void* logits, kd_dtype dtype, int64_t rows, int64_t vocab, int64_t ld,
                                       const int64_t* ids, int64_t tokens, int top, float* logprobs, float* lse,
                                       float* entropy, int64_t* top_ids, float* top_logprobs, void* stream) {
  using namespace kd;
  if (rows < 0 || rows > INT32_MAX || vocab < 1 || vocab > (1 << 30) || tokens < 0 || top < 0 || top > KD_MAX_TOP ||
      top > vocab || !float_type(dtype) || ld < vocab)
    return KD_ERR_INVALID_ARG;
  if (rows == 0) return KD_OK;
  if (!logits || !aligned(logits, (size_t)type_bytes(dtype)) || (tokens > 0 && (!ids || !logprobs)) ||
      (top > 0 && (!top_ids || !top_logprobs)) || !aligned(ids, 8) || !aligned(logprobs, 4) || !aligned(lse, 4) ||
      !aligned(entropy, 4) || !aligned(top_ids, 8) || !aligned(top_logprobs, 4))
    return KD_ERR_INVALID_ARG;
  // CTAs that share a row: until there are two for each of 152 SMs, as long as a thread
  // keeps two pieces of its row
  const int64_t pieces = vocab * type_bytes(dtype) / 16;
  int split = 1;
  while (split < 8 && rows * split < 304 && pieces >= 4 * (int64_t)split * kT) split *= 2;
  LogpParams p{logits, ids, logprobs, lse, entropy, top_ids, top_logprobs, rows, ld, tokens, (int)vocab, top, split};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = dtype == KD_F32   ? launch<KD_F32>(p, s)
                        : dtype == KD_F16 ? launch<KD_F16>(p, s)
                                          : launch<KD_BF16>(p, s);
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? KD_OK : KD_ERR_CUDA;
}
