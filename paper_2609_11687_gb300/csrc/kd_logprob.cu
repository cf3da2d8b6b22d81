// Log probabilities of given tokens, entropy and the largest alternatives of logit rows:
//
//     m = max x,  S = sum e^(x - m),  lse = m + ln S,  logprob(v) = (x_v - m) - ln S
//     entropy = ln S - sum e^(x - m) (x - m) / S
//
// One pass over a row: a thread walks 16-byte pieces of it, strided by the CTA, and keeps
// a running maximum m with the two sums relative to it (rescaled when m grows).
//
// For the k alternatives, the largest values that the threads of a warp have met (a few of
// each warp, 32 in all) are ranked: the k-th of them bounds the row's k-th largest value
// from below, by as little as a few dozen entries.  Only the pieces of threads whose maximum
// reaches that bar are read again (L2), and what reaches it is put on a list, entries above the bar
// at its front and entries equal to it at its back; a list's entries are ranked by
// counting.  An entry's key is its value's order above its index' complement, so that keys
// are distinct and equal values rank by lowest index.  Where more entries equal the bar
// than fit (masks: most of a row may hold one value), the lowest of them are looked up from
// the row's start; where more lie above it than fit, which takes a row whose largest
// values crowd in a few threads' pieces, they are taken one at a time.
//
// Few rows: a cluster of CTAs shares a row, and its first CTA joins their sums and their
// lists of alternatives.
//
// For many rows bound by memory and by the phases after a row's pass, during which its CTA
// loads nothing (2048 x 32000 bf16: 28 us, 4.7 TB/s or 70 % of the measured copy rate; 63 % of the
// issue slots used, warps wait for loads first, then at barriers); for few by the latency of
// those phases (one row of 32000 fp32 with 20 alternatives 6.5 us; 61 masked rows of 65537 11.1 us, 40 %
// of the slots used, warps wait at barriers first).
#include <cooperative_groups.h>

#include "kd_serve.cuh"

namespace kd {
namespace {

using namespace serve;
namespace cg = cooperative_groups;

constexpr int kT = 256;
constexpr int kWarps = kT / 32;
constexpr int kUnroll = 4;  // pieces a thread loads before it uses them
constexpr int kHalfList = 256;
constexpr int kMaxSplit = 8;
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
  int vocab, top, split, split_log;
};

__device__ __forceinline__ float ex2(float v) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}

// v - m, held above the exponents whose power is 0 anyway: entries of -infinity (also
// where m is, -inf - -inf) then count 0 in both sums.  The difference comes before the
// factor log2 e, which the type's lowest value would overflow.
__device__ __forceinline__ float under(float v, float m) { return fmaxf(v - m, -1000.f); }
__device__ __forceinline__ float power(float d) { return ex2(d * kLog2e); }
__device__ __forceinline__ uint32_t order_of(float v) {
  if (isnan(v)) return 0xFFFFFFFFu;
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

// the two halves of a cluster's barrier
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.aligned;" ::: "memory"); }

// running maximum m with s = sum e^(x - m) and t = sum e^(x - m) (x - m)
struct Run {
  float m, s, t;
};

struct Shared {
  Key list[2 * kHalfList];         // above the bar from the front, equal to it from the back
  Key best[KD_MAX_TOP];            // the CTA's alternatives, largest first; 0: none
  Key joined[kMaxSplit][KD_MAX_TOP];  // first CTA of a cluster: all lists
  Run runs[kMaxSplit];             // and all sums
  float2 sums[kWarps];             // of the warps, relative to the CTA's maximum
  uint32_t tops[32];               // largest values of the warps' threads, as orders
  uint32_t first;                  // top = 1: the maximum's lowest index
  int above, equal;
  uint32_t bar;
};

// two values at a time where the FMA pipe takes them packed
struct Pair {
  unsigned long long v;
};
__device__ __forceinline__ Pair pack(float a, float b) {
  Pair p;
  asm("mov.b64 %0, {%1, %2};" : "=l"(p.v) : "f"(a), "f"(b));
  return p;
}
__device__ __forceinline__ float2 unpack(Pair p) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(p.v));
  return r;
}
__device__ __forceinline__ Pair add2(Pair a, Pair b) {
  Pair r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ Pair mul2(Pair a, Pair b) {
  Pair r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
  Pair r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}

// calls f(value, index) for the entries of piece c (as loaded) that the row holds
template <int DT, class F>
__device__ __forceinline__ void each_entry(const Row<DT>& r, int c, uint4 piece, F f) {
  float v[kPiece<DT>];
  unpack<DT>(piece, v);
  const int i0 = r.first(c);
#pragma unroll
  for (int e = 0; e < kPiece<DT>; ++e)
    if (i0 + e >= 0 && i0 + e < r.vocab) f(v[e], i0 + e);
}

// entries on the list with a larger key, over both of its ends
__device__ __forceinline__ int rank_in(const Shared& sh, Key k, int above, int equal) {
  int n = 0;
#pragma unroll 4
  for (int j = 0; j < above; ++j) n += sh.list[j] > k;
#pragma unroll 4
  for (int j = 0; j < equal; ++j) n += sh.list[2 * kHalfList - 1 - j] > k;
  return n;
}

// One warp: the lowest indexes whose value's order is `bar` as best[from], best[from + 1], ...
// up to best[top - 1]: 32 pieces at a time from the front.
template <int DT>
__device__ __noinline__ void lowest_equal(Shared& sh, const Row<DT>& r, int c0, int c1, uint32_t bar, int from, int top) {
  const int lane = threadIdx.x & 31;
  for (int c = c0; c < c1 && from < top; c += 32) {
    const uint4 piece = c + lane < c1 ? r.load(c + lane) : lowest_piece<DT>();
    int n = 0;
    if (c + lane < c1) each_entry<DT>(r, c + lane, piece, [&](float v, int) { n += order_of(v) == bar; });
    int upto = n;  // with this lane's
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int b = __shfl_up_sync(~0u, upto, o);
      if (lane >= o) upto += b;
    }
    int at = from + upto - n;
    if (n && at < top)
      each_entry<DT>(r, c + lane, piece, [&](float v, int i) {
        if (order_of(v) == bar) {
          if (at < top) sh.best[at] = key_of(v, i);
          ++at;
        }
      });
    from += __shfl_sync(~0u, upto, 31);
  }
}

// a place of this thread's own behind *count, which the converged threads raise together
__device__ __forceinline__ int claim(int* count) {
  const uint32_t with = __activemask();
  const int lane = threadIdx.x & 31, leader = __ffs(with) - 1;
  int at = 0;
  if (lane == leader) at = atomicAdd(count, __popc(with));
  return __shfl_sync(with, at, leader) + __popc(with & ((1u << lane) - 1));
}

// the 32 largest of two lists in descending order (a, and b of which lane l holds entry 31 - l)
__device__ __forceinline__ Key merge_warp(Key a, Key b_reversed, int lane) {
  Key v = a > b_reversed ? a : b_reversed;
#pragma unroll 1
  for (int o = 16; o; o >>= 1) {
    const Key u = __shfl_xor_sync(~0u, v, o);
    v = ((lane & o) == 0) == (u > v) ? u : v;
  }
  return v;
}

// The entries of piece c (as loaded) that reach the bar, whose value is bar_v, to the list;
// more equal entries than it holds are not wanted.
template <int DT>
__device__ __noinline__ void collect(Shared& sh, const Row<DT>& r, int c, uint4 piece, uint32_t bar, float bar_v) {
  float v[kPiece<DT>];
  unpack<DT>(piece, v);
  uint32_t above = 0, reach = 0;
#pragma unroll
  for (int e = 0; e < kPiece<DT>; ++e) {
    above |= (v[e] > bar_v ? 1u : 0u) << e;
    reach |= (v[e] >= bar_v ? 1u : 0u) << e;
  }
  if (!reach) return;
  const int i0 = r.first(c);  // entries of the row only
  if (i0 < 0) reach &= ~0u << -i0;
  if (i0 + kPiece<DT> > r.vocab) reach &= (1u << (r.vocab - i0)) - 1;
  if (!bar) above = reach;  // a bar below everything
#pragma unroll 1
  for (uint32_t hits = above & reach; hits; hits &= hits - 1) {
    const int i = i0 + __ffs(hits) - 1, at = claim(&sh.above);
    if (at < kHalfList) sh.list[at] = key_of(Elem<DT>::get(r.x[i]), i);
  }
#pragma unroll 1
  for (uint32_t hits = reach & ~above; hits && *static_cast<volatile int*>(&sh.equal) <= kHalfList; hits &= hits - 1) {
    const int i = i0 + __ffs(hits) - 1, at = claim(&sh.equal);
    if (at < kHalfList) sh.list[2 * kHalfList - 1 - at] = (Key)bar << 32 | (0xFFFFFFFFu - (uint32_t)i);
  }
}

// SHARED: a cluster shares a row.  Registers: with many rows a fifth CTA of an SM helps more than
// the registers that it costs (2048 x 32000 bf16 28 us instead of 31), with few the reverse (61 x
// 65537 fp16 11.1 instead of 13.4).
template <int DT, bool SHARED>
__global__ void __launch_bounds__(kT, SHARED ? 4 : 5) logprob_kernel(const __grid_constant__ LogpParams p) {
  __shared__ Shared sh;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = SHARED ? special<kRank>() : 0;
  const int64_t step = special<kClusters>();
  const float low = __int_as_float(0xFF800000);
  if constexpr (SHARED) cluster_arrive();
  depend_on_last();

  for (int64_t row = special<kCluster>(); row < p.rows; row += step) {
    const Row<DT> r(p, row);
    // this CTA's pieces [c0, c1); this thread's: c0 + tid, c0 + tid + kT, ...
    const int per = SHARED ? (r.pieces + p.split - 1) >> p.split_log : r.pieces;
    const int c0 = min(r.pieces, rank * per), c1 = min(r.pieces, c0 + per);
    // the first given token of this thread, on its way meanwhile
    const bool reads = rank == 0 && tid < 32 && tid < p.tokens;
    int64_t id = reads ? p.ids[row * p.tokens + tid] : -1;
    if (tid == 0) {
      sh.first = 0xFFFFFFFFu;
      sh.above = sh.equal = 0;
    }
    if (tid < KD_MAX_TOP) sh.best[tid] = 0;

    float m = low;
    int where = 0;  // the batch of pieces that the maximum came from first
    Pair s2 = pack(0.f, 0.f), t2 = s2;
    const Pair l2e = pack(kLog2e, kLog2e);
    uint4 a[kUnroll];
    // pieces [from, upto) lie within the row
    const int from = r.before > 0, upto = min(c1, (int)(((int64_t)r.before + r.vocab) / kPiece<DT>));
    const uint4* pieces = reinterpret_cast<const uint4*>(r.x - r.before);
    for (int c = c0 + tid; c < c1; c += kUnroll * kT) {
      if (c >= from && c + (kUnroll - 1) * kT < upto) {
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) a[u] = pieces[c + u * kT];
      } else {
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) a[u] = c + u * kT < c1 ? r.load(c + u * kT) : lowest_piece<DT>();
      }
      uint4 am = a[0];
#pragma unroll
      for (int u = 1; u < kUnroll; ++u) am = max_piece<DT>(am, a[u]);
      const float bm = max_of<DT>(am);
      if (!(bm <= m)) {
        const float n = max_nan(m, bm), d = under(m, n), f = power(d);
        const Pair f2 = pack(f, f);
        t2 = mul2(f2, fma2(pack(d, d), s2, t2));
        s2 = mul2(f2, s2);
        m = n;
        where = c;
      }
      const Pair less = pack(-m, -m);
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        float v[kPiece<DT>];
        unpack<DT>(a[u], v);
#pragma unroll
        for (int e = 0; e < kPiece<DT>; e += 2) {
          float2 d = unpack(add2(pack(v[e], v[e + 1]), less));
          const Pair d2 = pack(fmaxf(d.x, -1000.f), fmaxf(d.y, -1000.f));  // as under()
          d = unpack(mul2(d2, l2e));
          const Pair x = pack(ex2(d.x), ex2(d.y));
          s2 = add2(s2, x);
          t2 = fma2(x, d2, t2);
        }
      }
    }
    float given = 0.f;
    if (id >= 0 && id < p.vocab) given = Elem<DT>::get(r.x[id]);

    // the warp's largest thread maxima: one, or as many as make `top` over the warps that
    // have pieces (where that is more than four, the first bar is below everything)
    const int busy = min(kWarps, max(1, (c1 - c0 + 31) / 32)), each = p.top > 1 ? (p.top + busy - 1) / busy : 1;
    uint32_t mine = order_of(m);
    for (int e = 0; e < 32 / kWarps; ++e) {
      uint32_t big = 0;
      if (e == 0 || (e < each && warp < busy)) {
        big = __reduce_max_sync(~0u, mine);
        if (each > 1 && lane == __ffs(__ballot_sync(~0u, mine == big)) - 1) mine = 0;
      }
      if (lane == 0) sh.tops[warp * (32 / kWarps) + e] = big;
    }
    __syncthreads();
    // every warp: the CTA's maximum; its own sums relative to it
    const uint32_t top = sh.tops[lane], most = __reduce_max_sync(~0u, top);
    const float cta_m = value_of(most);
    {
      const float2 s = unpack(s2), t = unpack(t2);
      const float d = under(m, cta_m), f = power(d);
      float ss = s.x + s.y;
      float tt = f * __fmaf_rn(d, ss, t.x + t.y);
      ss *= f;
#pragma unroll
      for (int o = 16; o; o >>= 1) {
        ss += __shfl_xor_sync(~0u, ss, o);
        tt += __shfl_xor_sync(~0u, tt, o);
      }
      if (lane == 0) sh.sums[warp] = make_float2(ss, tt);
    }
    const bool ranked = p.top > 0 && !isnan(cta_m);
    if (ranked && cta_m == low) {
      // nothing but -infinity here: the lowest indexes
      const int i0 = max(0, r.first(c0));
      if (tid < p.top && c0 < c1 && i0 + tid < min(r.vocab, r.first(c1))) sh.best[tid] = key_of(low, i0 + tid);
    } else if (ranked && p.top == 1) {
      // Its batch again, by the threads that hold it (looking for its place whenever a maximum is
      // new, with the pieces at hand, costs every warp in every batch a quarter of its
      // instructions: 34 us instead of 29 for 2048 x 32000 bf16).
      if (order_of(m) == most) {
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) a[u] = where + u * kT < c1 ? r.load(where + u * kT) : lowest_piece<DT>();
        uint32_t at = 0xFFFFFFFFu;
#pragma unroll
        for (int u = kUnroll - 1; u >= 0; --u) {
          float v[kPiece<DT>];
          unpack<DT>(a[u], v);
#pragma unroll
          for (int e = kPiece<DT> - 1; e >= 0; --e)
            if (v[e] == m) at = (uint32_t)(r.first(where + u * kT) + e);
        }
        atomicMin(&sh.first, at);
      }
    } else if (ranked) {
      // every warp: the bar
      uint32_t bar;
      {
        int larger = 0;
#pragma unroll 8
        for (int j = 0; j < 32; ++j) {
          const uint32_t o = __shfl_sync(~0u, top, j);
          larger += o > top || (o == top && j < lane);
        }
        bar = __shfl_sync(~0u, top, __ffs(__ballot_sync(~0u, larger == p.top - 1)) - 1);
      }
      const uint32_t mine = order_of(m);
      int above, equal;
      for (;;) {
        const float bar_v = bar ? value_of(bar) : low;
        // few threads with many pieces: each one's by its whole warp, a piece a lane, so that
        // each costs one wait for memory; else every thread its own, which it still holds
        // where they are one batch
        uint32_t whose = __ballot_sync(~0u, c0 + tid < c1 && mine >= bar);
        if (__popc(whose) * kUnroll * kT < c1 - c0) {
          for (; whose; whose &= whose - 1)
            for (int c = c0 + (tid & ~31) + __ffs(whose) - 1 + lane * kT; c < c1; c += 32 * kT)
              collect<DT>(sh, r, c, r.load(c), bar, bar_v);
        } else if (whose >> lane & 1) {
          for (int c = c0 + tid; c < c1; c += kUnroll * kT) {
            // nothing lies above a bar that is the maximum
            if (bar == most && *static_cast<volatile int*>(&sh.equal) > kHalfList) break;
            if (c1 - c0 > kUnroll * kT) {
#pragma unroll
              for (int u = 0; u < kUnroll; ++u) a[u] = c + u * kT < c1 ? r.load(c + u * kT) : lowest_piece<DT>();
            }
#pragma unroll
            for (int u = 0; u < kUnroll; ++u)
              if (c + u * kT < c1) collect<DT>(sh, r, c + u * kT, a[u], bar, bar_v);
          }
        }
        __syncthreads();
        above = sh.above;
        equal = sh.equal;
        if (above <= kHalfList) break;
        // every entry on the list lies above the bar: the next bar is higher
        for (int i = tid; i < kHalfList; i += kT) {
          const Key k = sh.list[i];
          if (rank_in(sh, k, kHalfList, 0) == p.top - 1) sh.bar = (uint32_t)(k >> 32);
        }
        __syncthreads();
        bar = sh.bar;
        if (tid == 0) sh.above = sh.equal = 0;
        __syncthreads();
      }
      if (equal > kHalfList) {
        if (warp == 0 && above < p.top) lowest_equal<DT>(sh, r, c0, c1, bar, above, p.top);
        equal = 0;
      }
      for (int i = tid; i < above + equal; i += kT) {
        const Key k = i < above ? sh.list[i] : sh.list[2 * kHalfList - 1 - (i - above)];
        const int at = rank_in(sh, k, above, equal);
        if (at < p.top) sh.best[at] = k;
      }
    }
    __syncthreads();

    // one warp goes on: sums in the warps' order, or of the cluster's CTAs in theirs
    Run all{cta_m, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      all.s += sh.sums[w].x;
      all.t += sh.sums[w].y;
    }
    if (ranked && p.top == 1 && tid == 0 && sh.first != 0xFFFFFFFFu) sh.best[0] = (Key)most << 32 | (0xFFFFFFFFu - sh.first);
    if constexpr (SHARED) {
      cg::cluster_group cl = cg::this_cluster();
      __syncwarp();
      cluster_wait();  // the first CTA runs: its shared memory may be written
      Shared* head = cl.map_shared_rank(&sh, 0);
      if (tid < KD_MAX_TOP) head->joined[rank][tid] = sh.best[tid];
      if (tid == 0) head->runs[rank] = all;
      cl.sync();
      if (rank != 0) return;
      if (warp == 0) {
        Run b = sh.runs[lane & (p.split - 1)];
        const uint32_t big = __reduce_max_sync(~0u, order_of(b.m));
        all.m = value_of(big);
        const float d = under(b.m, all.m), f = power(d);
        b.t = f * __fmaf_rn(d, b.s, b.t);
        b.s *= f;
        for (int o = 1; o < p.split; o <<= 1) {
          b.s += __shfl_xor_sync(~0u, b.s, o);
          b.t += __shfl_xor_sync(~0u, b.t, o);
        }
        all.s = b.s;
        all.t = b.t;
      }
      // the lists, each of them sorted, merged in pairs
      for (int w = 1; w < p.split && p.top > 0; w <<= 1) {
        if (warp < p.split / (2 * w)) {
          Key* list = sh.joined[2 * w * warp];
          list[lane] = merge_warp(list[lane], sh.joined[2 * w * warp + w][31 - lane], lane);
        }
        __syncthreads();
      }
      if (tid < p.top) sh.best[tid] = sh.joined[0][tid];
      __syncthreads();
    }

    if (warp == 0) {
      __syncwarp();
      const float nan = __int_as_float(0x7FC00000), inf = __int_as_float(0x7F800000);
      const bool none = all.m == -inf, over = all.m == inf;
      const float log_s = logf(all.s);
      const float lse = none || over || isnan(all.m) ? all.m : all.m + log_s;
      // (v - m) - ln S, not v - lse: beside a large m the logarithm would be rounded off
      auto logprob = [&](float v) { return none ? -inf : over ? nan : (v - all.m) - log_s; };
      if (lane == 0) {
        if (p.lse) p.lse[row] = lse;
        if (p.entropy) p.entropy[row] = none ? 0.f : over ? nan : log_s - all.t / all.s + (all.m - all.m);
      }
      for (int64_t i = lane; i < p.tokens; i += 32) {
        if (i != lane) {
          id = p.ids[row * p.tokens + i];
          if (id >= 0 && id < p.vocab) given = Elem<DT>::get(r.x[id]);
        }
        p.logprobs[row * p.tokens + i] = id < 0 ? 0.f : id >= p.vocab ? nan : logprob(given);
      }
      if (lane < p.top) {
        const Key k = sh.best[lane];
        const bool ok = !isnan(all.m);
        p.top_ids[row * p.top + lane] = ok ? (int64_t)(0xFFFFFFFFu - (uint32_t)k) : -1;
        p.top_logprobs[row * p.top + lane] = ok ? logprob(value_of((uint32_t)(k >> 32))) : nan;
      }
    }
    if constexpr (SHARED) return;  // a launch with clusters holds all rows at once
    __syncthreads();          // the shared values have been read
  }
}

template <int DT>
cudaError_t launch(const LogpParams& p, cudaStream_t s) {
  const int64_t rows = p.rows < (1 << 20) ? p.rows : 1 << 20;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(rows * p.split));
  cfg.blockDim = dim3(kT);
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  launch_early(attr[0]);
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)p.split;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = p.split > 1 ? 2 : 1;
  return p.split > 1 ? cudaLaunchKernelEx(&cfg, logprob_kernel<DT, true>, p)
                     : cudaLaunchKernelEx(&cfg, logprob_kernel<DT, false>, p);
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
  // CTAs that share a row: until there are four for each of 152 SMs, as long as a thread
  // keeps two pieces of its row
  const int64_t pieces = vocab * type_bytes(dtype) / 16;
  int split = 1;
  while (split < 8 && rows * split < 608 && pieces >= 4 * (int64_t)split * kT) split *= 2;
  LogpParams p{logits, ids, logprobs, lse, entropy, top_ids, top_logprobs, rows, ld, tokens, (int)vocab, top, split,
               split == 8 ? 3 : split == 4 ? 2 : split - 1};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = dtype == KD_F32   ? launch<KD_F32>(p, s)
                        : dtype == KD_F16 ? launch<KD_F16>(p, s)
                                          : launch<KD_BF16>(p, s);
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? KD_OK : KD_ERR_CUDA;
}
