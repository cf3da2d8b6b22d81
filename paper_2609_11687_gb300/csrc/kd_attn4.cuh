// Attention of few rows over a paged cache of 4-bit keys and values (kd_attention_4bit):
//
//     x_p = scale sum_g (step_g(p) sum_{c in g} code_c(p) q_c + low_g(p) sum_{c in g} q_c)
//     out_c = sum_p w_p (low_g(p) + step_g(p) code_c(p)) / sum_p w_p,   w_p = 2^(x_p log2 e - m)
//
// one pass over the codes with the running maximum m and sum of the softmax, on the tensor cores in
// fp16 (mma.sync m16n8k16), with the codes as the A operand of both products and the rows (query
// tokens times the heads that share a key head) as the eight columns of B: a decoded token of up to
// eight heads fills a tile, and the codes go from their word to the operand in registers.
//
// Codes.  A code masked out of its word is an fp16 number as it stands: c in a half's low bits is
// c 2^-24, four bits higher 16 c 2^-24, both below fp16's normal range, where the tensor cores
// are exact.  So a word of eight codes takes four masks and one shift.
// The 16 goes into q (keys: the odd channels' q over 16) and into the last step (values: the odd
// channels' sums over 16).  q is brought to 2^14 .. 2^15 by a power of two for each row, so that its
// fp16 or bf16 digits all stay; scores are exact products summed in fp32.
//
// Middles.  The tensor cores cut what does not fit their sums off (they do not round), so large sums
// that cancel in the end lose digits.  Codes therefore count from 8: value = low + 8 step + step (c - 8).
// Keys' sums over a group start at -8 sum q, which costs nothing; values, whose sums go over
// thousands of positions, have 8 taken off each pair of codes (measured without: 2.5 times the
// error of an fp16 output's own rounding over 5000 positions).
//
// Values.  w step is the B operand, rounded to fp16: the one rounding to fewer bits here.  It is scaled by a
// power of two that the largest step so far sets (like m, with the sums rescaled where it grows), so that
// nothing underflows that counts.  w times the middle, low + 8 step, is summed in fp32, so the error is
// 2^-12 of a value's distance from the middle of its group.
//
// Maximum.  m follows the scores only where one exceeds it by more than 8 (w up to 2^8, for which
// the scaling leaves room): a vote of the warp instead of a reduction over it for each tile.
//
// Mapping.  A CTA has one key head of one sequence, 8 NT of its rows and a share of its positions;
// its eight warps take 16 positions in turn, each with its own m and sums, joined once at the end
// in a fixed order.  Codes and scales of 16 positions, one contiguous block each in a page, stream
// through each warp's own ring (cp.async): no barrier of the CTA stands in the loop.  Rows of codes are an odd
// number of 16-byte pieces apart there, so that reads for both products are free of bank conflicts.  Where
// sequences are few their positions are split over CTAs and joined by a second launch.
#pragma once
#include <atomic>

#include "kd_cache4.cuh"

namespace kd {
namespace attn4 {

using namespace cache4;

constexpr int kWarps = 8;
constexpr int kTile = 16;     // positions of one step of a warp
constexpr int kBatch = 256;   // tiles whose places are looked up at a time

struct Params {
  Pages c;
  const uint16_t* q;
  uint16_t* out;
  float* lse;
  int64_t q_token, q_head, out_token, out_head;
  int64_t tokens;
  int heads, shared;            // query heads; of one key head
  int row_blocks, splits, per;  // of a sequence: blocks of rows; shares of positions, of at least `per` tiles
  int causal, window;
  int bf16, q_vec;
  float scale2;                 // scale log2 e
  float* part;                  // partial sums [sequence][key head][row block][split][row][d], then (m, sum) pairs
  float2* part_ml;
};

// The rows and positions of a block of rows: the same for the kernel that sums and the one that joins.
struct Work {
  int64_t first;       // row of the sequence's first query token
  int64_t before;      // position of that token
  int length, rows;    // rows: tokens times heads, from the block's first on
  int lo, hi;          // positions that some row sees
  int all_lo, all_hi;  // positions that every row sees
  int tile, tiles;     // of the positions lo .. hi
  int per, splits;     // tiles of a share, shares that have any (at least one)
};
__device__ __forceinline__ int clamp_to(int64_t v, int most) { return (int)(v < 0 ? 0 : v > most ? most : v); }
__device__ __forceinline__ Work work_of(const Params& p, int s, int block, int of_block) {
  Work w;
  int64_t count = p.c.most;
  w.first = (int64_t)s * p.c.most;
  if (p.c.starts) {
    w.first = p.c.starts[s];
    count = (int64_t)p.c.starts[s + 1] - w.first;
  }
  const int64_t tokens = min(count, (int64_t)p.c.most);
  w.length = max(p.c.lengths[s], 0);
  w.before = (int64_t)p.c.lengths[s] - count;
  const int64_t r0 = (int64_t)block * of_block, rows = tokens * p.shared - r0;
  w.rows = (int)max((int64_t)0, min(rows, (int64_t)of_block));
  const int64_t a = w.before + r0 / p.shared, b = w.before + (r0 + w.rows - 1) / p.shared;  // first, last position
  w.lo = w.all_lo = 0;
  w.hi = w.all_hi = w.length;
  if (p.causal) {
    w.hi = clamp_to(b + 1, w.length);
    w.all_hi = clamp_to(a + 1, w.length);
    if (p.window) {
      w.lo = clamp_to(a + 1 - p.window, w.length);
      w.all_lo = clamp_to(b + 1 - p.window, w.length);
    }
  }
  // positions past the table's room have no page: none is visited, and rows that see one are NaN
  w.hi = (int)min((int64_t)w.hi, (int64_t)p.c.wide * p.c.page);
  w.tile = w.lo / kTile;
  w.tiles = w.hi > w.lo ? (w.hi + kTile - 1) / kTile - w.tile : 0;
  w.per = max(p.per, (w.tiles + p.splits - 1) / p.splits);  // lengths past the host's hint: longer shares
  w.splits = w.tiles > w.per ? (w.tiles + w.per - 1) / w.per : 1;
  return w;
}

// does the row of a token, `nth` of its sequence's, see positions past the table's room?
__device__ __forceinline__ bool past_table(const Params& p, const Work& w, int nth) {
  const int64_t end = p.causal ? min(w.before + nth + 1, (int64_t)w.length) : w.length;
  return end > (int64_t)p.c.wide * p.c.page;
}

__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void wait_group() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                    uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};\n"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// an 8 x 8 matrix of halves, a row to four lanes, turned
__device__ __forceinline__ uint32_t turned(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
// two halves less two others
__device__ __forceinline__ uint32_t minus2(uint32_t a, uint32_t b) {
  const __half2 d = __hsub2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&d);
}
__device__ __forceinline__ float exp2_of(float x) {  // 2^-22 of its value off at most
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float low_half(uint32_t w) { return __half2float(__ushort_as_half((unsigned short)w)); }
__device__ __forceinline__ float high_half(uint32_t w) { return __half2float(__ushort_as_half((unsigned short)(w >> 16))); }

constexpr float kNone = -__builtin_inff();

// NC: 32-channel pieces of a row (the next of 1, 2, 3, 4, 6, 8); GS: of a group; NT: blocks of eight rows
template <int NC, int GS, int NT>
struct Shape {
  static constexpr int kGroups = (NC + GS - 1) / GS;
  static constexpr int kRows = 8 * NT;
  static constexpr int kStages = NC <= 4 ? 4 : 3;
  static constexpr int kStride = 4 * (NC | 1);                       // words of a row of codes in the ring
  static constexpr int kCodes = kTile * kStride, kScales = kTile * kGroups;  // words of a stage, keys or values
  static constexpr int kStage = 2 * (kCodes + kScales);
  // a value's 64 channels at a time (four tiles of 16), or 32 (two) where those have one scale
  static constexpr int kUnits = GS == 1 ? NC : (NC + 1) / 2, kOfUnit = GS == 1 ? 2 : 4;
  static constexpr int kSums = 32 * NC + 4;                          // floats of a row of a warp's sums
  static constexpr size_t kRing = (size_t)kWarps * kStages * kStage * 4, kJoin = (size_t)kWarps * kRows * kSums * 4;
  static constexpr size_t kBytes = (kRing > kJoin ? kRing : kJoin) + kBatch * 8 + (size_t)kWarps * kRows * 8;
};

// fp16 or bf16 bits as a float
__device__ __forceinline__ float wide(const Params& p, uint32_t bits) {
  return p.bf16 ? __uint_as_float(bits << 16) : __half2float(__ushort_as_half((unsigned short)bits));
}
__device__ __forceinline__ uint16_t narrow(const Params& p, float v) {
  return p.bf16 ? __bfloat16_as_ushort(__float2bfloat16_rn(v)) : __half_as_ushort(__float2half_rn(v));
}

template <int NC, int GS, int NT>
__global__ void __launch_bounds__(32 * kWarps, NC <= 4 && NT == 1 ? 2 : 1) attn4_kernel(const __grid_constant__ Params p) {
  using Z = Shape<NC, GS, NT>;
  constexpr int GN = Z::kGroups, ST = Z::kStages, S = Z::kStride;
  extern __shared__ uint4 smem[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g8 = lane >> 2, t4 = lane & 3;
  int64_t* place = reinterpret_cast<int64_t*>(reinterpret_cast<char*>(smem) + (Z::kRing > Z::kJoin ? Z::kRing : Z::kJoin));
  float2* ml = reinterpret_cast<float2*>(place + kBatch);
  depend_on_last();

  int at = blockIdx.x;
  const int block = at % p.row_blocks;
  at /= p.row_blocks;
  const int split = at % p.splits;
  at /= p.splits;
  const int head = at % p.c.heads, s = at / p.c.heads;
  const Work w = work_of(p, s, block, Z::kRows);
  if (w.rows == 0 || split >= w.splits) return;
  const int first_tile = w.tile + split * w.per, tiles = min(w.per, w.tiles - split * w.per);

  // Where a batch's tiles lie: the first row's number for this head, -1 on a bad page.
  auto look_up = [&](int b0, int n) {
    for (int i = threadIdx.x; i < n; i += 32 * kWarps) {
      const int64_t row = row_of(p.c, s, (int64_t)(first_tile + b0 + i) * kTile);
      place[i] = row < 0 ? -1 : row + (int64_t)head * p.c.page;
    }
  };
  look_up(0, min(tiles, kBatch));

  // The rows: this lane has row 8 nt + g8 and of each piece the eight channels of word t4.
  const int r0 = block * Z::kRows;
  uint32_t qb[2 * NC][NT][2];
  // of columns 2 t4, 2 t4 + 1: power of two of the row, and its sums over groups, both times scale log2 e
  float qs[GN][NT][2], qe[NT][2], q8[GN][NT][2];  // q8: where the sums over a group's codes start
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int r = 8 * nt + g8, token = (r0 + r) / p.shared;
    const int64_t t = w.first + token;
    const bool live = r < w.rows && t >= 0 && t < p.tokens;
    const uint16_t* q = p.q + (live ? t * p.q_token + (int64_t)(head * p.shared + (r0 + r) - token * p.shared) * p.q_head : 0);
    uint32_t raw[NC][4];  // pairs of channels
    uint32_t top = 0;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int ch = 32 * c + 8 * t4;
#pragma unroll
      for (int e = 0; e < 4; ++e) raw[c][e] = 0;
      if (live) {
        if (p.q_vec) {
          if (ch < p.c.d) {
            const uint4 u = *reinterpret_cast<const uint4*>(q + ch);
            raw[c][0] = u.x; raw[c][1] = u.y; raw[c][2] = u.z; raw[c][3] = u.w;
          }
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (ch + e < p.c.d) raw[c][e / 2] |= (uint32_t)q[ch + e] << (16 * (e % 2));
        }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e)
        top = max(top, __float_as_uint(wide(p, raw[c][e / 2] >> (16 * (e % 2)) & 0xFFFFu)) & 0x7FFFFFFFu);
    }
    top = max(top, __shfl_xor_sync(~0u, top, 1));
    top = max(top, __shfl_xor_sync(~0u, top, 2));
    // 2^e <= max |q| < 2^(e + 1); an infinity or NaN stays what it is under any factor
    const int e2 = top >> 23 == 255 || top == 0 ? 0 : max((int)(top >> 23) - 127, -100);
    const float up = __uint_as_float((uint32_t)(14 - e2 + 127) << 23);
    float sum[GN];
#pragma unroll
    for (int g = 0; g < GN; ++g) sum[g] = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v[e] = wide(p, raw[c][e / 2] >> (16 * (e % 2)) & 0xFFFFu);
        v[e] *= up;
        sum[c / GS] += v[e];
        if (e % 2) v[e] *= 0.0625f;
      }
      qb[2 * c][nt][0] = pack2<KD_F16>(v[0], v[4]);
      qb[2 * c][nt][1] = pack2<KD_F16>(v[1], v[5]);
      qb[2 * c + 1][nt][0] = pack2<KD_F16>(v[2], v[6]);
      qb[2 * c + 1][nt][1] = pack2<KD_F16>(v[3], v[7]);
    }
    const float down = __uint_as_float((uint32_t)(e2 + 127) << 23) * p.scale2;
#pragma unroll
    for (int j = 0; j < 2; ++j) qe[nt][j] = __shfl_sync(~0u, down, 4 * (2 * t4 + j));
#pragma unroll
    for (int g = 0; g < GN; ++g) {
      sum[g] += __shfl_xor_sync(~0u, sum[g], 1);
      sum[g] += __shfl_xor_sync(~0u, sum[g], 2);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float of_column = __shfl_sync(~0u, sum[g] * 0x1p-14f, 4 * (2 * t4 + j));
        qs[g][nt][j] = of_column * qe[nt][j];
        q8[g][nt][j] = of_column * -0x1p-7f;  // 8 times 2^14 / 2^24
      }
    }
  }
  // what the columns' rows see: positions from sees_lo on, below sees_hi
  int sees_lo[NT][2], sees_hi[NT][2];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int r = 8 * nt + 2 * t4 + j;
      const int64_t pos = w.before + (r0 + r) / p.shared;
      sees_hi[nt][j] = r >= w.rows ? 0 : p.causal ? clamp_to(pos + 1, w.length) : w.length;
      sees_lo[nt][j] = p.window ? clamp_to(pos + 1 - p.window, w.length) : 0;
    }

  // the ring: this lane's pieces of a stage
  uint32_t* ring = reinterpret_cast<uint32_t*>(smem) + warp * ST * Z::kStage;
  const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring);
  const int pieces = kTile * p.c.chunks;  // 16-byte pieces of a tile's keys
  uint32_t to[(NC + 1) / 2];
#pragma unroll
  for (int i = 0; i < (int)(sizeof(to) / 4); ++i) {
    const int n = lane + 32 * i, row = n / p.c.chunks;
    to[i] = (uint32_t)(row * S * 4 + (n - row * p.c.chunks) * 16);
  }
  const int row_bytes = 16 * p.c.chunks, scale_bytes = 4 * p.c.groups;
  auto issue = [&](int i, int stage) {
    const int64_t row = max(place[i], (int64_t)0);
    const uint32_t base = ring_at + stage * (Z::kStage * 4);
    const char* k = reinterpret_cast<const char*>(p.c.codes[0]) + row * row_bytes + lane * 16;
    const char* v = reinterpret_cast<const char*>(p.c.codes[1]) + row * row_bytes + lane * 16;
#pragma unroll
    for (int n = 0; n < (int)(sizeof(to) / 4); ++n)
      if (lane + 32 * n < pieces) {
        copy16(base + to[n], k + 512 * n);
        copy16(base + Z::kCodes * 4 + to[n], v + 512 * n);
      }
    if (lane < 4 * p.c.groups) {
      copy16(base + 2 * Z::kCodes * 4 + lane * 16, reinterpret_cast<const char*>(p.c.scales[0]) + row * scale_bytes + lane * 16);
      copy16(base + (2 * Z::kCodes + Z::kScales) * 4 + lane * 16,
             reinterpret_cast<const char*>(p.c.scales[1]) + row * scale_bytes + lane * 16);
    }
  };

  float acc[Z::kUnits * Z::kOfUnit][NT][4];
  float mids[GN][NT][2], m[NT][2], sum[NT][2];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int i = 0; i < Z::kUnits * Z::kOfUnit; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[i][nt][e] = 0.f;
#pragma unroll
    for (int g = 0; g < GN; ++g) mids[g][nt][0] = mids[g][nt][1] = 0.f;
    m[nt][0] = m[nt][1] = kNone;
    sum[nt][0] = sum[nt][1] = 0.f;
  }
  uint32_t step_cap = 0;  // fp16 bits: no step so far lies above
  float step_up = 1.f;    // the power of two of the values' weights: step_cap becomes 2^5 .. 2^6

  // One tile.  EDGE: some row does not see all of it, or its page is bad.
  auto tile = [&](auto edge, const uint32_t* stage, int position, bool bad) {
    constexpr bool EDGE = decltype(edge)::value;
    const uint32_t* ks = stage;
    const uint32_t* vs = stage + Z::kCodes;
    const uint32_t* kp = stage + 2 * Z::kCodes;
    const uint32_t* vp = kp + Z::kScales;
    float x[NT][4], part[NT][4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[nt][e] = 0.f;
        part[nt][e] = q8[0][nt][e & 1];
      }
    float mid[NT][4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 4; ++e) mid[nt][e] = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      uint32_t a = ks[g8 * S + 4 * c + t4], b = ks[(g8 + 8) * S + 4 * c + t4];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
          mma(part[nt], a & 0x000F000Fu, b & 0x000F000Fu, a & 0x00F000F0u, b & 0x00F000F0u, qb[2 * c + h][nt][0], qb[2 * c + h][nt][1]);
        a >>= 8;
        b >>= 8;
      }
      if ((c + 1) % GS == 0 || c == NC - 1) {
        // a piece past the row's last group meets q of 0: any group's scale will do
        const int g = min(c / GS, p.c.groups - 1);
        const uint32_t u = kp[g8 * p.c.groups + g], v = kp[(g8 + 8) * p.c.groups + g];
        const float s0 = low_half(u), m0 = __fmaf_rn(8.f, s0, high_half(u));
        const float s1 = low_half(v), m1 = __fmaf_rn(8.f, s1, high_half(v));
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            x[nt][e] = __fmaf_rn(e < 2 ? s0 : s1, part[nt][e], x[nt][e]);
            mid[nt][e] = __fmaf_rn(e < 2 ? m0 : m1, qs[c / GS][nt][e & 1], mid[nt][e]);
            part[nt][e] = q8[c / GS + 1 < GN ? c / GS + 1 : 0][nt][e & 1];
          }
      }
    }
    bool seen[NT][4];
    bool grow = false;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[nt][e] = __fmaf_rn(x[nt][e] * 1024.f, qe[nt][e & 1], mid[nt][e]);  // codes' 2^24 less q's 2^14
        if constexpr (EDGE) {
          const int pos = position + g8 + 8 * (e >> 1);
          seen[nt][e] = pos < sees_hi[nt][e & 1] && pos >= sees_lo[nt][e & 1];
          x[nt][e] = !seen[nt][e] ? kNone : bad ? __int_as_float(0x7FC00000) : x[nt][e];
        }
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) grow |= fmaxf(x[nt][j], x[nt][j + 2]) > m[nt][j] + 8.f;
    }
    uint32_t vscale[GN][2];
    uint32_t top = 0;
#pragma unroll
    for (int g = 0; g < GN; ++g)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        vscale[g][i] = vp[(g8 + 8 * i) * p.c.groups + min(g, p.c.groups - 1)];
        uint32_t bits = vscale[g][i] & 0xFFFFu;
        if constexpr (EDGE) {  // a position that no row sees may hold anything
          const int pos = position + g8 + 8 * i;
          if (pos >= w.hi || pos < w.lo) bits = 0;
        }
        if (bits <= 0x7BFFu) top = max(top, bits);
      }
    if (__any_sync(~0u, grow || top > step_cap)) {
      float by_step = 1.f;
      top = __reduce_max_sync(~0u, top);
      if (top > step_cap) {
        // 2^e <= step < 2^(e + 1) at most e = top's exponent, for subnormal ones the lowest normal
        const int e2 = max((int)(top >> 10) - 15, -14);
        const float up = __uint_as_float((uint32_t)(5 - e2 + 127) << 23);
        step_cap = min((uint32_t)(e2 + 15) << 10 | 0x3FFu, 0x7BFFu);
        by_step = up / step_up;
        step_up = up;
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          float to = fmaxf(x[nt][j], x[nt][j + 2]);
          to = fmaxf(to, __shfl_xor_sync(~0u, to, 4));
          to = fmaxf(to, __shfl_xor_sync(~0u, to, 8));
          to = fmaxf(to, __shfl_xor_sync(~0u, to, 16));
          to = fmaxf(to, m[nt][j]);
          const float f = m[nt][j] == kNone ? 0.f : exp2_of(m[nt][j] - to);
          m[nt][j] = to;
          sum[nt][j] *= f;
#pragma unroll
          for (int g = 0; g < GN; ++g) mids[g][nt][j] *= f;
          const float fs = f * by_step;
#pragma unroll
          for (int i = 0; i < Z::kUnits * Z::kOfUnit; ++i) {
            acc[i][nt][j] *= fs;
            acc[i][nt][j + 2] *= fs;
          }
        }
    }
    float wt[NT][4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float top_of = m[nt][e & 1];
        wt[nt][e] = exp2_of(x[nt][e] - (top_of == kNone ? 0.f : top_of));
        sum[nt][e & 1] += wt[nt][e];
      }
    // the values
    uint32_t bw[GN][NT][2];
#pragma unroll
    for (int g = 0; g < GN; ++g) {
      float up[2], mid[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float step = low_half(vscale[g][i]);
        mid[i] = __fmaf_rn(8.f, step, high_half(vscale[g][i]));
        up[i] = step * step_up;
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float b[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          b[e] = wt[nt][e] * up[e >> 1];
          float add = wt[nt][e] * mid[e >> 1];
          if constexpr (EDGE) {  // whatever stands where a row does not see: 0
            if (!seen[nt][e]) b[e] = add = 0.f;
          }
          mids[g][nt][e & 1] += add;
        }
        bw[g][nt][0] = turned(pack2<KD_F16>(b[0], b[1]));
        bw[g][nt][1] = turned(pack2<KD_F16>(b[2], b[3]));
      }
    }
#pragma unroll
    for (int u = 0; u < Z::kUnits; ++u) {
      const int g = GS == 1 ? u : 2 * u / GS;
      // the words of positions 2 t4, 2 t4 + 1, and of the same 8 on
      const int word = GS == 1 ? 4 * u + (g8 >> 1) : min(8 * u + g8, 4 * NC - 1);
      const uint32_t* at = vs + 2 * t4 * S + word;
      const uint32_t w0 = at[0], w1 = at[S], w2 = at[8 * S], w3 = at[9 * S];
#pragma unroll
      for (int half = 0; half < (GS == 1 ? 1 : 2); ++half) {
        const uint32_t pick = GS == 1 ? (g8 & 1 ? 0x7632u : 0x5410u) : half ? 0x7632u : 0x5410u;
        uint32_t a = __byte_perm(w0, w1, pick), b = __byte_perm(w2, w3, pick);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint32_t a0 = minus2(a & 0x000F000Fu, 0x00080008u), a1 = minus2(a & 0x00F000F0u, 0x00800080u);
          const uint32_t a2 = minus2(b & 0x000F000Fu, 0x00080008u), a3 = minus2(b & 0x00F000F0u, 0x00800080u);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) mma(acc[u * Z::kOfUnit + 2 * half + i][nt], a0, a1, a2, a3, bw[g][nt][0], bw[g][nt][1]);
          a >>= 8;
          b >>= 8;
        }
      }
    }
  };

  for (int b0 = 0; b0 < tiles; b0 += kBatch) {
    const int n = min(kBatch, tiles - b0);
    if (b0) {
      __syncthreads();  // no warp still reads the last batch's places
      look_up(b0, n);
    }
    __syncthreads();
    const int mine = (n - warp + kWarps - 1) / kWarps;
#pragma unroll
    for (int i = 0; i < ST - 1; ++i) {
      if (i < mine) issue(warp + i * kWarps, i);
      commit();
    }
    int stage = 0, next = ST - 1;
    for (int i = 0; i < mine; ++i) {
      if (i + ST - 1 < mine) issue(warp + (i + ST - 1) * kWarps, next);
      commit();
      wait_group<ST - 1>();
      __syncwarp();  // the lanes' copies are each other's
      const int nth = warp + i * kWarps, position = (first_tile + b0 + nth) * kTile;
      const bool bad = place[nth] < 0;
      if (bad || position < w.all_lo || position + kTile > w.all_hi) tile(std::true_type{}, ring + stage * Z::kStage, position, bad);
      else tile(std::false_type{}, ring + stage * Z::kStage, position, false);
      __syncwarp();
      stage = stage + 1 == ST ? 0 : stage + 1;
      next = next + 1 == ST ? 0 : next + 1;
    }
    wait_group<0>();
  }

  // The warps' sums, in fp32 without the scaling, then joined.
  __syncthreads();
  float* sums = reinterpret_cast<float*>(smem);
  const float back = 0x1p24f / step_up;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int r = 8 * nt + 2 * t4 + j;
#pragma unroll
      for (int o = 4; o < 32; o *= 2) {
        sum[nt][j] += __shfl_xor_sync(~0u, sum[nt][j], o);
#pragma unroll
        for (int g = 0; g < GN; ++g) mids[g][nt][j] += __shfl_xor_sync(~0u, mids[g][nt][j], o);
      }
      if (g8 == 0) ml[warp * Z::kRows + r] = make_float2(m[nt][j], sum[nt][j]);
      float* to = sums + (warp * Z::kRows + r) * Z::kSums;
#pragma unroll
      for (int u = 0; u < Z::kUnits; ++u) {
        const int g = GS == 1 ? u : 2 * u / GS;
#pragma unroll
        for (int i = 0; i < Z::kOfUnit; ++i) {
          const int ch = GS == 1 ? 32 * u + 4 * g8 + 2 * i : 64 * u + 8 * g8 + 2 * i;
          if (ch < 32 * NC) {
            to[ch] = __fmaf_rn(acc[u * Z::kOfUnit + i][nt][j], back, mids[g][nt][j]);
            to[ch + 1] = __fmaf_rn(acc[u * Z::kOfUnit + i][nt][j + 2], back * 0.0625f, mids[g][nt][j]);
          }
        }
      }
    }
  __syncthreads();
  const int64_t item = ((int64_t)s * p.c.heads + head) * p.row_blocks + block;
  for (int r = warp; r < w.rows; r += kWarps) {
    const int token = (r0 + r) / p.shared, h = head * p.shared + (r0 + r) - token * p.shared;
    const int64_t t = w.first + token;
    if (t < 0 || t >= p.tokens) continue;
    float top = kNone, total = 0.f, f[kWarps];
#pragma unroll
    for (int k = 0; k < kWarps; ++k) top = fmaxf(top, ml[k * Z::kRows + r].x);
#pragma unroll
    for (int k = 0; k < kWarps; ++k) {
      const float2 v = ml[k * Z::kRows + r];
      f[k] = v.x == kNone ? 0.f : exp2_of(v.x - top);
      total += v.x == kNone ? v.y : v.y * f[k];  // a warp without a maximum has summed nothing, or NaN
    }
    if (past_table(p, w, token)) total = __int_as_float(0x7FC00000);
    const bool none = total == 0.f;
    const float over = w.splits > 1 ? 1.f : none ? 0.f : 1.f / total;
    for (int ch = lane; ch < p.c.d; ch += 32) {
      float o = 0.f;
#pragma unroll
      for (int k = 0; k < kWarps; ++k) o = __fmaf_rn(sums[(k * Z::kRows + r) * Z::kSums + ch], f[k], o);
      o *= over;
      if (total != total) o = total;
      if (w.splits > 1) p.part[((item * p.splits + split) * Z::kRows + r) * p.c.d + ch] = o;
      else p.out[t * p.out_token + h * p.out_head + ch] = narrow(p, o);
    }
    if (lane == 0) {
      if (w.splits > 1) p.part_ml[(item * p.splits + split) * Z::kRows + r] = make_float2(top, total);
      else if (p.lse) p.lse[t * p.heads + h] = none ? kNone : (top + log2f(total)) * 0.693147180559945f;
    }
  }
}

// lets a kernel have all of an SM's shared memory; `ready` holds the devices where it does
template <class Kernel>
cudaError_t allow_shared_memory(Kernel kernel, std::atomic<uint64_t>& ready) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess || (dev < 64 && ready.load(std::memory_order_relaxed) >> dev & 1)) return e;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024);
  if (e == cudaSuccess && dev < 64) ready.fetch_or((uint64_t)1 << dev, std::memory_order_relaxed);
  return e;
}

template <int NC, int GS, int NT>
cudaError_t launch_one(const Params& p, cudaStream_t s) {
  static_assert(Shape<NC, GS, NT>::kBytes <= 227 * 1024, "shared memory");
  auto kernel = attn4_kernel<NC, GS, NT>;
  static std::atomic<uint64_t> ready{0};
  const cudaError_t e = allow_shared_memory(kernel, ready);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((int64_t)p.c.seqs * p.c.heads * p.row_blocks * p.splits));
  cfg.blockDim = dim3(32 * kWarps);
  cfg.dynamicSmemBytes = Shape<NC, GS, NT>::kBytes;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  launch_early(attr[0]);
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, p);
}
// gs: 32-channel pieces of a group; nt: blocks of eight rows
template <int NC, int NT>
cudaError_t launch(const Params& p, int gs, cudaStream_t s) {
  if constexpr (NC > 2)
    if (gs == 4) return launch_one<NC, 4, NT>(p, s);
  if constexpr (NC > 1)
    if (gs >= 2) return launch_one<NC, 2, NT>(p, s);
  return launch_one<NC, 1, NT>(p, s);
}

cudaError_t launch_small(const Params& p, int nc, int gs, int nt, cudaStream_t s);  // up to 64 channels
cudaError_t launch_96(const Params& p, int gs, int nt, cudaStream_t s);
cudaError_t launch_128(const Params& p, int gs, int nt, cudaStream_t s);
cudaError_t launch_192(const Params& p, int gs, cudaStream_t s);
cudaError_t launch_256(const Params& p, int gs, cudaStream_t s);

}  // namespace attn4
}  // namespace kd
