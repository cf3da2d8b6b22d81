// Products of few activation rows with 4-bit weights and group scales (kd_matmul_4bit):
//
//     y[r][j] = xs[r] sum_g s[g][j] sum_{i in g} (c[j][i] - z[g][j]) x[r][i]
//
// on the tensor cores in 16 bits (mma.sync m16n8k16), with the weights as the A operand (16
// channels) and the activation rows as B, so that 8 rows fill a tile.  e4m3 rows are taken
// as the fp16 values they are.
//
// Codes.  Masked into the mantissa of a power of two a code makes 1024 + c (fp16, in a
// half's low bits) or 64 + c (four bits higher) or 128 + c (bf16), and a packed subtraction
// leaves the integer c - z.  Products are exact, sums fp32.  A word of eight takes one shift
// (bf16, whose mantissa holds one place only: three) and four mask-ors, on the integer pipe
// of half the issue rate that this costs most.  (Products in e4m3, in which a code is a byte
// without any arithmetic, were measured at half the speed: mma.sync runs them as fp16 with
// conversions of both operands.)
//
// Mapping.  One CTA per SM stays and walks tiles of channels.  A warp owns 32 channels of
// the tile; kw warps split the inputs among them (chunks of 128), and where that is not
// enough CTAs of a cluster do too.  The partial sums are added in a fixed order.  The rows
// of the CTA's inputs are laid out once in shared memory as the B operands that the lanes
// will want.  The codes stream through a ring of stages that each lane fills and reads for
// itself (cp.async; smaller groups: the lanes of a warp for each other): no barrier of the CTA
// stands in the loop, and the copies of the next tile are in flight while this one's sums are
// joined.  Sixteen warps hide each other's waits, and two stages each are enough then (eight
// warps of up to 177 registers at 9 to 16 rows: 36 us instead of 24 for 32000 x 4096; three
// stages 32, their shared memory leaves room for half the rows only).
//
// No unit is saturated: at 8 rows of 32000 x 4096 the SMs that have a CTA (125 of 152, two tiles
// each) use 60 % of their issue slots and 55 % of the integer pipe, the tensor pipe 23 %, DRAM
// 38 %.  A warp issues 341 instructions a chunk: 112 on the integer pipe (of about 157 there) and 64
// subtractions decode, 16 are products, the rest are addresses, scales, copies and the loop.  3.5 TB/s
// there, 19.9 us for a floor of 10.1; one row of 11008 x 4096 7.9 us, of 4096 x 4096 4.1.  At 16 e4m3
// rows of 4096 x 11008 in groups of 64 (13.3 us) 597 instructions a chunk, 44 % of the slots used:
// warps wait for memory and for each other.  The registers of sixteen warps (128 a thread)
// make these instances spill: groups of 32 at 9 to 16 rows (60 to 100 bytes) and with zero points
// below (20), groups of 64 (8, with zero points 76) and of 128 with zero points (8) at 9 to 16 fp16 rows.
//
// K order.  The product is a sum over inputs, so A and B may enumerate them in any common
// order.  A group of GS x 32 inputs is 4 GS code words of a channel; the lanes with
// t = lane % 4 take the words GS t .. GS t + GS - 1, one a step, and the same inputs of
// their row.
//
// Channel order.  Rows g, g + 8 of the two mma tiles (g = lane / 4) are channels 4g .. 4g + 3
// of the warp's 32, so that a lane's four scales are one load of 8 bytes.
#pragma once
#include <cooperative_groups.h>
#include <cuda_fp8.h>

#include <atomic>

#include "kd_weight4.cuh"

namespace kd {
namespace mat4 {

using namespace serve;

constexpr int kTile = 32;    // output channels of a warp: two m16 tiles
constexpr int kChunk = 128;  // inputs of a chunk
constexpr int kStages = 2;
constexpr int kStageUnits = 128;  // 16-byte units of a stage: 32 channels x 64 bytes

struct Params {
  const uint8_t* codes;
  const uint16_t* scales;
  const uint8_t* zeros;
  const uint8_t* x;
  const float* xs;
  void* y;
  int64_t ldx, ldy;
  int n, m, rows;
  int e4m3;                    // x holds bytes
  int groups, pieces, chunks;  // per channel: scales, 16-byte pieces of codes; chunks of 128 inputs
  int per;                     // chunks of one CTA of a cluster
  float turns_of_row_inv;      // 1 / (32-item turns of a row's inputs in one CTA)
  int split;                   // CTAs of a cluster
  int kw, kw_log;              // warps that split the inputs of a tile (a power of two)
  int tiles;                   // of 32 * warps / kw channels
  int x_vec, scale_vec, scale_bf16, ydtype;
};

constexpr int kWarps = 16;  // of a CTA
// Shared memory, in bytes: the ring; the warps' partial sums; the rows; for clusters two
// sets of the CTA's sums.
constexpr size_t kRingBytes = (size_t)kStages * kStageUnits * 16;  // of a warp
constexpr size_t kRedBytes = (size_t)8 * kTile * 4;                // of a warp, for each 8 rows
inline size_t smem_bytes(int nt, int rows, int per, int split, int kw) {
  const size_t outputs = (size_t)kTile * (kWarps / kw) * rows;
  return kWarps * (kRingBytes + nt * kRedBytes) + (size_t)per * nt * 2048 +
         (split > 1 ? 2 * outputs * 4 : 0);
}

__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void wait_group() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// D = A B (+ D unless FIRST)
template <bool BF, bool FIRST>
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                    uint32_t b1) {
#define KD_MMA(TYPE)                                                                                             \
  if constexpr (FIRST)                                                                                           \
    asm("mma.sync.aligned.m16n8k16.row.col.f32." TYPE "." TYPE ".f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, " \
        "{%10, %10, %10, %10};\n"                                                                                \
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])                                                         \
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));                                       \
  else                                                                                                           \
    asm("mma.sync.aligned.m16n8k16.row.col.f32." TYPE "." TYPE ".f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, " \
        "{%0, %1, %2, %3};\n"                                                                                    \
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])                                                         \
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1))
  if constexpr (BF) {
    KD_MMA("bf16");
  } else {
    KD_MMA("f16");
  }
#undef KD_MMA
}

// (a & MASK) | b in one operation: b comes in a register, the mask is its one immediate
template <uint32_t MASK>
__device__ __forceinline__ uint32_t mask_or(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(a), "n"(MASK), "r"(b));
  return r;
}
// What the codes are or-ed into, in registers whose values the compiler does not know (a
// constant would be a second immediate, and a second operation).
template <bool BF>
struct Magic {
  uint32_t low, high;
  __device__ __forceinline__ Magic() {
    if constexpr (BF) {
      asm volatile("mov.u32 %0, 0x43004300;" : "=r"(low));
      high = 0;
    } else {
      asm volatile("mov.u32 %0, 0x64006400;" : "=r"(low));
      asm volatile("mov.u32 %0, 0x54005400;" : "=r"(high));
    }
  }
};
// a zero point as it comes off: 1024 + z and 64 + z (fp16), or 128 + z (bf16), twice a word
template <bool BF>
__device__ __forceinline__ uint2 zero_words(uint32_t z) {
  if constexpr (BF) return make_uint2((0x4300u + z) * 0x10001u, 0u);
  else return make_uint2((0x6400u + z) * 0x10001u, (0x5400u + 16u * z) * 0x10001u);
}
template <bool BF>
__device__ __forceinline__ uint32_t minus2(uint32_t a, uint32_t b) {
  if constexpr (BF) {
    const __nv_bfloat162 d =
        __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
    return *reinterpret_cast<const uint32_t*>(&d);
  } else {
    const __half2 d = __hsub2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
    return *reinterpret_cast<const uint32_t*>(&d);
  }
}
// codes 2h, 2h + 4 and 2h + 1, 2h + 5 of a word, less the zero point
template <bool BF>
__device__ __forceinline__ uint2 code_pairs(uint32_t w, int h, const Magic<BF>& k, uint2 zero) {
  w >>= 8 * h;
  if constexpr (BF)
    return make_uint2(minus2<BF>(mask_or<0x000F000Fu>(w, k.low), zero.x),
                      minus2<BF>(mask_or<0x000F000Fu>(w >> 4, k.low), zero.x));
  else
    return make_uint2(minus2<BF>(mask_or<0x000F000Fu>(w, k.low), zero.x),
                      minus2<BF>(mask_or<0x00F000F0u>(w, k.high), zero.y));
}

// eight consecutive inputs of a row from k on as four words of 16-bit values (e4m3: two words
// of bytes): all of them and aligned, or one by one and zero past n
__device__ __forceinline__ uint4 load_inputs(const Params& p, int64_t at) {
  if (p.e4m3) {
    const uint2 u = *reinterpret_cast<const uint2*>(p.x + at);
    return make_uint4(u.x, u.y, 0, 0);
  }
  return *reinterpret_cast<const uint4*>(p.x + 2 * at);
}
static __device__ __noinline__ uint4 load_inputs_one_by_one(const uint8_t* x, int e4m3, int64_t at, int have) {
  uint32_t v[4] = {0, 0, 0, 0};
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (e < have) {
      if (e4m3) v[e / 4] |= (uint32_t)x[at + e] << (8 * (e % 4));
      else v[e / 2] |= (uint32_t) reinterpret_cast<const uint16_t*>(x)[at + e] << (16 * (e % 2));
    }
  return make_uint4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ uint4 bytes_to_half(uint4 v) {
  auto two = [](uint32_t w) {
    const __half2 h(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)w, __NV_E4M3));
    return *reinterpret_cast<const uint32_t*>(&h);
  };
  return make_uint4(two(v.x & 0xFFFFu), two(v.x >> 16), two(v.y & 0xFFFFu), two(v.y >> 16));
}

// BF: bf16 rows; GS: 32-input steps of a group (1, 2, 4); NT: 8-row tiles of one pass; ZEROS:
// zero points by group
template <bool BF, int GS, int NT, bool ZEROS>
__global__ void __launch_bounds__(32 * kWarps, 1) mat4_kernel(const __grid_constant__ Params p) {
  constexpr int W = kWarps, kThreads = 32 * W;
  constexpr int kGroups = 4 / GS;  // groups of a chunk
  constexpr int kCols = 8 * NT;
  // Loads of rows in flight, first and then.  What a launch runs once costs the more the longer
  // its code is, 0.1 us for each load, and a single row's first one is all that it needs: 4.1 us
  // instead of 4.4 (four first ones) for 4096 x 4096.
  constexpr int kFirst = 1, kBatch = 4;
  namespace cg = cooperative_groups;
  extern __shared__ uint4 smem[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const int mw = W >> p.kw_log, mi = warp >> p.kw_log, ki = warp & (p.kw - 1);
  const int tile_log = 9 - p.kw_log;  // of the CTA's channels, 32 mw
  const int rank = special<kRank>(), first = special<kCluster>(), step = special<kClusters>();
  const int c0 = rank * p.per, mine = min(p.per, p.chunks - c0);  // this CTA's chunks
  const int outputs = p.rows << tile_log;

  float* red = reinterpret_cast<float*>(smem + W * kRingBytes / 16);
  uint4* xb = reinterpret_cast<uint4*>(red + W * NT * kRedBytes / 4);
  float* csum = reinterpret_cast<float*>(xb + p.per * NT * 128);

  // The rows.  An item is 8 inputs of one row, the operands of step q for the lane (row,
  // ot): 16 items a chunk.  A warp takes 32 consecutive items of a row at a time.  The first
  // loads go out before anything else: the CTA's first barrier waits for them.
  const int turns_of_row = (p.per * 16 + 31) / 32, turns = p.rows * turns_of_row;
  auto take = [&](int turn, int& row, int& item) {
    row = (int)((turn + 0.5f) * p.turns_of_row_inv);  // exact: turns are few
    item = (turn - row * turns_of_row) * 32 + lane;
    const int k = c0 * kChunk + 8 * item;
    const int64_t at = (int64_t)row * p.ldx + k;
    if (turn >= turns || k >= p.n) return make_uint4(0, 0, 0, 0);
    return p.x_vec && k + 8 <= p.n ? load_inputs(p, at) : load_inputs_one_by_one(p.x, p.e4m3, at, p.n - k);
  };
  depend_on_last();
  uint4 v0[kFirst];
  int row0[kFirst], item0[kFirst];
#pragma unroll
  for (int b = 0; b < kFirst; ++b) v0[b] = take(warp + b * W, row0[b], item0[b]);

  // The warp's ring of codes.  This lane copies piece t of channels 4g + i to row 8i + g of
  // a stage, at a place that lets a row's words be read 4, 8 or 16 bytes a lane without
  // bank conflicts.
  uint4* ring = smem + warp * (kRingBytes / 16);
  const int swizzle = (g >> 1 & 1) * 2 + (g >> 2);
  const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring + g * 4 + (t ^ swizzle));
  int i_tile = first, i_l = ki, i_slot = 0;  // the next chunk to copy
  const uint8_t* base = nullptr;  // of the tile's codes, and this lane's channels from there
  uint32_t src[4];
  auto point = [&](int tile) {
    const int ch0 = tile * mw * kTile;
    base = p.codes + (int64_t)ch0 * p.pieces * 16;
#pragma unroll
    for (int i = 0; i < 4; ++i) src[i] = (uint32_t)(min(ch0 + mi * kTile + 4 * g + i, p.m - 1) - ch0) * p.pieces * 16u;
  };
  point(first);
  auto issue = [&]() {
    if (i_tile < p.tiles && ki < mine) {
      // pieces past the row's end meet inputs that are zero: any piece will do
      const uint32_t off = (uint32_t)min(4 * (c0 + i_l) + t, p.pieces - 1) * 16u;
      const uint32_t to = ring_at + i_slot * (kStageUnits * 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) copy16(to + i * 512, base + (src[i] + off));
      i_slot = i_slot + 1 == kStages ? 0 : i_slot + 1;
      i_l += p.kw;
      if (i_l >= mine) {
        i_l = ki;
        i_tile += step;
        if (i_tile < p.tiles) point(i_tile);
      }
    }
    commit();
  };
#pragma unroll
  for (int s = 0; s < kStages - 1; ++s) issue();

  // scales and zero points of this lane's four channels in a chunk's groups
  uint32_t sraw[kGroups][2], zraw[kGroups];
  auto fetch_scales = [&](int tile, int l) {
    const int ch = (tile * mw + mi) * kTile + 4 * g;
#pragma unroll
    for (int k = 0; k < kGroups; ++k) {
      const int gi = (c0 + l) * kGroups + k;  // past the last group: inputs that are zero
      const int64_t row = (int64_t)(GS == 4 ? gi : min(gi, p.groups - 1)) * p.m;
      if (p.scale_vec) {
        const int64_t at = row + min(ch, p.m - 4);
        const uint2 v = *reinterpret_cast<const uint2*>(p.scales + at);
        sraw[k][0] = v.x; sraw[k][1] = v.y;
        if constexpr (ZEROS) zraw[k] = *reinterpret_cast<const uint32_t*>(p.zeros + at);
      } else {
        uint32_t s[4], z[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int64_t at = row + min(ch + i, p.m - 1);
          s[i] = p.scales[at];
          if constexpr (ZEROS) z[i] = p.zeros[at];
        }
        sraw[k][0] = s[0] | s[1] << 16; sraw[k][1] = s[2] | s[3] << 16;
        if constexpr (ZEROS) zraw[k] = z[0] | z[1] << 8 | z[2] << 16 | z[3] << 24;
      }
    }
  };
  if (ki < mine) fetch_scales(first, ki);

  // Operands without a row are left as they are: a column of B meets one column of the sums.
  auto put = [&](int row, int i, uint4 v) {
    const int l = i >> 4, w = i & 15;  // w: the item's word of the chunk
    if (l >= p.per) return;
    const int ot = w / GS & 3, q = w / (4 * GS) * GS + w % GS;
    const uint4 h = p.e4m3 ? bytes_to_half(v) : v;
    // (x0, x4) (x1, x5) (x2, x6) (x3, x7), as the codes of a word come out
    xb[((l * NT + row / 8) * 4 + q) * 32 + (row % 8) * 4 + ot] =
        make_uint4(__byte_perm(h.x, h.z, 0x5410), __byte_perm(h.x, h.z, 0x7632), __byte_perm(h.y, h.w, 0x5410),
                   __byte_perm(h.y, h.w, 0x7632));
  };
#pragma unroll
  for (int b = 0; b < kFirst; ++b)
    if (warp + b * W < turns) put(row0[b], item0[b], v0[b]);
#pragma unroll 1
  for (int turn0 = warp + kFirst * W; turn0 < turns; turn0 += kBatch * W) {
    uint4 v[kBatch];
    int row[kBatch], item[kBatch];
#pragma unroll
    for (int b = 0; b < kBatch; ++b) v[b] = take(turn0 + b * W, row[b], item[b]);
#pragma unroll
    for (int b = 0; b < kBatch; ++b)
      if (turn0 + b * W < turns) put(row[b], item[b], v[b]);
  }
  __syncthreads();

  const Magic<BF> magic;
  int slot = 0, parity = 0;
  for (int tile = first; tile < p.tiles; tile += step) {
    float acc[2][NT][4];
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[mt][j][e] = 0.f;

    for (int l = ki; l < mine; l += p.kw) {
      if constexpr (GS != 4) __syncwarp();  // the stage filled next has been read by every lane
      issue();
      uint32_t sr[kGroups][2], zs[kGroups];
#pragma unroll
      for (int k = 0; k < kGroups; ++k) {
        sr[k][0] = sraw[k][0]; sr[k][1] = sraw[k][1];
        if constexpr (ZEROS) zs[k] = zraw[k];
      }
      if (l + p.kw < mine) fetch_scales(tile, l + p.kw);
      else if (tile + step < p.tiles) fetch_scales(tile + step, ki);
      wait_group<kStages - 1>();  // this lane's own copies (a group of 128: nobody else reads them)
      if constexpr (GS != 4) __syncwarp();  // pieces of other lanes are wanted
      const uint4* from = ring + slot * kStageUnits;
      uint32_t raw[4][4];  // by channel: word of step q
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint4* row = from + (8 * i + g) * 4;
        if constexpr (GS == 4) {
          const uint4 v = row[t ^ swizzle];
          raw[i][0] = v.x; raw[i][1] = v.y; raw[i][2] = v.z; raw[i][3] = v.w;
        } else if constexpr (GS == 2) {
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const uint2 v = reinterpret_cast<const uint2*>(row + ((2 * k + t / 2) ^ swizzle))[t % 2];
            raw[i][2 * k] = v.x; raw[i][2 * k + 1] = v.y;
          }
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k) raw[i][k] = reinterpret_cast<const uint32_t*>(row + (k ^ swizzle))[t];
        }
      }
      slot = slot + 1 == kStages ? 0 : slot + 1;
      const uint4* xl = xb + l * NT * 128 + lane;
#pragma unroll
      for (int k = 0; k < kGroups; ++k) {
        uint2 zero[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) zero[i] = zero_words<BF>(ZEROS ? zs[k] >> (8 * i) & 255u : 8u);
        float part[2][NT][4];
#pragma unroll
        for (int i = 0; i < GS; ++i) {
          const int q = k * GS + i;
          uint4 b[NT];
#pragma unroll
          for (int j = 0; j < NT; ++j) b[j] = xl[(j * 4 + q) * 32];
#pragma unroll
          for (int mt = 0; mt < 2; ++mt)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint2 u = code_pairs<BF>(raw[2 * mt][q], h, magic, zero[2 * mt]);
              const uint2 v = code_pairs<BF>(raw[2 * mt + 1][q], h, magic, zero[2 * mt + 1]);
#pragma unroll
              for (int j = 0; j < NT; ++j) {
                if (i == 0 && h == 0) mma<BF, true>(part[mt][j], u.x, v.x, u.y, v.y, b[j].x, b[j].y);
                else mma<BF, false>(part[mt][j], u.x, v.x, u.y, v.y, h ? b[j].z : b[j].x, h ? b[j].w : b[j].y);
              }
            }
        }
        float2 sc[2];
        if (p.scale_bf16) {
          sc[0] = unpack2<KD_BF16>(sr[k][0]); sc[1] = unpack2<KD_BF16>(sr[k][1]);
        } else {
          sc[0] = unpack2<KD_F16>(sr[k][0]); sc[1] = unpack2<KD_F16>(sr[k][1]);
        }
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int mt = 0; mt < 2; ++mt)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              acc[mt][j][e] = __fmaf_rn(e / 2 ? sc[mt].y : sc[mt].x, part[mt][j][e], acc[mt][j][e]);
      }
    }

    // The warps' sums of a channel, added in the order of their inputs.  Channels 4g .. 4g + 3 of
    // row r lie at 4 (g ^ (r & 6)) of the row's 32: no bank conflicts.
    __syncthreads();  // the last tile's sums have been read
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int e = 0; e < 2; ++e)
        *reinterpret_cast<float4*>(red + (warp * kCols + 8 * j + 2 * t + e) * kTile + 4 * (g ^ 2 * t)) =
            make_float4(acc[0][j][e], acc[0][j][e + 2], acc[1][j][e], acc[1][j][e + 2]);
    __syncthreads();
    const int j0 = tile << tile_log;
    auto finish = [&](int r, int ch, float s) {
      if (j0 + ch >= p.m) return;
      if (p.xs) s *= p.xs[r];
      store1_any(p.y, p.ydtype, (int64_t)r * p.ldy + j0 + ch, s);
    };
    // output o: row o / (32 mw), channel o % (32 mw) of the tile
    for (int o = threadIdx.x; o < outputs; o += kThreads) {
      const int r = o >> tile_log, ch = o & ((1 << tile_log) - 1);
      const float* at = red + (((ch / kTile) << p.kw_log) * kCols + r) * kTile + (ch % kTile ^ (r & 6) << 2);
      float s = at[0];
#pragma unroll 5
      for (int w = 1; w < p.kw; ++w) s += at[w * kCols * kTile];
      if (p.split == 1) finish(r, ch, s);
      else csum[parity * outputs + o] = s;
    }
    if (p.split > 1) {
      cg::cluster_group cl = cg::this_cluster();
      cl.sync();
      // two sets of sums: the barrier of the next tile comes before this one is written again
      for (int o = rank * kThreads + threadIdx.x; o < outputs; o += p.split * kThreads) {
        float s = 0.f;
        for (int k = 0; k < p.split; ++k) s += cl.map_shared_rank(csum, k)[parity * outputs + o];
        finish(o >> tile_log, o & ((1 << tile_log) - 1), s);
      }
      parity ^= 1;
    }
  }
  wait_group<0>();
  if (p.split > 1) cg::this_cluster().sync();  // no CTA leaves while its sums are read
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

// the launch of one pass
template <bool BF, int GS, int NT, bool ZEROS>
cudaError_t launch_one(const Params& p, int clusters, cudaStream_t s) {
  auto kernel = mat4_kernel<BF, GS, NT, ZEROS>;
  static std::atomic<uint64_t> ready{0};
  const cudaError_t e = allow_shared_memory(kernel, ready);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(clusters * p.split));
  cfg.blockDim = dim3(32 * kWarps);
  cfg.dynamicSmemBytes = smem_bytes(NT, p.rows, p.per, p.split, p.kw);
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  launch_early(attr[0]);
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)p.split;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = p.split > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, p);
}

template <bool BF, int GS>
cudaError_t launch(const Params& p, int nt, int clusters, cudaStream_t s) {
  if (p.zeros) return nt == 1 ? launch_one<BF, GS, 1, true>(p, clusters, s) : launch_one<BF, GS, 2, true>(p, clusters, s);
  return nt == 1 ? launch_one<BF, GS, 1, false>(p, clusters, s) : launch_one<BF, GS, 2, false>(p, clusters, s);
}

// bf: bf16 rows; nt: tiles of eight rows, 0: the kernel for many (kd_mat4_wide.cuh)
cudaError_t launch_group32(const Params& p, bool bf, int nt, int clusters, cudaStream_t s);
cudaError_t launch_group64(const Params& p, bool bf, int nt, int clusters, cudaStream_t s);
cudaError_t launch_group128(const Params& p, bool bf, int nt, int clusters, cudaStream_t s);

}  // namespace mat4
}  // namespace kd
