// Attention of few rows over a paged cache of 4-bit keys and values (kd_attention_4bit):
//
//     x_p = scale sum_g (step_g(p) sum_{c in g} code_c(p) q_c + low_g(p) sum_{c in g} q_c)
//     out_c = sum_p w_p (low_g(p) + step_g(p) code_c(p)) / sum_p w_p,   w_p = 2^(x_p log2 e - m)
//
// one pass over the codes with the running maximum m and sum of the softmax, on the tensor cores in
// fp16 (mma.sync m16n8k16), with the codes as the A operand of both products and the rows (query
// tokens times the heads that share a key head) as the eight columns of B.  The codes go from their word to
// the operand in registers; tcgen05 would want them stored as 16-bit operands first, and its
// smallest products have no use for eight rows.
//
// Codes.  A code masked out of its word is an fp16 number as it stands: c in a half's low bits is
// c 2^-24, four bits higher 16 c 2^-24, both below fp16's normal range.  No arithmetic makes them
// operands.  The tensor cores take such numbers exactly but sum products by the operands' exponents, of which these
// have the lowest: what lies far below the largest product is cut off, the more the smaller c 2^-24
// is.  So keys' codes all stand four bits higher (a shift for three of four), for log-sum-exps within 1e-6;
// values' tiles have even channels' codes in one half of their rows and even plus 16 odd ones (a byte as it
// stands) in the other, from whose sums the odd channels' come off in the end.  Cut off there is up to 2^-12 of the largest
// weight times step of sixteen positions, half as much as that one's own rounding takes from a code next to the middle (four bits
// higher it is 2^-16, for 1 to 5 % of the time: drafted tokens 37.7 -> 39.1 us, a long document 37.3 -> 38.1; outputs of 40 to
// 131072 positions are as near either way).
//
// Middles.  Values count from 8, value = low + 8 step + step (c - 8), or rounded weights would be
// off by a share of the whole range: 8 times the step's weights as they are rounded (a product with ones) comes
// off the sums before each step's products, and w times the middle, low + 8 step, is summed in fp32.
//
// Weights.  w step is the B operand, rounded to fp16: the one rounding to fewer bits here, an error
// of up to 2^-11 of a value's distance from its group's middle.  Each row has a power of two for each group that brings the
// largest w step that the row has seen so far to 2^5 .. 2^14 (the sums are rescaled where it changes), so that what
// falls below fp16's normal range is off by 2^-30 of the largest at most: other rows' steps, large steps without weight and other
// groups' take no digits.  (One power of two for all, from the largest step, was 1 to 3 % faster, with groups of 32 11 to 16 %, and
// lost them.)  q is brought to 2^14 .. 2^15 by a power of two for each row: its digits stay but those below 2^-38 of the row's
// largest channel, where fp16 ends; scores are exact products summed in fp32.  (16-bit outputs of 5000 positions
// are off by 2.9e-4 of 64 bits' in the root of the mean square, of which 2.1e-4 are their own rounding; with the ones as
// small as the codes it was 7.6e-4.)
//
// Maximum.  m follows the scores only where one exceeds it by more than 8 (w up to 2^8, for which
// the scaling leaves room): a vote of the warp instead of a reduction over it for each step.
//
// A step of a warp is 32 positions, two tiles.  Rows and weights cost as much as the codes do, so blocks of at most
// four rows (PACK) give each tile four of the eight columns: scores of both tiles are picked into one set of
// registers, exponentials, scales and the transposed weights (movmatrix) are made once for both, and
// the values' operands have zeros in the other tile's columns.
//
// Copies.  Codes and scales of 16 positions are contiguous blocks of a page; they stream through each warp's own
// ring of two steps (cp.async): no barrier of the CTA stands in the loop.  Rows of codes are an odd number of
// 16-byte pieces apart there, and ldmatrix (transposing for the values) reads them free of bank conflicts
// as the operands' lanes want them.
//
// Mapping.  Four warps a CTA, two to four CTAs an SM, take the steps of an item (a sequence, a key head, a block of rows) in
// turn, each with its own m and sums, joined once at the end in a fixed order.  Two ways to share out
// the work (kd_attn4.cu has the rule): a cluster of up to eight CTAs has an item to itself and joins in
// distributed shared memory (TEAM; short items), or all CTAs of one round have equal shares of all
// positions of all items, which each finds from the lengths, and a second launch joins what is cut.
//
// Long batches are bound by these copies: without any arithmetic those of 32 sequences of 8192 positions (8 key heads of
// 128, 0.30 GB) take 64 us, with it 62, where HBM would take 44.  The start (2.4 us until the share is known, 6.5 until the
// first codes are there), shares that end unlike on SMs unlike far from memory (45 to 66 us) and the join (3 us) are in
// both.  The next wait of these kernels is for instructions: the step stands twice, unrolled, in each.  Measured (device
// time, inputs larger than L2): 32 sequences of 2000 to 8192 positions 53 us (floor 27), one of 131072 38 us (22), 16 of
// up to 4096 with up to 8 drafted tokens 38 us (6.6), one of 1001 positions with 32 key heads 6.9 us (0.7).
// 128 or 168 registers (255 above 128 channels) spill up to 116 bytes in some instances, groups of 32 the most.
#pragma once
#include <cooperative_groups.h>

#include <atomic>

#include "kd_cache4.cuh"

namespace kd {
namespace attn4 {

using namespace cache4;

constexpr int kWarps = 4;
constexpr int kRows = 8;      // of a block: columns of a tensor-core tile
constexpr int kTile = 16;     // positions of a tensor-core tile, all on one page
constexpr int kTiles = 2;     // of one step of a warp
constexpr int kChunk = kTiles * kWarps;  // tiles of one step of a CTA: what work is shared out in
constexpr int kTeam = 8;      // CTAs of a cluster at most
constexpr int kBatch = 256;   // tiles whose places are looked up at a time

struct Params {
  Pages c;
  const uint16_t* q;
  uint16_t* out;
  float* lse;
  int64_t q_token, q_head, out_token, out_head;
  int64_t tokens;
  int heads, shared;            // query heads; of one key head
  int row_blocks;               // of a sequence: blocks of rows
  int team;                     // CTAs of a cluster with an item (sequence, key head, block of rows); 0: equal shares
  int causal, window;
  int room;                     // positions that the table has room for
  int bf16, q_vec, out_vec;
  float scale2;                 // scale log2 e
  struct Cut* cuts;             // of each item: where its parts are, in equal shares
  float2* part_ml;              // (m, sum) of each row of a CTA's first item and of its last, where they are cut
  float* part;                  // and their sums [CTA][first, last][row][part_row]
  int part_row;                 // d, up to a multiple of 4
};

// An item's parts: in place `slot` (two a CTA), then in the first places of the `more` CTAs that follow `owner`.
struct Cut {
  int owner, slot, more, unused;
};

// The rows and positions of a block of rows: the same for the kernel that sums and the one that joins.
struct Work {
  int64_t first;       // row of the sequence's first query token
  int before;          // position of that token
  int length, rows;    // rows: tokens times heads, from the block's first on
  int lo, hi;          // positions that some row sees
  int all_lo, all_hi;  // positions that every row sees
  int tile, tiles;     // of the positions lo .. hi
  int chunks;          // of kChunk tiles; one for rows that see nothing, none for no rows
};
__device__ __forceinline__ int clamp_to(int v, int most) { return max(0, min(v, most)); }
// the first position that the row at `pos` sees through its window
__device__ __forceinline__ int window_from(const Params& p, int pos, int length) {
  return (int)max((int64_t)0, min((int64_t)pos + 1 - p.window, (int64_t)length));
}
// token of a row, of its sequence's
__device__ __forceinline__ int token_of(const Params& p, int row) {
  return p.shared == 1 ? row : (int)((unsigned)row / (unsigned)p.shared);
}
__device__ __forceinline__ Work work_of(const Params& p, int s, int block, int of_block) {
  Work w;
  const int length = p.c.lengths[s];
  int count = p.c.most;
  w.first = (int64_t)s * p.c.most;
  if (p.c.starts) {
    w.first = p.c.starts[s];
    count = (int)max((int64_t)0, min((int64_t)p.c.starts[s + 1] - w.first, (int64_t)INT32_MAX));
  }
  w.length = max(length, 0);
  w.before = w.length - count;
  const int r0 = block * of_block, rows = min(count, p.c.most) * p.shared;  // the host has checked their range
  w.rows = clamp_to(rows - r0, of_block);
  w.lo = w.all_lo = 0;
  w.hi = w.all_hi = w.length;
  if (p.causal) {
    const int a = w.before + token_of(p, r0), b = w.before + token_of(p, max(r0 + w.rows - 1, r0));  // first, last position
    w.hi = clamp_to(b + 1, w.length);
    w.all_hi = clamp_to(a + 1, w.length);
    if (p.window) {
      w.lo = window_from(p, a, w.length);
      w.all_lo = window_from(p, b, w.length);
    }
  }
  // positions past the table's room have no page: none is visited, and rows that see one are NaN
  w.hi = min(w.hi, p.room);
  w.tile = w.lo / kTile;
  w.tiles = w.hi > w.lo ? (w.hi + kTile - 1) / kTile - w.tile : 0;
  w.chunks = w.rows == 0 ? 0 : max((w.tiles + kChunk - 1) / kChunk, 1);
  return w;
}

// does the row of a token, `nth` of its sequence's, see positions past the table's room?
__device__ __forceinline__ bool past_table(const Params& p, const Work& w, int nth) {
  return (p.causal ? min(w.before + nth + 1, w.length) : w.length) > p.room;
}

// The first row's number of a tile (of 16 positions on one page) for the first key head, -1 on a bad page.
__device__ __forceinline__ int64_t tile_row(const Params& p, int s, int tile) {
  const unsigned of_page = (unsigned)p.c.page / kTile, nth = p.c.page_log >= 0 ? (unsigned)tile >> (p.c.page_log - 4) : (unsigned)tile / of_page;
  const int page = p.c.table[s * p.c.ld_table + nth];  // tiles lie within the table's room
  if ((unsigned)page >= (unsigned)p.c.pages) return -1;
  return (int64_t)page * p.c.heads * p.c.page + (int)(tile - nth * of_page) * kTile;
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
// the same with sums that start from 0
__device__ __forceinline__ void mma_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                          uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%10, %10, %10, %10};\n"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
// Matrices of 8 rows of 16 bytes, as 16-bit units: to a lane units 2 t4, 2 t4 + 1 of row g8, or (TURN) unit g8 of
// rows 2 t4, 2 t4 + 1.  Lane l gives the address of row l % 8 of matrix l / 8.
template <bool TURN>
__device__ __forceinline__ void load_matrices(uint32_t (&d)[4], uint32_t at) {
  if constexpr (TURN)
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(d[0]), "=r"(d[1]), "=r"(d[2]), "=r"(d[3]) : "r"(at) : "memory");
  else
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(d[0]), "=r"(d[1]), "=r"(d[2]), "=r"(d[3]) : "r"(at) : "memory");
}
template <bool TURN>
__device__ __forceinline__ void load_two_matrices(uint32_t (&d)[4], uint32_t at) {
  if constexpr (TURN)
    asm volatile("ldmatrix.sync.aligned.m8n8.x2.trans.shared.b16 {%0, %1}, [%2];" : "=r"(d[0]), "=r"(d[1]) : "r"(at) : "memory");
  else asm volatile("ldmatrix.sync.aligned.m8n8.x2.shared.b16 {%0, %1}, [%2];" : "=r"(d[0]), "=r"(d[1]) : "r"(at) : "memory");
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
__device__ __forceinline__ float log2_of(float x) {  // off by 2^-22 of it at most, or of 1 where it is less
  float r;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float low_half(uint32_t w) { return __half2float(__ushort_as_half((unsigned short)w)); }
__device__ __forceinline__ float high_half(uint32_t w) { return __half2float(__ushort_as_half((unsigned short)(w >> 16))); }

constexpr float kNone = -__builtin_inff();
// Weights times steps as fp16 operands: the largest so far between 2^5 and kMost (small ones as many times larger as that takes,
// kUpMost at most, which brings the smallest step there)
constexpr float kMost = 0x1p14f, kUpMost = 0x1p29f;
constexpr float kMostLog = 13.99f;  // the logarithm of kMost, less what log2_of is off by

// NC: 32-channel pieces of a row; GS: of a group
template <int NC, int GS>
struct Shape {
  static constexpr int kGroups = (NC + GS - 1) / GS;
  static constexpr int kRows = attn4::kRows;
  static constexpr int kStages = 2;
  static constexpr int kStride = 4 * (NC | 1);                       // words of a row of codes in the ring
  // words of a stage, keys or values
  static constexpr int kCodes = kTiles * kTile * kStride, kScales = kTiles * kTile * kGroups;
  static constexpr int kStage = 2 * (kCodes + kScales);
  static constexpr int kSumTiles = 2 * NC;                           // tiles of 16 channels of the values' sums
  static constexpr int kSums = 32 * NC + 4;                          // floats of a row of a warp's sums
  static constexpr int kQueries = 64 * NC + 64;                      // bytes of a row of queries as operands
  static constexpr size_t kRing = (size_t)kWarps * kStages * kStage * 4, kJoin = (size_t)kWarps * kRows * kSums * 4;
  static constexpr size_t kBytes = (kRing > kJoin ? kRing : kJoin) + kBatch * 16 + (size_t)kWarps * kRows * 8 +
                                    kRows * (kQueries + 4 * (kGroups + 1));
};

// fp16 or bf16 bits as a float
__device__ __forceinline__ float wide(const Params& p, uint32_t bits) {
  return p.bf16 ? __uint_as_float(bits << 16) : __half2float(__ushort_as_half((unsigned short)bits));
}
__device__ __forceinline__ uint16_t narrow(const Params& p, float v) {
  return p.bf16 ? __bfloat16_as_ushort(__float2bfloat16_rn(v)) : __half_as_ushort(__float2half_rn(v));
}

// The item (s, head, block) and its chunk that chunk `from` of all falls on, and all chunks' number; the whole warp
// looks, 32 sequences at a time.
struct Start {
  int s, head, block, chunk, total;
};
__device__ __forceinline__ int chunks_of_head(const Params& p, int s) {
  int n = 0;
  if (s < p.c.seqs)
    for (int b = 0; b < p.row_blocks; ++b) {
      const int of = work_of(p, s, b, kRows).chunks;
      if (of == 0) break;  // no rows from here on
      n += of;
  }
  return n;
}
__device__ __forceinline__ Start start_of(const Params& p, int blocks, int block, int& per) {
  const int lane = threadIdx.x & 31;
  Start at{-1, 0, 0, 0, 0};
  int first = chunks_of_head(p, lane);  // of the first 32 sequences, which are often all
  int total = first;
#pragma unroll 4
  for (int s = 32 + lane; s - lane < p.c.seqs; s += 32) total += chunks_of_head(p, s);
  at.total = __reduce_add_sync(~0u, total) * p.c.heads;
  per = (at.total + blocks - 1) / blocks;  // blocks are fewer than chunks fit 31 bits
  const int64_t from64 = (int64_t)block * per;
  if (from64 >= at.total) return at;
  int from = (int)from64;
  for (int s0 = 0;; s0 += 32) {
    const int mine = (s0 ? chunks_of_head(p, s0 + lane) : first) * p.c.heads;
    int in = mine;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
      const int up = __shfl_up_sync(~0u, in, o);
      if (lane >= o) in += up;
    }
    const unsigned past = __ballot_sync(~0u, from < in);
    if (past) {
      const int which = __ffs(past) - 1, before = __shfl_sync(~0u, in - mine, which), of = __shfl_sync(~0u, mine, which) / p.c.heads;
      at.s = s0 + which;
      at.chunk = from - before;
      at.head = at.chunk / of;
      at.chunk -= at.head * of;
      for (int n; at.chunk >= (n = work_of(p, at.s, at.block, kRows).chunks); ++at.block) at.chunk -= n;
      return at;
    }
    from -= __shfl_sync(~0u, in, 31);
  }
}

// four channels of a row from ch on, over the row's total (0: nothing was seen)
__device__ __forceinline__ void put(const Params& p, uint16_t* out, int ch, float4 v, float total) {
  const float over = total == 0.f ? 0.f : 1.f / total;
  const float of[4] = {v.x * over, v.y * over, v.z * over, v.w * over};
  uint16_t bits[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) bits[e] = narrow(p, total != total ? total : of[e]);
  if (p.out_vec) {
    *reinterpret_cast<uint2*>(out + ch) = make_uint2(bits[0] | (uint32_t)bits[1] << 16, bits[2] | (uint32_t)bits[3] << 16);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (ch + e < p.c.d) out[ch + e] = bits[e];
  }
}
__device__ __forceinline__ void put_lse(const Params& p, int64_t at, float top, float total) {
  if (p.lse) p.lse[at] = total == 0.f ? kNone : (top + log2f(total)) * 0.693147180559945f;
}

// Joins the parts of a cluster's CTAs, which lie in the first rows of their `sums` and `ml` (where a CTA has any),
// in the order of their ranks; a row is one CTA's.
template <class Z>
__device__ __forceinline__ void join_team(const Params& p, const Work& w, int head, int block, bool any, float* sums, float2* ml) {
  namespace cg = cooperative_groups;
  cg::cluster_group cl = cg::this_cluster();
  if (!any)
    for (int r = threadIdx.x; r < Z::kRows; r += 32 * kWarps) ml[r] = make_float2(kNone, 0.f);
  cl.sync();
  const int rank = special<kRank>(), quads = p.part_row / 4;
  for (int i = threadIdx.x;; i += 32 * kWarps) {
    const int nth = i / quads, r = rank + nth * p.team, ch = 4 * (i - nth * quads);
    if (r >= w.rows) break;
    const int in = block * Z::kRows + r, token = token_of(p, in), h = head * p.shared + in - token * p.shared;
    const int64_t t = w.first + token;
    if (t < 0 || t >= p.tokens) continue;
    float top = kNone, total = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    float2 n[kTeam];
#pragma unroll
    for (int k = 0; k < kTeam; ++k) {
      n[k] = k < p.team ? cl.map_shared_rank(ml, k)[r] : make_float2(kNone, 0.f);
      top = fmaxf(top, n[k].x);
    }
    float4 v[kTeam];  // all on their way together
#pragma unroll
    for (int k = 0; k < kTeam; ++k) {
      v[k] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (n[k].x != kNone) v[k] = *reinterpret_cast<const float4*>(cl.map_shared_rank(sums, k) + r * Z::kSums + ch);
    }
#pragma unroll
    for (int k = 0; k < kTeam; ++k) {
      const float f = n[k].x == kNone ? 0.f : exp2_of(n[k].x - top);
      total += n[k].x == kNone ? n[k].y : n[k].y * f;  // no sums there, or NaN
      o.x = __fmaf_rn(v[k].x, f, o.x);
      o.y = __fmaf_rn(v[k].y, f, o.y);
      o.z = __fmaf_rn(v[k].z, f, o.z);
      o.w = __fmaf_rn(v[k].w, f, o.w);
    }
    put(p, p.out + t * p.out_token + h * p.out_head, ch, o, total);
    if (ch == 0) put_lse(p, t * p.heads + h, top, total);
  }
  cl.sync();  // no CTA leaves while its sums are read
}

// CTAs that an SM has: of heads of up to 128 channels four where they are many and short, three where each has a share of
// everything (168 registers instead of 128: 32 sequences of 8192 positions 2.7 us less)
constexpr int on_sm(int nc, bool team) { return nc > 4 ? 2 : team ? 4 : 3; }

// TEAM: a cluster of p.team CTAs has an item to itself; else all CTAs have equal shares of all of them
// PACK: blocks have at most four rows, and the two tiles of a step four columns each: what follows the key
// products is done once for both
template <int NC, int GS, bool TEAM, bool PACK>
__global__ void __launch_bounds__(32 * kWarps, on_sm(NC, TEAM)) attn4_kernel(const __grid_constant__ Params p) {
  using Z = Shape<NC, GS>;
  constexpr int GN = Z::kGroups, ST = Z::kStages, S = Z::kStride;
  // rows; and sets of elements of a step: a tile's, or those of both tiles together
  constexpr int kColumns = PACK ? 4 : 8, kSets = PACK ? 1 : kTiles;
  extern __shared__ uint4 smem[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g8 = lane >> 2, t4 = lane & 3;
  // shared memory: the ring, where sums are joined too; places; (m, sum) of the warps' rows; queries, their
  // groups' sums and powers of two
  char* after = reinterpret_cast<char*>(smem) + (Z::kRing > Z::kJoin ? Z::kRing : Z::kJoin);
  longlong2* place = reinterpret_cast<longlong2*>(after);
  float2* ml = reinterpret_cast<float2*>(place + kBatch);
  char* queries = reinterpret_cast<char*>(ml + kWarps * Z::kRows);
  float* query_sums = reinterpret_cast<float*>(queries + Z::kRows * Z::kQueries);
  depend_on_last();

  // This CTA's share: `left` chunks from chunk `chunk` of item (s, head, block) on.
  int s, head, block, chunk = 0, left;
  if constexpr (TEAM) {
    int at = special<kCluster>();
    block = at % p.row_blocks;
    at /= p.row_blocks;
    head = at % p.c.heads;
    s = at / p.c.heads;
    left = INT32_MAX;
  } else {
    int per;
    const Start at = start_of(p, gridDim.x, blockIdx.x, per);
    if (at.s < 0) return;
    left = min(per, at.total - (int)blockIdx.x * per);
    s = at.s;
    head = at.head;
    block = at.block;
    chunk = at.chunk;
  }
  const int share = left;
  constexpr int row_bytes = 16 * NC, scale_bytes = 4 * GN;
  // the ring: this lane's pieces of a tile
  uint32_t* ring = reinterpret_cast<uint32_t*>(smem) + warp * ST * Z::kStage;
  const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring);
  constexpr int pieces = kTile * NC;  // 16-byte pieces of a tile's keys
  uint32_t to[(NC + 1) / 2];
#pragma unroll
  for (int i = 0; i < (int)(sizeof(to) / 4); ++i) {
    const int n = lane + 32 * i, row = n / NC;
    to[i] = (uint32_t)(row * S * 4 + (n - row * NC) * 16);
  }

  for (;;) {
    const Work w = work_of(p, s, block, Z::kRows);
    if constexpr (TEAM) {
      if (w.rows == 0) return;
      left = (w.chunks + p.team - 1) / p.team;
      chunk = special<kRank>() * left;
    }
    const int n_chunks = min(w.chunks - chunk, left);
    // only a part of the item; in a cluster the same for all its CTAs, of which all or none take part in the join
    const bool cut = (TEAM ? left : n_chunks) < w.chunks;
    if (n_chunks > 0) {
      const int first_tile = w.tile + chunk * kChunk, tiles = min(n_chunks * kChunk, w.tiles - chunk * kChunk);
      const int share_hi = min(w.hi, (first_tile + tiles) * kTile);  // where the part's positions end

      // Where a batch's tiles lie, in bytes of codes and scales from the cache's first row: -1 on a bad page.
      auto look_up = [&](int b0, int n) {
        bool bad = false;
        for (int i = threadIdx.x; i < n; i += 32 * kWarps) {
          const int64_t first = tile_row(p, s, first_tile + b0 + i), row = first + (int64_t)head * p.c.page;
          place[i] = first < 0 ? make_longlong2(-1, 0) : make_longlong2(row * row_bytes, row * scale_bytes);
          bad |= first < 0;
        }
        return bad;
      };
      auto issue = [&](int first, int n, int stage) {  // tiles first, first + 1 of the batch's n
#pragma unroll
        for (int i = 0; i < kTiles; ++i) {
          if (first + i >= n) break;
          const longlong2 from = place[first + i];
          const int64_t code = max((int64_t)from.x, (int64_t)0) + lane * 16, scale = from.y + lane * 16;
          const uint32_t codes = ring_at + stage * (Z::kStage * 4) + i * kTile * S * 4;
#pragma unroll
          for (int k = 0; k < (int)(sizeof(to) / 4); ++k)
            if (lane + 32 * k < pieces) {
              copy16(codes + to[k], reinterpret_cast<const char*>(p.c.codes[0]) + code + 512 * k);
              copy16(codes + Z::kCodes * 4 + to[k], reinterpret_cast<const char*>(p.c.codes[1]) + code + 512 * k);
          }
          if (lane < 4 * GN) {
            const uint32_t scales = ring_at + stage * (Z::kStage * 4) + 2 * Z::kCodes * 4 + i * kTile * scale_bytes + lane * 16;
            copy16(scales, reinterpret_cast<const char*>(p.c.scales[0]) + scale);
            copy16(scales + Z::kScales * 4, reinterpret_cast<const char*>(p.c.scales[1]) + scale);
          }
        }
      };

      // The rows as operands, a warp a row: fp16 in eights of channels 0 4 1 5 2 6 3 7, with the
      // row's power of two and its sums over groups.
      const int r0 = block * Z::kRows;
      constexpr int kOfWarp = Z::kRows / kWarps;
      uint32_t raw[kOfWarp][4];  // lane l has channels 8 l .. 8 l + 7 (of 256)
#pragma unroll
      for (int i = 0; i < kOfWarp; ++i) {
        const int r = warp + i * kWarps, token = token_of(p, r0 + r);
        const int64_t t = w.first + token;
        raw[i][0] = raw[i][1] = raw[i][2] = raw[i][3] = 0;
        if (r < w.rows && t >= 0 && t < p.tokens && 8 * lane < p.c.d) {
          const uint16_t* q = p.q + t * p.q_token + (int64_t)(head * p.shared + (r0 + r) - token * p.shared) * p.q_head + 8 * lane;
          if (p.q_vec) {
            const uint4 u = *reinterpret_cast<const uint4*>(q);
            raw[i][0] = u.x; raw[i][1] = u.y; raw[i][2] = u.z; raw[i][3] = u.w;
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (8 * lane + e < p.c.d) raw[i][e / 2] |= (uint32_t)q[e] << (16 * (e % 2));
          }
        }
      }
      // the first batch's copies go out before the rows are worked on
      bool bad_pages = __syncthreads_or(look_up(0, min(tiles, kBatch)));
      auto prefetch = [&](int n) {
#pragma unroll
        for (int i = 0; i < ST - 1; ++i) {
          issue(kTiles * warp + i * kChunk, n, i);
          commit();
        }
      };
      prefetch(min(tiles, kBatch));
#pragma unroll
      for (int i = 0; i < kOfWarp; ++i) {
        const int r = warp + i * kWarps;
        float v[8];
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          v[e] = wide(p, raw[i][e / 2] >> (16 * (e % 2)) & 0xFFFFu);
          top = max(top, __float_as_uint(v[e]) & 0x7FFFFFFFu);
        }
        top = __reduce_max_sync(~0u, top);
        // 2^e <= max |q| < 2^(e + 1); an infinity or NaN stays what it is under any factor
        const int e2 = top >> 23 == 255 || top == 0 ? 0 : max((int)(top >> 23) - 127, -100);
        const float up = __uint_as_float((uint32_t)(14 - e2 + 127) << 23);
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          v[e] *= up;
          sum += v[e];
        }
        if (lane < 4 * NC)
          *reinterpret_cast<uint4*>(queries + r * Z::kQueries + 16 * lane) =
              make_uint4(pack2<KD_F16>(v[0], v[4]), pack2<KD_F16>(v[1], v[5]), pack2<KD_F16>(v[2], v[6]), pack2<KD_F16>(v[3], v[7]));
        // four lanes a piece of 32 channels
#pragma unroll
        for (int o = 1; o < 4 * GS && o < 32; o *= 2) sum += __shfl_xor_sync(~0u, sum, o);
        if (lane % (4 * GS) == 0 && lane / (4 * GS) < GN) query_sums[r * (GN + 1) + lane / (4 * GS)] = sum * 0x1p-14f;
        if (lane == 0) query_sums[r * (GN + 1) + GN] = __uint_as_float((uint32_t)(e2 + 127) << 23) * p.scale2;
      }
      __syncthreads();
      uint32_t qb[2 * NC][2];
      // of columns 2 t4, 2 t4 + 1: power of two of the row, and its sums over groups, both times scale log2 e
      float qs[GN][2], qe[2];
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const uint4 u = *reinterpret_cast<const uint4*>(queries + g8 % kColumns * Z::kQueries + 16 * (4 * c + t4));
        qb[2 * c][0] = u.x;
        qb[2 * c][1] = u.y;
        qb[2 * c + 1][0] = u.z;
        qb[2 * c + 1][1] = u.w;
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float* of_column = query_sums + (2 * t4 + j) % kColumns * (GN + 1);
        const float down = of_column[GN];
#pragma unroll
        for (int g = 0; g < GN; ++g) qs[g][j] = of_column[g] * down;
        qe[j] = down * 64.f;  // codes' 2^20 less q's 2^14
      }
      float acc[Z::kSumTiles][4];
      // of the columns: sums of weights times middles and of weights (of the positions g8 and g8 + 8 of the tiles
      // apart), m (0 before the first), and how far above it a score may lie (nothing may, before the first)
      float2 mids[GN][2], sum[2];
      float m[2], room[2];
#pragma unroll
      for (int i = 0; i < Z::kSumTiles; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][e] = 0.f;
#pragma unroll
      for (int g = 0; g < GN; ++g) mids[g][0] = mids[g][1] = make_float2(0.f, 0.f);
      m[0] = m[1] = 0.f;
      room[0] = room[1] = kNone;
      sum[0] = sum[1] = make_float2(0.f, 0.f);
      float up[GN][2];  // the columns' weights times steps, by powers of two
#pragma unroll
      for (int g = 0; g < GN; ++g) up[g][0] = up[g][1] = kUpMost;

      // One step.  EDGE: some row does not see all of it, or a page is bad.
      const uint32_t matrix_at = (lane & 15) * S * 4 + (lane >> 4) * 16;  // this lane's row of four matrices
      const int own = PACK ? t4 >> 1 : 0;  // whose elements are the lane's of a set: the second tile's, in the upper columns
      auto step = [&](auto edge, int stage, int position, bool bad0, bool bad1) {
        constexpr bool EDGE = decltype(edge)::value;
        const uint32_t codes = ring_at + stage * (Z::kStage * 4) + matrix_at;
        const uint32_t* kp = ring + stage * Z::kStage + 2 * Z::kCodes + (kTile * own + g8) * GN;
        const uint32_t* vp = kp + Z::kScales;
        float x[kSets][4];  // scores less m
        bool seen[kSets][4];
        int sees_lo[2], sees_hi[2];  // what the columns' rows see: positions from sees_lo on, below sees_hi
        if constexpr (EDGE) {
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int r = (2 * t4 + j) % kColumns, pos = w.before + token_of(p, r0 + r);
            sees_hi[j] = r >= w.rows ? 0 : min(share_hi, p.causal ? clamp_to(pos + 1, w.length) : w.length);
            sees_lo[j] = p.window ? window_from(p, pos, w.length) : 0;
          }
        }
#pragma unroll
        for (int i = 0; i < kSets; ++i) {
          float part[kTiles][4], low[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            x[i][e] = 0.f;
            low[e] = -m[e & 1];
          }
          uint32_t w[kTiles][4];  // positions g8, g8 + 8 of one piece, and of the next
#pragma unroll
          for (int c = 0; c < NC; ++c) {
#pragma unroll
            for (int n = 0; n < (PACK ? kTiles : 1); ++n) {
              const int of = PACK ? n : i;  // the tile
              if (c % 2 == 0) {
                if (c + 1 < NC) load_matrices<false>(w[n], codes + of * kTile * S * 4 + c * 16);
                else load_two_matrices<false>(w[n], codes + of * kTile * S * 4 + c * 16);
              }
              const uint32_t a = w[n][c % 2 * 2], b = w[n][c % 2 * 2 + 1];
              constexpr uint32_t mask = 0x00F000F0u;
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const uint32_t a0 = (h ? a >> 4 : a << 4) & mask, a1 = (h ? b >> 4 : b << 4) & mask;
                const uint32_t a2 = (h ? a >> 8 : a) & mask, a3 = (h ? b >> 8 : b) & mask;
                if (c % GS == 0 && h == 0) mma_first(part[n], a0, a1, a2, a3, qb[2 * c][0], qb[2 * c][1]);
                else mma(part[n], a0, a1, a2, a3, qb[2 * c + h][0], qb[2 * c + h][1]);
              }
            }
            if ((c + 1) % GS == 0 || c == NC - 1) {
              const uint32_t u = kp[i * kTile * GN + c / GS], v = kp[(i * kTile + 8) * GN + c / GS];
              const float s0 = low_half(u), l0 = high_half(u), s1 = low_half(v), l1 = high_half(v);
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                x[i][e] = __fmaf_rn(e < 2 ? s0 : s1, PACK && own ? part[1][e] : part[0][e], x[i][e]);
                low[e] = __fmaf_rn(e < 2 ? l0 : l1, qs[c / GS][e & 1], low[e]);
              }
            }
          }
#pragma unroll
          for (int e = 0; e < 4; e += 2) {
            const float2 of = fma2(make_float2(x[i][e], x[i][e + 1]), make_float2(qe[0], qe[1]), make_float2(low[e], low[e + 1]));
            x[i][e] = of.x;
            x[i][e + 1] = of.y;
            if constexpr (EDGE) {
              const int pos = position + kTile * (i + own) + g8 + 4 * e;
              const bool bad = i + own ? bad1 : bad0;
#pragma unroll
              for (int j = 0; j < 2; ++j) {
                seen[i][e + j] = pos < sees_hi[j] && pos >= sees_lo[j];
                x[i][e + j] = !seen[i][e + j] ? kNone : bad ? __int_as_float(0x7FC00000) : x[i][e + j];
              }
            }
          }
        }
        uint32_t vscale[kSets][GN][2];
        __half2 tops[GN];  // the largest step, in the low half
#pragma unroll
        for (int g = 0; g < GN; ++g) tops[g] = __half2half2(__ushort_as_half(0));
#pragma unroll
        for (int i = 0; i < kSets; ++i)
#pragma unroll
          for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int g = 0; g < GN; ++g) {
              uint32_t v = vp[(kTile * i + 8 * k) * GN + g];
              if constexpr (EDGE) {  // a position that no row sees may hold anything
                const int pos = position + kTile * (i + own) + g8 + 8 * k;
                if (pos >= share_hi || pos < w.lo) v = 0;
              }
              vscale[i][g][k] = v;
              tops[g] = __hmax2(tops[g], *reinterpret_cast<const __half2*>(&v));
            }
        bool grow = false;
        float most[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          most[j] = fmaxf(x[0][j], x[0][j + 2]);
          if (kSets == 2) most[j] = fmaxf(most[j], fmaxf(x[kSets - 1][j], x[kSets - 1][j + 2]));
          // the heaviest weight times the largest step, which need not be one position's, come to kMost at most
          float most_step = 0.f;
#pragma unroll
          for (int g = 0; g < GN; ++g) most_step = fmaxf(most_step, __low2float(tops[g]) * up[g][j]);
          grow |= most[j] > fminf(room[j], kMostLog - log2_of(most_step));
        }
        // A column moves for what it sees alone, so that what its row does not see changes none of its bits.
        if (__any_sync(~0u, grow)) {
          float f[2], less[2];  // what weighs less now, by `less` about, leaves room to what comes
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            float top = most[j];
            top = fmaxf(top, __shfl_xor_sync(~0u, top, 4));
            top = fmaxf(top, __shfl_xor_sync(~0u, top, 8));
            top = fmaxf(top, __shfl_xor_sync(~0u, top, 16));
            const bool moves = top > room[j], fresh = room[j] == kNone;
            // m moves up by `to`; a first one by whatever it is, with sums that are 0
            const float to = moves ? top : 0.f;
            f[j] = !moves ? 1.f : fresh ? 0.f : exp2_of(-to);
            less[j] = fresh ? 1.f : __uint_as_float((uint32_t)((int)ceilf(fminf(to, 64.f)) + 127) << 23);
            m[j] += to;
            if (moves) room[j] = 8.f;
#pragma unroll
            for (int i = 0; i < kSets; ++i) {
              x[i][j] -= to;
              x[i][j + 2] -= to;
            }
            sum[j] = mul2(sum[j], make_float2(f[j], f[j]));
#pragma unroll
            for (int g = 0; g < GN; ++g) mids[g][j] = mul2(mids[g][j], make_float2(f[j], f[j]));
          }
          // the largest weights times steps, down to a power of two
          __nv_bfloat162 bars[GN];
#pragma unroll
          for (int g = 0; g < GN; ++g) bars[g] = __floats2bfloat162_rn(0.f, 0.f);
#pragma unroll
          for (int i = 0; i < kSets; ++i)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const float a = exp2_of(x[i][2 * k]), b = exp2_of(x[i][2 * k + 1]);
#pragma unroll
              for (int g = 0; g < GN; ++g) {  // (what is not seen weighs 0, and 0 times an infinity is not the larger)
                const float step = low_half(vscale[i][g][k]);
                const uint32_t of = __byte_perm(__float_as_uint(a * step), __float_as_uint(b * step), 0x7632);
                bars[g] = __hmax2(bars[g], *reinterpret_cast<const __nv_bfloat162*>(&of));
              }
            }
#pragma unroll
          for (int g = 0; g < GN; ++g) {
#pragma unroll
            for (int o = 4; o < 32; o *= 2) bars[g] = __hmax2(bars[g], __shfl_xor_sync(~0u, bars[g], o));
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const float bar = j ? __high2float(bars[g]) : __low2float(bars[g]);
              // `want` brings 2^e <= bar < 2^(e + 1) to 2^5; an infinity leaves nothing finite in any case
              const int e2 = max((int)(__float_as_uint(bar) >> 23) - 127, -24);
              const float was = up[g][j], want = e2 == 128 ? was : __uint_as_float((uint32_t)(5 - e2 + 127) << 23);
              up[g][j] = bar * was >= kMost ? want : fmaxf(was, fminf(was * less[j], want));
              const float by = f[j] * up[g][j] * __uint_as_float(0x7F000000u - __float_as_uint(was));  // powers of two
#pragma unroll
              for (int i = 2 * g * GS; i < Z::kSumTiles && i < 2 * (g + 1) * GS; ++i) {
                acc[i][j] *= by;
                acc[i][j + 2] *= by;
              }
            }
          }
        }
        // weights, and the operands of the values
        uint32_t bw[kTiles][GN][2];
        float all[GN][4];  // of each column, in every row: the step's weights as they are rounded
#pragma unroll
        for (int i = 0; i < kSets; ++i) {
          float2 wt[2];  // of a column, positions g8 and g8 + 8
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            wt[j] = make_float2(exp2_of(x[i][j]), exp2_of(x[i][j + 2]));
            sum[j] = add2(sum[j], wt[j]);
          }
#pragma unroll
          for (int g = 0; g < GN; ++g) {
            const float2 step = make_float2(low_half(vscale[i][g][0]), low_half(vscale[i][g][1]));
            const float2 mid = fma2(make_float2(8.f, 8.f), step, make_float2(high_half(vscale[i][g][0]), high_half(vscale[i][g][1])));
            {
              float2 b[2];
#pragma unroll
              for (int j = 0; j < 2; ++j) {
                b[j] = mul2(wt[j], mul2(step, make_float2(up[g][j], up[g][j])));
                if constexpr (EDGE) {  // whatever stands where a row does not see: 0
                  b[j].x = seen[i][j] ? b[j].x : 0.f;
                  b[j].y = seen[i][j + 2] ? b[j].y : 0.f;
                  const float2 of = make_float2(seen[i][j] ? mid.x : 0.f, seen[i][j + 2] ? mid.y : 0.f);
                  mids[g][j] = fma2(wt[j], of, mids[g][j]);
                } else {
                  mids[g][j] = fma2(wt[j], mid, mids[g][j]);
                }
              }
              const uint32_t b0 = turned(pack2<KD_F16>(b[0].x, b[1].x)), b1 = turned(pack2<KD_F16>(b[0].y, b[1].y));
              constexpr uint32_t one = 0x3C003C00u;
              if (i == 0) mma_first(all[g], one, one, one, one, b0, b1);
              else mma(all[g], one, one, one, one, b0, b1);
              if constexpr (PACK) {  // each tile's operand has its own columns only
                bw[0][g][0] = g8 < 4 ? b0 : 0u;
                bw[0][g][1] = g8 < 4 ? b1 : 0u;
                bw[1][g][0] = g8 < 4 ? 0u : b0;
                bw[1][g][1] = g8 < 4 ? 0u : b1;
              } else {
                bw[i][g][0] = b0;
                bw[i][g][1] = b1;
              }
            }
          }
        }
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int k = 0; k < 2; ++k)
            {
              float(&d)[4] = acc[2 * c + k];
              const float2 eight = make_float2(all[c / GS][0], all[c / GS][1]);
              const float2 even = fma2(eight, make_float2(-8.f * 0x1p-24f, -8.f * 0x1p-24f), make_float2(d[0], d[1]));
              const float2 both = fma2(eight, make_float2(-136.f * 0x1p-24f, -136.f * 0x1p-24f), make_float2(d[2], d[3]));
              d[0] = even.x;
              d[1] = even.y;
              d[2] = both.x;
              d[3] = both.y;
        }
#pragma unroll
        for (int i = 0; i < kTiles; ++i) {
          uint32_t w[4];  // positions 2 t4, 2 t4 + 1, and the same 8 on, of one piece; of the next
#pragma unroll
          for (int c = 0; c < NC; ++c) {
            if (c % 2 == 0) {
              if (c + 1 < NC) load_matrices<true>(w, codes + Z::kCodes * 4 + i * kTile * S * 4 + c * 16);
              else load_two_matrices<true>(w, codes + Z::kCodes * 4 + i * kTile * S * 4 + c * 16);
            }
            uint32_t a = w[c % 2 * 2], b = w[c % 2 * 2 + 1];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              if (k) {  // the upper bytes down
                a = __byte_perm(a, 0, 0x4341);
                b = __byte_perm(b, 0, 0x4341);
              }
              mma(acc[2 * c + k], a & 0x000F000Fu, k ? a : a & 0x00FF00FFu, b & 0x000F000Fu, k ? b : b & 0x00FF00FFu,
                  bw[i][c / GS][0], bw[i][c / GS][1]);
            }
          }
        }
      };

      for (int b0 = 0; b0 < tiles; b0 += kBatch) {
        const int n = min(kBatch, tiles - b0);
        if (b0) {
          __syncthreads();  // no warp still reads the last batch's places
          bad_pages = __syncthreads_or(look_up(b0, n));
          prefetch(n);
        }
        // this warp's steps: tiles kTiles * warp on, kChunk apart
        int fetch = kTiles * warp + (ST - 1) * kChunk;
        int stage = 0, next = ST - 1;
        for (int nth = kTiles * warp; nth < n; nth += kChunk, fetch += kChunk) {
          issue(fetch, n, next);
          commit();
          wait_group<ST - 1>();
          __syncwarp();  // the lanes' copies are each other's
          const int position = (first_tile + b0 + nth) * kTile;
          // `position` may be the last of 31 bits: nothing is added to it
          if (bad_pages || position < w.all_lo || position > min(w.all_hi, share_hi) - kTiles * kTile)
            step(std::true_type{}, stage, position, place[nth].x < 0, nth + 1 < n && place[nth + 1].x < 0);
          else step(std::false_type{}, stage, position, false, false);
          __syncwarp();
          stage = stage + 1 == ST ? 0 : stage + 1;
          next = next + 1 == ST ? 0 : next + 1;
        }
        wait_group<0>();
      }

      // The warps' sums, in fp32 without the scaling, then joined.
      __syncthreads();
      float* sums = reinterpret_cast<float*>(smem);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int r = 2 * t4 + j;
        float total = sum[j].x + sum[j].y, of[GN];
#pragma unroll
        for (int g = 0; g < GN; ++g) of[g] = mids[g][j].x + mids[g][j].y;
#pragma unroll
        for (int o = 4; o < 32; o *= 2) {
          total += __shfl_xor_sync(~0u, total, o);
#pragma unroll
          for (int g = 0; g < GN; ++g) of[g] += __shfl_xor_sync(~0u, of[g], o);
        }
        if (g8 == 0) ml[warp * Z::kRows + r] = make_float2(room[j] == kNone ? kNone : m[j], total);
        float* to = sums + (warp * Z::kRows + r) * Z::kSums + 4 * g8;
#pragma unroll
        for (int c = 0; c < NC; ++c) {  // even channels, and these plus 16 times the odd ones
          const float back = 0x1p24f / up[c / GS][j];
          const float(&d0)[4] = acc[2 * c];
          const float(&d1)[4] = acc[2 * c + 1];
          *reinterpret_cast<float4*>(to + 32 * c) =
              make_float4(__fmaf_rn(d0[j], back, of[c / GS]), __fmaf_rn(d0[j + 2] - d0[j], back * 0.0625f, of[c / GS]),
                          __fmaf_rn(d1[j], back, of[c / GS]), __fmaf_rn(d1[j + 2] - d1[j], back * 0.0625f, of[c / GS]));
        }
      }
      __syncthreads();
      // the part's place for partial sums: the share's first item, or its last
      const int64_t slot = 2 * (int64_t)blockIdx.x + (left == share ? 0 : 1);
      for (int r = warp; r < w.rows; r += kWarps) {
        const int token = token_of(p, r0 + r), h = head * p.shared + (r0 + r) - token * p.shared;
        const int64_t t = w.first + token;
        if (t < 0 || t >= p.tokens) continue;
        // the parts of a row: each warp's, of one tile and the other where they have columns of their own
        constexpr int kParts = PACK ? 2 * kWarps : kWarps, kApart = PACK ? 4 : Z::kRows;
        float top = kNone, total = 0.f, f[kParts];
#pragma unroll
        for (int k = 0; k < kParts; ++k) top = fmaxf(top, ml[k * kApart + r].x);
#pragma unroll
        for (int k = 0; k < kParts; ++k) {
          const float2 v = ml[k * kApart + r];
          f[k] = v.x == kNone ? 0.f : exp2_of(v.x - top);
          total += v.x == kNone ? v.y : v.y * f[k];  // a part without a maximum has summed nothing, or NaN
        }
        if (past_table(p, w, token)) total = __int_as_float(0x7FC00000);
        for (int ch = 4 * lane; ch < p.part_row; ch += 128) {
          float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
          for (int k = 0; k < kParts; ++k) {
            const float4 v = *reinterpret_cast<const float4*>(sums + (k * kApart + r) * Z::kSums + ch);
            o.x = __fmaf_rn(v.x, f[k], o.x);
            o.y = __fmaf_rn(v.y, f[k], o.y);
            o.z = __fmaf_rn(v.z, f[k], o.z);
            o.w = __fmaf_rn(v.w, f[k], o.w);
          }
          if (!cut) put(p, p.out + t * p.out_token + h * p.out_head, ch, o, total);
          else if (TEAM) *reinterpret_cast<float4*>(sums + r * Z::kSums + ch) = o;
          else *reinterpret_cast<float4*>(p.part + (slot * Z::kRows + r) * p.part_row + ch) = o;
        }
        __syncwarp();  // all lanes have read the warps' sums
        if (lane == 0) {
          if (!cut) put_lse(p, t * p.heads + h, top, total);
          else if (TEAM) ml[r] = make_float2(top, total);
          else p.part_ml[slot * Z::kRows + r] = make_float2(top, total);
        }
      }
      if (!TEAM && chunk == 0 && threadIdx.x == 0)  // what is left of the item is the CTAs' that follow
        p.cuts[((int64_t)s * p.c.heads + head) * p.row_blocks + block] = Cut{(int)blockIdx.x, (int)slot, (w.chunks - n_chunks + share - 1) / share, 0};
      left -= n_chunks;
    }
    if constexpr (TEAM) {
      if (cut) join_team<Z>(p, w, head, block, n_chunks > 0, reinterpret_cast<float*>(smem), ml);
      return;
    }
    if (left <= 0) return;
    // the next item
    chunk = 0;
    if (w.rows == 0 || ++block == p.row_blocks) {
      block = 0;
      if (++head == p.c.heads) {
        head = 0;
        ++s;
      }
    }
    __syncthreads();  // the sums are read before the ring is written again
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

template <int NC, int GS, bool TEAM, bool PACK>
cudaError_t launch_one(const Params& p, int grid, cudaStream_t s) {
  static_assert(Shape<NC, GS>::kBytes <= 227 * 1024, "shared memory");
  auto kernel = attn4_kernel<NC, GS, TEAM, PACK>;
  static std::atomic<uint64_t> ready{0};
  const cudaError_t e = allow_shared_memory(kernel, ready);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3(32 * kWarps);
  cfg.dynamicSmemBytes = Shape<NC, GS>::kBytes;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  launch_early(attr[0]);
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)p.team;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = p.team > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, p);
}
// gs: 32-channel pieces of a group
template <int NC, bool TEAM, bool PACK>
cudaError_t launch(const Params& p, int gs, int grid, cudaStream_t s) {
  if constexpr (NC > 2)
    if (gs == 4) return launch_one<NC, 4, TEAM, PACK>(p, grid, s);
  if constexpr (NC > 1)
    if (gs >= 2) return launch_one<NC, 2, TEAM, PACK>(p, grid, s);
  return launch_one<NC, 1, TEAM, PACK>(p, grid, s);
}

// Of one translation unit each: with NC = 1 to 4 or 5 to 8, clusters or equal shares, blocks of eight rows or of
// four.  nc: 32-channel pieces of a row
using Launch = cudaError_t(const Params& p, int nc, int gs, int grid, cudaStream_t s);
Launch launch_team_128, launch_team_256, launch_shares_128, launch_shares_256;
Launch launch_team_128_pack, launch_team_256_pack, launch_shares_128_pack, launch_shares_256_pack;

}  // namespace attn4
}  // namespace kd
