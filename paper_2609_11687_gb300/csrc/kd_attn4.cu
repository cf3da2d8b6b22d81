// kd_attention_4bit: checks, how positions are split, and the launch that joins the shares (the
// kernels are kd_attn4.cuh's).
#include <algorithm>
#include <cmath>

#include "kd_attn4.cuh"

namespace kd {
namespace attn4 {
namespace {

// A block for an item and 32 of its channels: eight lanes have a part, so that a warp has four and the block up to 32 of
// them in flight; four rows at a time, each with a running maximum, joined over lanes and warps in a fixed order.
constexpr int kJoinWarps = 8, kJoinRows = 4;  // warps at most
constexpr float kLog2e = 1.4426950408889634f;

struct Sum {  // of one row: maximum, weights, four channels
  float m, l;
  float4 o;
  __device__ __forceinline__ void add(const Sum& b) {
    const float top = fmaxf(m, b.m);
    // without a maximum a part has summed nothing, or NaN, which its weights' sum says
    const float f = m == kNone ? 0.f : exp2_of(m - top), g = b.m == kNone ? 0.f : exp2_of(b.m - top);
    l = l * (m == kNone ? 1.f : f) + b.l * (b.m == kNone ? 1.f : g);
    m = top;
    o.x = __fmaf_rn(b.o.x, g, o.x * f);
    o.y = __fmaf_rn(b.o.y, g, o.y * f);
    o.z = __fmaf_rn(b.o.z, g, o.z * f);
    o.w = __fmaf_rn(b.o.w, g, o.w * f);
  }
};

__global__ void __launch_bounds__(32 * kJoinWarps) attn4_join_kernel(const __grid_constant__ Params p) {
  __shared__ Sum sums[kJoinWarps][kJoinRows][8];
  depend_on_last();
  const int64_t item = blockIdx.x;
  const int block = (int)(item % p.row_blocks), head = (int)(item / p.row_blocks % p.c.heads);
  const int s = (int)(item / p.row_blocks / p.c.heads);
  const Work w = work_of(p, s, block, kRows);
  const Cut c = p.cuts[item];
  if (w.chunks == 0 || c.more == 0) return;  // an item without rows has nothing in `cuts`
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  const int nth = lane >> 3, ch = 32 * blockIdx.y + 4 * (lane & 7);
  const bool has = ch < p.part_row;
  for (int r0 = 0; r0 < w.rows; r0 += kJoinRows) {
    Sum sum[kJoinRows];
#pragma unroll
    for (int r = 0; r < kJoinRows; ++r) sum[r] = Sum{kNone, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
    for (int k = 4 * warp + nth; k <= c.more; k += 4 * warps) {
      const int64_t row = (int64_t)(k ? 2 * (c.owner + k) : c.slot) * kRows + r0;
      Sum part[kJoinRows];
#pragma unroll
      for (int r = 0; r < kJoinRows; ++r) {
        part[r] = Sum{kNone, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
        if (r0 + r < w.rows) {
          const float2 ml = p.part_ml[row + r];
          part[r].m = ml.x;
          part[r].l = ml.y;
          if (has) part[r].o = *reinterpret_cast<const float4*>(p.part + (row + r) * p.part_row + ch);
        }
      }
#pragma unroll
      for (int r = 0; r < kJoinRows; ++r) sum[r].add(part[r]);
    }
#pragma unroll
    for (int r = 0; r < kJoinRows; ++r) {
#pragma unroll
      for (int o = 8; o < 32; o *= 2) {
        Sum other;
        other.m = __shfl_xor_sync(~0u, sum[r].m, o);
        other.l = __shfl_xor_sync(~0u, sum[r].l, o);
        other.o.x = __shfl_xor_sync(~0u, sum[r].o.x, o);
        other.o.y = __shfl_xor_sync(~0u, sum[r].o.y, o);
        other.o.z = __shfl_xor_sync(~0u, sum[r].o.z, o);
        other.o.w = __shfl_xor_sync(~0u, sum[r].o.w, o);
        sum[r].add(other);
      }
      if (lane < 8) sums[warp][r][lane] = sum[r];
    }
    __syncthreads();
    const int r = threadIdx.x >> 3, in = block * kRows + r0 + r, token = token_of(p, in), h = head * p.shared + in - token * p.shared;
    const int64_t t = w.first + token;
    if (r < kJoinRows && r0 + r < w.rows && t >= 0 && t < p.tokens) {
      Sum all = sums[0][r][lane & 7];
      for (int k = 1; k < warps; ++k) all.add(sums[k][r][lane & 7]);
      if (has) put(p, p.out + t * p.out_token + h * p.out_head, ch, all.o, all.l);
      if (ch == 0) put_lse(p, t * p.heads + h, all.m, all.l);
    }
    __syncthreads();
  }
}

struct Plan {
  int nc, gs;  // of the kernel: 32-channel pieces, of a group
  int row_blocks, team;
  int grid;          // CTAs
  int64_t items;
  size_t workspace;  // bytes
};

// How the work is cut: a cluster for each item (sequence, key head, block of rows), or equal shares of all of it.
// Clusters need no search and no second launch, but are done when the longest is; equal shares take all SMs
// whatever the lengths.  The rule estimates both in microseconds from the longest length that the host knows:
//   clusters: 4, 1.2 for their join, 2.5 ns a CTA, and their steps of 128 positions at 0.69, or 0.24 + 0.45 for each
//   CTA that an SM has (0.63 of that for 64 channels; above 128 channels 0.98, or 0.95 for each, and clusters of eight
//   put two on some SMs early); times the rounds of CTAs where they do not all fit;
//   equal shares: 11, and 3.2 ns for each such step of all items (HBM's rate; 2 for 64 channels, 5.8 for 256), 3.0 of
//   several sequences, which are seldom all as long as the longest.
// Measured for heads of 128 channels, groups of 64, four rows, clusters of 1 / 2 / 4 / 8 and equal shares:
//     8 items of  1024 positions   9.8 / 8.9 / 7.3 / 6.6,     8.6
//     8 items of  8192             50 / 29 / 17.4 / 11.7,     12.2
//    32 items of  4096             27 / 17.5 / 12.0 / 10.6,   15.8
//    32 items of 16384             101 / 54 / 30 / 23.6,      25.1
//   256 items of  1024             14.0 / 16.0 / 21 / 32,     20
//   256 items of  4096             39 / 37 / 41 / 50,         38
//   256 items of  2000 to 8192     66 / 59 / 55 / 60,         53
//   512 items of  8192             120 / 112 / 117 / 135,     112;  of 2000 to 8192  107 / 91 / 93 / 110,  84
// Several blocks of rows of a key head read the same codes, as CTAs side by side from L2 (steps at 1.7 at most) but in equal
// shares one after the other: 14, and 3.7 ns a step.  Where sequences have rows of their own number, a part of the blocks
// is empty and lengths differ too: 0.7 of the items and 0.65 of their steps are counted.  Four blocks of eight rows, groups
// of 128:
//   512 items of  1000 to 4096, 1 to 8 tokens    56 / 38 / 44 / 59,        45
//   256 items of  the same                       43 / 33 / 23 / 30,        31
//  2048 items of  the same                       99 / 108 / 139 / 201,     115
//  1024 items of  4096, 8 tokens                 103 / 114 / 134 / 179,    113;  of 16384  380 / 380 / 391 / 428,  388
// From eight blocks on (parts of prompts) there are clusters only: each CTA of equal shares would walk the blocks to find its
// own, and join what each of its many short items is cut into.  Clusters of 1 / 2 / 4 and equal shares:
//  1024 items of  1000, 16 sequences of 32 tokens     72 / 100 / 148,     88;   of up to 1000 and 32    32 / 44 / 69,      51
//  2048 items of  4096, 32 sequences of 16            221 / 240 / 287,    233;  of up to 4096 and 16    114 / 124 / 156,   123
// 16000 items of  1000, 4 prompts of as many tokens   349 / 582 / 932,    849;  of up to as many        151 / 256 / 428,   519
//  4000 items, one prompt of 1000 tokens              97 / 151 / 236,     386
constexpr int64_t kBlocksInShares = 7;
bool plan(const kd_cache4* c, const kd_sequences* s, int64_t heads, int64_t window, Plan& pl) {
  const int64_t shared = heads / c->heads;
  if (s->most * shared > INT32_MAX) return false;
  const int chunks = (int)((c->d + 31) / 32);
  pl.nc = chunks;
  pl.gs = (int)(c->group / 32);
  const int64_t blocks = (s->most * shared + kRows - 1) / kRows;
  const int64_t items = s->seqs * c->heads;
  // chunks of positions of all items together, were all as long as the table has room for
  auto chunks_of = [&](int64_t positions) { return std::max<int64_t>(1, (positions + kTile * kChunk - 1) / (kTile * kChunk) + 1); };
  const int64_t room = std::min(s->wide * c->page, (int64_t)INT32_MAX - kTile);
  if (blocks > INT32_MAX || items > INT32_MAX || (blocks && items > INT32_MAX / blocks) ||
      (blocks && items * blocks > INT32_MAX / chunks_of(room)))
    return false;
  pl.row_blocks = (int)blocks;
  pl.items = items * blocks;
  int64_t longest = std::min(s->longest, room);
  if (window > 0) longest = std::min(longest, window + kRows + kTile);
  const int64_t all = items * blocks, places = 152 * on_sm(pl.nc, true);
  const double chunks_each = (double)((longest + kTile * kChunk - 1) / (kTile * kChunk));
  pl.team = 0;
  const bool several = blocks > 1, uneven = several && s->seqs > 1 && s->starts;
  const double live = (uneven ? 0.7 : 1) * (double)all, mean = uneven ? 0.65 : 1, wide = pl.nc <= 4 ? 0.25 + 0.1875 * pl.nc : 0.2 + 0.2 * pl.nc;
  double least = blocks > kBlocksInShares ? HUGE_VAL : several ? 14 + 0.0037 * wide * live * mean * chunks_each : 11 + (s->seqs > 1 ? 0.003 : 0.0032) * wide * live * chunks_each;
  for (int team = 1; team <= kTeam && (team <= chunks_each || (team == 1 && blocks > kBlocksInShares)); team *= 2) {
    const double ctas = live * team, fit = std::min(ctas, (double)places), of_sm = fit / 152;
    double step = pl.nc <= 4 ? wide * std::max(0.69, 0.24 + 0.45 * of_sm) : std::max(0.98, 0.95 * std::min(2.0, team == kTeam ? 2 * of_sm : of_sm));
    if (several) step = std::min(step, 1.7 * wide);
    const double start = 4 + (team > 1 ? 1.2 : 0) + 0.0025 * fit, steps = std::ceil(chunks_each / team) * step;
    const double cost = std::max(start + steps, ctas / fit * (start + mean * steps));
    if (cost < least) {
      least = cost;
      pl.team = team;
    }
  }
  pl.grid = (int)(pl.team ? all * pl.team : std::min<int64_t>(152 * on_sm(pl.nc, false), all * chunks_of(longest)));
  pl.workspace = 0;
  if (!pl.team) pl.workspace = (size_t)all * sizeof(Cut) + (size_t)pl.grid * 2 * kRows * (8 + 4 * (size_t)((c->d + 3) / 4 * 4));
  pl.workspace = (pl.workspace + 15) / 16 * 16;
  return true;
}

kd_status check(const kd_cache4* cache, const kd_sequences* seqs, int64_t heads, int causal, int64_t window) {
  if (!cache_sizes_ok(cache) || !sequences_sizes_ok(seqs) || heads < 1 || heads > INT32_MAX || heads % cache->heads != 0 ||
      window < 0 || window > INT32_MAX || (window > 0 && !causal))
    return KD_ERR_INVALID_ARG;
  return cache->d < 1 || cache->d > kMaxD ? KD_ERR_UNSUPPORTED_N : KD_OK;
}

}  // namespace
}  // namespace attn4
}  // namespace kd

extern "C" size_t kd_attention_4bit_workspace(const kd_cache4* cache, const kd_sequences* seqs, int64_t heads, int64_t window) {
  using namespace kd::attn4;
  Plan pl;
  if (check(cache, seqs, heads, 1, window) != KD_OK || seqs->seqs == 0 || !plan(cache, seqs, heads, window, pl)) return 0;
  return pl.workspace;
}

extern "C" kd_status kd_attention_4bit(const kd_cache4* cache, const kd_sequences* seqs, int64_t tokens, int64_t heads,
                                       const void* q, int64_t q_token, int64_t q_head, kd_dtype dtype, void* out,
                                       int64_t out_token, int64_t out_head, float* lse, float scale, int causal,
                                       int64_t window, void* workspace, size_t ws_bytes, void* stream) {
  using namespace kd;
  using namespace kd::attn4;
  const kd_status st = check(cache, seqs, heads, causal, window);
  if (st != KD_OK) return st;
  if (tokens < 0 || tokens > INT32_MAX || (dtype != KD_F16 && dtype != KD_BF16) || !std::isfinite(scale * kLog2e) || q_token < 0 ||
      q_head < 0 || out_token < 0 || out_head < 0)
    return KD_ERR_INVALID_ARG;
  Plan pl;
  if (!plan(cache, seqs, heads, window, pl)) return KD_ERR_INVALID_ARG;
  if (tokens == 0 || seqs->seqs == 0 || seqs->most == 0) return KD_OK;
  if (!cache_pointers_ok(cache) || !sequences_pointers_ok(seqs) || !q || !out || !aligned(q, 2) || !aligned(out, 2) ||
      !aligned(lse, 4) || !rows_apart(tokens, heads, cache->d, out_token, out_head))
    return KD_ERR_INVALID_ARG;
  if (pl.workspace && (!workspace || !aligned(workspace, 16) || ws_bytes < pl.workspace)) return KD_ERR_WORKSPACE;
  Params p{};
  p.c = pages_of(cache, seqs);
  p.q = static_cast<const uint16_t*>(q);
  p.out = static_cast<uint16_t*>(out);
  p.lse = lse;
  p.q_token = q_token;
  p.q_head = q_head;
  p.out_token = out_token;
  p.out_head = out_head;
  p.tokens = tokens;
  p.heads = (int)heads;
  p.shared = (int)(heads / cache->heads);
  p.row_blocks = pl.row_blocks;
  p.team = pl.team;
  p.part_row = (int)((cache->d + 3) / 4 * 4);
  p.causal = causal != 0;
  p.window = (int)window;
  p.room = (int)std::min(seqs->wide * cache->page, (int64_t)INT32_MAX - kTile);
  p.bf16 = dtype == KD_BF16;
  p.q_vec = cache->d % 8 == 0 && aligned(q, 16) && (tokens == 1 || q_token % 8 == 0) && (heads == 1 || q_head % 8 == 0);
  p.out_vec = cache->d % 4 == 0 && aligned(out, 8) && (tokens == 1 || out_token % 4 == 0) && (heads == 1 || out_head % 4 == 0);
  p.scale2 = scale * kLog2e;
  if (!pl.team) {
    p.cuts = static_cast<Cut*>(workspace);
    p.part_ml = reinterpret_cast<float2*>(p.cuts + pl.items);
    p.part = reinterpret_cast<float*>(p.part_ml + (int64_t)pl.grid * 2 * kRows);
  }
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  static constexpr Launch* kLaunch[2][2][2] = {{{launch_shares_128, launch_shares_128_pack}, {launch_shares_256, launch_shares_256_pack}},
                                               {{launch_team_128, launch_team_128_pack}, {launch_team_256, launch_team_256_pack}}};
  Launch* launch = kLaunch[pl.team > 0][pl.nc > 4][seqs->most * p.shared <= 4];
  cudaError_t e = launch(p, pl.nc, pl.gs, pl.grid, s);
  if (e == cudaSuccess && !pl.team) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)pl.items, (unsigned)((cache->d + 31) / 32));
    const int64_t warps = (pl.grid / pl.items + 2 + 3) / 4;  // four parts of an item each
    cfg.blockDim = dim3(32 * (unsigned)std::min<int64_t>(warps, kJoinWarps));
    cfg.stream = s;
    // not early: its blocks would wait on the SMs whose shares end first, and be joined there (15 us more)
    e = cudaLaunchKernelEx(&cfg, attn4_join_kernel, p);
  }
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? KD_OK : KD_ERR_CUDA;
}
