// kd_attention_4bit: checks, how positions are split, and the launch that joins the shares (the
// kernels are kd_attn4.cuh's).
#include <algorithm>
#include <cmath>

#include "kd_attn4.cuh"

namespace kd {
namespace attn4 {
namespace {

constexpr int kJoinThreads = 256;

// A block for each CTA's cut item, eight rows and 128 channels at a time: a warp takes every eighth part with a
// running maximum of each row, all its loads independent of each other; then the warps' sums are joined in
// their order.
__global__ void __launch_bounds__(kJoinThreads) attn4_join_kernel(const __grid_constant__ Params p) {
  constexpr int kJoinWarps = kJoinThreads / 32;
  __shared__ float4 sums[kJoinWarps][kRows][32];
  __shared__ float2 ml[kJoinWarps][kRows];
  depend_on_last();
  const Cut c = p.cuts[blockIdx.x];
  if (c.more == 0) return;
  const int parts = c.more + 1, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int c0 = 0; c0 < p.part_row; c0 += 128) {
      const bool has = c0 + 4 * lane < p.part_row;
      float4 o[kRows];
      float2 at[kRows];
#pragma unroll
      for (int r = 0; r < kRows; ++r) {
        o[r] = make_float4(0.f, 0.f, 0.f, 0.f);
        at[r] = make_float2(kNone, 0.f);
      }
      for (int k = warp; k < parts; k += kJoinWarps) {
        // the part's rows: in the item's first place, or the first one of a CTA that follows
        const int64_t row = (int64_t)(k ? 2 * ((int)blockIdx.x + k) : c.slot) * kRows;
        float4 v[kRows];
        float2 n[kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r)
          if (r < c.rows) {
            n[r] = p.part_ml[row + r];
            v[r] = has ? *reinterpret_cast<const float4*>(p.part + (row + r) * p.part_row + c0 + 4 * lane) : make_float4(0.f, 0.f, 0.f, 0.f);
          }
#pragma unroll
        for (int r = 0; r < kRows; ++r)
          if (r < c.rows) {
            const float top = fmaxf(at[r].x, n[r].x);
            const float f = at[r].x == kNone ? 0.f : exp2_of(at[r].x - top), g = n[r].x == kNone ? 0.f : exp2_of(n[r].x - top);
            at[r].y = __fmaf_rn(at[r].y, at[r].x == kNone ? 1.f : f, n[r].y * (n[r].x == kNone ? 1.f : g));  // without a maximum: 0, or NaN
            at[r].x = top;
            o[r].x = __fmaf_rn(v[r].x, g, o[r].x * f);
            o[r].y = __fmaf_rn(v[r].y, g, o[r].y * f);
            o[r].z = __fmaf_rn(v[r].z, g, o[r].z * f);
            o[r].w = __fmaf_rn(v[r].w, g, o[r].w * f);
          }
      }
#pragma unroll
      for (int r = 0; r < kRows; ++r) {
        sums[warp][r][lane] = o[r];
        if (lane == 0) ml[warp][r] = at[r];
      }
      __syncthreads();
      const int r = warp;  // a row of a warp
      const int in = c.block * kRows + r, token = token_of(p, in), h = c.head * p.shared + in - token * p.shared;
      const int64_t t = c.first + token;
      if (r < c.rows && t >= 0 && t < p.tokens) {
        float top = kNone, total = 0.f;
        float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int k = 0; k < kJoinWarps; ++k) top = fmaxf(top, ml[k][r].x);
#pragma unroll
        for (int k = 0; k < kJoinWarps; ++k) {
          const float2 n = ml[k][r];
          const float f = n.x == kNone ? 0.f : exp2_of(n.x - top);
          total += n.y * (n.x == kNone ? 1.f : f);
          const float4 v = sums[k][r][lane];
          y.x = __fmaf_rn(v.x, f, y.x);
          y.y = __fmaf_rn(v.y, f, y.y);
          y.z = __fmaf_rn(v.z, f, y.z);
          y.w = __fmaf_rn(v.w, f, y.w);
        }
        if (has) put(p, p.out + t * p.out_token + h * p.out_head, c0 + 4 * lane, y, total);
        if (lane == 0 && c0 == 0) put_lse(p, t * p.heads + h, top, total);
      }
      __syncthreads();
    }
}

struct Plan {
  int nc, gs;  // of the kernel: 32-channel pieces, of a group
  int row_blocks, team;
  int grid;          // CTAs
  size_t workspace;  // bytes
};

// How the work is cut: into items (sequence, key head, block of rows) where those are short, else into equal
// shares of all of it, however long each sequence is, as many as CTAs fit the GPU at a time.
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
  int64_t longest = std::min(s->longest, room);
  if (window > 0) longest = std::min(longest, window + kRows + kTile);
  const int64_t all = items * blocks, places = 152 * (pl.nc <= 4 ? 4 : 2);
  const double chunks_each = (double)((longest + kTile * kChunk - 1) / (kTile * kChunk));
  // us: a CTA's step by how many share an SM, and a tile of equal shares
  pl.team = 0;
  double least = 13 + (all < 64 ? 4 : 0) + 0.8 * 0.0036 * all * chunks_each;
  for (int team = 1; team <= 8 && team <= chunks_each; team *= 2) {
    const double rounds = std::ceil((double)all * team / places), on_sm = std::min((double)all * team, (double)places) / 152;
    const double cost = 4.5 + (team > 1 ? 1.2 : 0) + rounds * std::ceil(chunks_each / team) * std::max(0.86, 0.5 + 0.38 * on_sm);
    if (cost < least) {
      least = cost;
      pl.team = team;
    }
  }
  pl.grid = (int)(pl.team ? all * pl.team : std::min(places, all * chunks_of(longest)));
  pl.workspace = 0;
  if (!pl.team) pl.workspace = (size_t)pl.grid * (sizeof(Cut) + 2 * kRows * (8 + 4 * (size_t)((c->d + 3) / 4 * 4)));
  pl.workspace = (pl.workspace + 15) / 16 * 16;
  return true;
}

kd_status check(const kd_cache4* cache, const kd_sequences* seqs, int64_t heads, int causal, int64_t window) {
  if (!cache_sizes_ok(cache) || !sequences_sizes_ok(seqs) || heads < 1 || heads > INT32_MAX || heads % cache->heads != 0 ||
      window < 0 || window > INT32_MAX || (window > 0 && !causal))
    return KD_ERR_INVALID_ARG;
  return cache->d < 1 || cache->d > kMaxD ? KD_ERR_UNSUPPORTED_N : KD_OK;
}

// rows of `heads` x `tokens` vectors of d elements do not overlap
bool rows_apart(int64_t tokens, int64_t heads, int64_t d, int64_t token, int64_t head) {
  if (tokens > 1 && heads > 1)
    return (head >= d && token >= d && (token - d) / head >= heads - 1) ||
           (token >= d && head >= d && (head - d) / token >= tokens - 1);
  return (tokens <= 1 || token >= d) && (heads <= 1 || head >= d);
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
  if (tokens < 0 || tokens > INT32_MAX || (dtype != KD_F16 && dtype != KD_BF16) || !std::isfinite(scale) || q_token < 0 ||
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
  p.scale2 = scale * 1.4426950408889634f;
  if (!pl.team) {
    p.cuts = static_cast<Cut*>(workspace);
    p.part_ml = reinterpret_cast<float2*>(p.cuts + pl.grid);
    p.part = reinterpret_cast<float*>(p.part_ml + (int64_t)pl.grid * 2 * kRows);
  }
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  auto launch = pl.team ? (pl.nc <= 4 ? launch_team_128 : launch_team_256) : (pl.nc <= 4 ? launch_shares_128 : launch_shares_256);
  cudaError_t e = launch(p, pl.nc, pl.gs, pl.grid, s);
  if (e == cudaSuccess && !pl.team) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)pl.grid);
    cfg.blockDim = dim3(kJoinThreads);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    launch_early(attr[0]);
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, attn4_join_kernel, p);
  }
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? KD_OK : KD_ERR_CUDA;
}
