// kd_attention_4bit: checks, how positions are split, and the launch that joins the shares (the
// kernels are kd_attn4.cuh's).
#include <algorithm>
#include <cmath>

#include "kd_attn4.cuh"

namespace kd {
namespace attn4 {
namespace {

constexpr int kJoinWarps = 4;

// One warp a row: the shares' sums, weighted by their maxima, in the shares' order.
__global__ void __launch_bounds__(32 * kJoinWarps) attn4_join_kernel(const __grid_constant__ Params p, int of_block, int64_t rows) {
  depend_on_last();
  const int lane = threadIdx.x & 31;
  const int64_t n = (int64_t)blockIdx.x * kJoinWarps + (threadIdx.x >> 5);
  if (n >= rows) return;
  const int r = (int)(n % of_block);
  const int64_t item = n / of_block;
  const int block = (int)(item % p.row_blocks), head = (int)(item / p.row_blocks % p.c.heads);
  const int s = (int)(item / p.row_blocks / p.c.heads);
  const Work w = work_of(p, s, block, of_block);
  if (r >= w.rows || w.splits == 1) return;
  const int in = block * of_block + r, token = in / p.shared, h = head * p.shared + in - token * p.shared;
  const int64_t t = w.first + token;
  if (t < 0 || t >= p.tokens) return;
  const float2* ml = p.part_ml + (item * p.splits) * of_block + r;
  const float* part = p.part + ((item * p.splits) * of_block + r) * p.c.d;
  float top = kNone;
  for (int k = lane; k < w.splits; k += 32) top = fmaxf(top, ml[(int64_t)k * of_block].x);
#pragma unroll
  for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
  float total = 0.f, o[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll 4
  for (int k = 0; k < w.splits; ++k) {
    const float2 v = ml[(int64_t)k * of_block];
    const float f = v.x == kNone ? 0.f : exp2_of(v.x - top);
    total += v.x == kNone ? v.y : v.y * f;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (lane + 32 * i < p.c.d) o[i] = __fmaf_rn(part[(int64_t)k * of_block * p.c.d + lane + 32 * i], f, o[i]);
  }
  if (past_table(p, w, token)) total = __int_as_float(0x7FC00000);
  const bool none = total == 0.f;
  const float over = none ? 0.f : 1.f / total;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (lane + 32 * i < p.c.d)
      p.out[t * p.out_token + h * p.out_head + lane + 32 * i] = narrow(p, total != total ? total : o[i] * over);
  if (lane == 0 && p.lse) p.lse[t * p.heads + h] = none ? kNone : (top + log2f(total)) * 0.693147180559945f;
}

struct Plan {
  int nc, gs, nt;  // of the kernel: 32-channel pieces, of a group; blocks of eight rows
  int row_blocks, splits, per;
  int64_t blocks;    // of the launch
  size_t workspace;  // bytes
};

// How the work is cut.  Where there are fewer items (sequences, key heads, blocks of rows) than
// places for CTAs, each one's positions go to as many CTAs as make one full round; else to as many as
// make four rounds, over which unlike lengths even out.
bool plan(const kd_cache4* c, const kd_sequences* s, int64_t heads, int64_t window, Plan& pl) {
  const int64_t shared = heads / c->heads;
  if (s->most * shared > INT32_MAX) return false;
  const int chunks = (int)((c->d + 31) / 32);
  pl.nc = chunks <= 4 ? chunks : chunks <= 6 ? 6 : 8;
  pl.gs = (int)(c->group / 32);
  pl.nt = s->most * shared > 8 && pl.nc <= 4 ? 2 : 1;
  const int64_t blocks = (s->most * shared + 8 * pl.nt - 1) / (8 * pl.nt);
  const int64_t items = s->seqs * c->heads;
  if (blocks > INT32_MAX || items > INT32_MAX || (blocks && items > INT32_MAX / blocks)) return false;
  pl.row_blocks = (int)blocks;
  int64_t longest = std::min({s->longest, s->wide * c->page, (int64_t)INT32_MAX});
  if (window > 0) longest = std::min(longest, window + 8 * pl.nt + kTile);
  const int64_t tiles = std::max<int64_t>(1, (longest + kTile - 1) / kTile);
  const int64_t places = 152 * (pl.nt == 1 && pl.nc <= 4 ? 2 : 1), all = std::max<int64_t>(1, items * blocks);
  const bool few = all < places;
  const int64_t want = few ? places / all : (4 * places + all - 1) / all;
  const int64_t splits = std::max<int64_t>(1, std::min(want, tiles / (few ? 16 : 64)));
  pl.per = (int)((tiles + splits - 1) / splits);
  pl.splits = (int)((tiles + pl.per - 1) / pl.per);
  if (all > INT32_MAX / pl.splits) {
    pl.per = (int)tiles;
    pl.splits = 1;
  }
  pl.blocks = items * blocks * pl.splits;
  pl.workspace = pl.splits == 1 ? 0 : (size_t)pl.blocks * (8 * pl.nt) * (4 * (size_t)c->d + 8);
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
  p.splits = pl.splits;
  p.per = pl.per;
  p.causal = causal != 0;
  p.window = (int)window;
  p.bf16 = dtype == KD_BF16;
  p.q_vec = cache->d % 8 == 0 && aligned(q, 16) && (tokens == 1 || q_token % 8 == 0) && (heads == 1 || q_head % 8 == 0);
  p.scale2 = scale * 1.4426950408889634f;
  if (pl.splits > 1) {
    p.part_ml = static_cast<float2*>(workspace);  // pairs first: sums of odd d after them stay aligned
    p.part = reinterpret_cast<float*>(p.part_ml + pl.blocks * (8 * pl.nt));
  }
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e = pl.nc <= 2   ? launch_small(p, pl.nc, pl.gs, pl.nt, s)
                  : pl.nc == 3 ? launch_96(p, pl.gs, pl.nt, s)
                  : pl.nc == 4 ? launch_128(p, pl.gs, pl.nt, s)
                  : pl.nc == 6 ? launch_192(p, pl.gs, s)
                               : launch_256(p, pl.gs, s);
  if (e == cudaSuccess && pl.splits > 1) {
    const int of_block = 8 * pl.nt;
    const int64_t rows = pl.blocks / pl.splits * of_block;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((rows + kJoinWarps - 1) / kJoinWarps));
    cfg.blockDim = dim3(32 * kJoinWarps);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    launch_early(attr[0]);
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, attn4_join_kernel, p, of_block, rows);
  }
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? KD_OK : KD_ERR_CUDA;
}
