// kd_attention_4bit: checks, how positions are split, and the launch that joins the shares (the
// kernels are kd_attn4.cuh's).
#include <algorithm>
#include <cmath>

#include "kd_attn4.cuh"

namespace kd {
namespace attn4 {
namespace {

constexpr int kJoinThreads = 256;

// A block for each CTA's cut item.  First the parts' weights, from their maxima, for all rows; then a thread has four
// channels of a row and adds the parts in order, its loads independent of each other.
__global__ void __launch_bounds__(kJoinThreads) attn4_join_kernel(const __grid_constant__ Params p, int of_block) {
  extern __shared__ float weights[];  // [part][row], then a row's maxima and sums
  depend_on_last();
  const Cut c = p.cuts[blockIdx.x];
  if (c.more == 0) return;
  const int parts = c.more + 1, lane = threadIdx.x & 31;
  float* totals = weights + (gridDim.x + 1) * of_block;
  // part k's rows: the item's first place, then the first ones of the CTAs that follow
  auto first_row = [&](int k) { return (int64_t)(k ? 2 * ((int)blockIdx.x + k) : c.slot) * of_block; };
  for (int r = threadIdx.x >> 5; r < c.rows; r += kJoinThreads / 32) {
    float top = kNone;
    for (int k = lane; k < parts; k += 32) top = fmaxf(top, p.part_ml[first_row(k) + r].x);
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
    float total = 0.f;
    for (int k = lane; k < parts; k += 32) {
      const float2 v = p.part_ml[first_row(k) + r];
      const float f = v.x == kNone ? 0.f : exp2_of(v.x - top);
      total += v.x == kNone ? v.y : v.y * f;
      weights[k * of_block + r] = f;
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) total += __shfl_xor_sync(~0u, total, o);
    if (lane == 0) {
      totals[r] = total;
      const int in = c.block * of_block + r, token = token_of(p, in);
      const int64_t t = c.first + token;
      if (p.lse && t >= 0 && t < p.tokens)
        p.lse[t * p.heads + c.head * p.shared + in - token * p.shared] =
            total == 0.f ? kNone : (top + log2f(total)) * 0.693147180559945f;
    }
  }
  __syncthreads();
  const int quads = (p.c.d + 3) / 4;
  for (int i = threadIdx.x; i < c.rows * quads; i += kJoinThreads) {
    const int r = i / quads, ch = 4 * (i - r * quads);
    const int in = c.block * of_block + r, token = in / p.shared, h = c.head * p.shared + in - token * p.shared;
    const int64_t t = c.first + token;
    if (t < 0 || t >= p.tokens) continue;
    float o[4] = {0.f, 0.f, 0.f, 0.f};
    const float* from = p.part + (int64_t)r * p.part_row + ch;
    const int64_t apart = (int64_t)of_block * p.part_row;  // of two places
    constexpr int kAhead = 8;
    for (int k0 = 0; k0 < parts; k0 += kAhead) {
      float4 v[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int n = min(k0 + k, parts - 1);
        v[k] = *reinterpret_cast<const float4*>(from + apart * (n ? 2 * ((int)blockIdx.x + n) : c.slot));
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const float f = k0 + k < parts ? weights[(k0 + k) * of_block + r] : 0.f;
        if (k0 + k >= parts) continue;
        o[0] = __fmaf_rn(v[k].x, f, o[0]);
        o[1] = __fmaf_rn(v[k].y, f, o[1]);
        o[2] = __fmaf_rn(v[k].z, f, o[2]);
        o[3] = __fmaf_rn(v[k].w, f, o[3]);
      }
    }
    const float total = totals[r], over = total == 0.f ? 0.f : 1.f / total;
    uint16_t* out = p.out + t * p.out_token + h * p.out_head + ch;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (ch + e < p.c.d) out[e] = narrow(p, total != total ? total : o[e] * over);
  }
}

struct Plan {
  int nc, gs, nt;  // of the kernel: 32-channel pieces, of a group; blocks of eight rows
  int row_blocks, whole;
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
  pl.nt = s->most * shared > 8 && pl.nc <= 4 ? 2 : 1;
  const int64_t blocks = (s->most * shared + 8 * pl.nt - 1) / (8 * pl.nt);
  const int64_t items = s->seqs * c->heads;
  // chunks of positions of all items together, were all as long as the table has room for
  auto chunks_of = [&](int64_t positions) { return std::max<int64_t>(1, (positions + kTile * kChunk - 1) / (kTile * kChunk) + 1); };
  const int64_t room = std::min(s->wide * c->page, (int64_t)INT32_MAX - kTile);
  if (blocks > INT32_MAX || items > INT32_MAX || (blocks && items > INT32_MAX / blocks) ||
      (blocks && items * blocks > INT32_MAX / chunks_of(room)))
    return false;
  pl.row_blocks = (int)blocks;
  int64_t longest = std::min(s->longest, room);
  if (window > 0) longest = std::min(longest, window + 8 * pl.nt + kTile);
  const int64_t all = items * blocks, places = 152 * (pl.nt == 1 && pl.nc <= 4 ? 4 : 2);
  pl.whole = longest <= 2 * kTile * kChunk;
  pl.grid = (int)(pl.whole ? all : std::min(places, all * chunks_of(longest)));
  pl.workspace = 0;
  if (!pl.whole) pl.workspace = (size_t)pl.grid * (sizeof(Cut) + 2 * (8 * pl.nt) * (8 + 4 * (size_t)((c->d + 3) / 4 * 4)));
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
  p.whole = pl.whole;
  p.part_row = (int)((cache->d + 3) / 4 * 4);
  p.causal = causal != 0;
  p.window = (int)window;
  p.room = (int)std::min(seqs->wide * cache->page, (int64_t)INT32_MAX - kTile);
  p.page_log = -1;
  for (int log = 0; log <= 12; ++log)
    if (cache->page == (int64_t)kTile << log) p.page_log = log;
  p.bf16 = dtype == KD_BF16;
  p.q_vec = cache->d % 8 == 0 && aligned(q, 16) && (tokens == 1 || q_token % 8 == 0) && (heads == 1 || q_head % 8 == 0);
  p.scale2 = scale * 1.4426950408889634f;
  if (!pl.whole) {
    p.cuts = static_cast<Cut*>(workspace);
    p.part_ml = reinterpret_cast<float2*>(p.cuts + pl.grid);
    p.part = reinterpret_cast<float*>(p.part_ml + (int64_t)pl.grid * 2 * (8 * pl.nt));
  }
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e = pl.nc <= 2   ? launch_small(p, pl.nc, pl.gs, pl.nt, pl.grid, s)
                  : pl.nc == 3 ? launch_96(p, pl.gs, pl.nt, pl.grid, s)
                  : pl.nc == 4 ? launch_128(p, pl.gs, pl.nt, pl.grid, s)
                  : pl.nc <= 6 ? launch_192(p, pl.nc, pl.gs, pl.grid, s)
                               : launch_256(p, pl.nc, pl.gs, pl.grid, s);
  if (e == cudaSuccess && !pl.whole) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)pl.grid);
    cfg.blockDim = dim3(kJoinThreads);
    cfg.dynamicSmemBytes = (size_t)(pl.grid + 2) * (8 * pl.nt) * sizeof(float);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    launch_early(attr[0]);
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, attn4_join_kernel, p, 8 * pl.nt);
  }
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? KD_OK : KD_ERR_CUDA;
}
