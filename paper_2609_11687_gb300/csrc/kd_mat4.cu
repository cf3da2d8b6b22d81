// kd_matmul_4bit: argument checks and the choice of the launch (kernels: kd_mat4.cuh).
#include "kd_mat4.cuh"

namespace kd {
namespace mat4 {
namespace {

constexpr int64_t kMaxN = 65536;
// channels are counted in 32 bits up to the end of the last tile, of 512 at most
constexpr int64_t kMaxM = INT32_MAX - kTile * kWarps + 1;
constexpr size_t kSmem = 227 * 1024;

// CTAs of one launch that run at a time, one an SM: clusters of `split` on 152 SMs, less what
// the GPU's partitions leave over.
int room(int split) { return split == 1 ? 152 : split == 2 ? 76 : split == 4 ? 36 : 15; }

// How the work is split: CTAs of a cluster (split) and warps (kw) that share a tile's
// inputs, for `rows` rows in nt tiles of eight.  The cost counts chunks of one warp, one
// after the other: a tile's chunks, half a chunk to join its sums, across a cluster another
// one and a part for each output, and once the time to lay out the CTA's rows.  Fitted to all
// splits of 24 products (64 to 32000 channels of 700 to 16384 inputs, 1 to 16 rows): the
// choice is the fastest within 2 %, but for one of rows that are not aligned (11 %).  Without the rows' part 4096 x
// 4096 at 16 rows took 8.3 us instead of 7.2, 64 x 8192 6.2 instead of 4.5.
// False if the rows fit no CTA's shared memory (eight rows always do).
bool plan(Params& p, int nt, int rows) {
  bool found = false;
  double least = 0;
  for (int split = 1; split <= 8; split *= 2) {
    const int per = (p.chunks + split - 1) / split;
    if (split > 1 && per < 2) break;
    for (int kw = kWarps; kw >= 1; kw /= 2) {
      if (smem_bytes(nt, rows, per, split, kw) > kSmem) continue;
      const int channels = kTile * kWarps / kw;
      const int tiles = (p.m + channels - 1) / channels;
      const int at_once = room(split);
      const double rounds = (tiles + at_once - 1) / at_once;
      const double join = split > 1 ? 1.5 + channels * rows / 16384. : 0.5;
      const double cost = rounds * ((per + kw - 1) / kw + join) + 0.005 * per * rows;
      if (!found || cost < least) {
        found = true;
        least = cost;
        p.split = split;
        p.kw = kw;
        p.kw_log = kw == 16 ? 4 : kw == 8 ? 3 : kw == 4 ? 2 : kw - 1;
        p.per = per;
        p.tiles = tiles;
      }
    }
  }
  return found;
}

// The same for the kernel for many rows, whose CTAs do not stay: 128 channels each, two an SM,
// a cost of a chunk, three for a CTA's start and end and two more for a cluster's.  Against all
// splits of 51 products (128 to 65536 channels of 512 to 16384 inputs, at 32 and 64 rows): the
// choice is the fastest within 1 % from 4096 inputs on, but for 11008 x 11008 (45 us at 32 rows in four
// CTAs and 41 in eight, 47 in the two chosen).  Of shorter inputs the joins cost less and a cluster
// more than counted: up to 23 % for a few channels of 512 (8 CTAs 5.3 us, 4 chosen 6.5), 35 %
// for 11008 or 14336 channels of 1024 (alone 10.5 us, 2 chosen 14).
void plan_wide(Params& p) {
  double least = 0;
  p.tiles = (p.m + 127) / 128;
  p.kw = 1;
  for (int split = 1; split <= 8; split *= 2) {
    const int per = (p.chunks + split - 1) / split, at_once = split == 1 ? 304 : split == 2 ? 152 : split == 4 ? 74 : 36;
    const double rounds = (p.tiles + at_once - 1) / at_once;
    const double cost = rounds * (per + (split > 1 ? 5 : 3));
    if (split == 1 || cost < least) {
      least = cost;
      p.split = split;
      p.per = per;
    }
  }
}

}  // namespace
}  // namespace mat4
}  // namespace kd

extern "C" kd_status kd_matmul_4bit(const kd_weight4* w, const void* x, kd_dtype x_dtype, const float* x_scale,
                                    int64_t rows, int64_t ldx, void* y, kd_dtype y_dtype, int64_t ldy,
                                    void* stream) {
  using namespace kd;
  using namespace kd::mat4;
  if (!weight4_sizes_ok(w) || w->m > kMaxM || rows < 0 || (x_dtype != KD_F16 && x_dtype != KD_BF16 && x_dtype != KD_E4M3) ||
      !float_type(y_dtype) || ldx < w->n || ldy < w->m)
    return KD_ERR_INVALID_ARG;
  if (w->n > kMaxN) return KD_ERR_UNSUPPORTED_N;
  if (w->m == 0 || rows == 0) return KD_OK;
  const int64_t xb = type_bytes(x_dtype), yb = type_bytes(y_dtype);
  if (!x || !y || !weight4_pointers_ok(w) || !aligned(x, (size_t)xb) || !aligned(y, (size_t)yb) ||
      !aligned(x_scale, 4))
    return KD_ERR_INVALID_ARG;
  Params p{};
  p.codes = reinterpret_cast<const uint8_t*>(w->codes);
  p.scales = static_cast<const uint16_t*>(w->scales);
  p.zeros = w->zeros;
  p.ldx = ldx;
  p.ldy = ldy;
  p.n = (int)w->n;
  p.m = (int)w->m;
  p.groups = (int)((w->n + w->group - 1) / w->group);
  p.pieces = (int)((w->n + 31) / 32);
  p.chunks = (int)((w->n + kChunk - 1) / kChunk);
  p.scale_vec = w->m % 4 == 0 && aligned(w->scales, 8) && aligned(w->zeros, 4);
  p.scale_bf16 = w->scale_dtype == KD_BF16;
  p.ydtype = (int)y_dtype;
  p.e4m3 = x_dtype == KD_E4M3;
  const bool bf = x_dtype == KD_BF16;
  const int gs = w->group / 32;
  const size_t wide = p.e4m3 ? 8 : 16;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  // Passes of equal numbers of rows: from 17 rows on of at most 64, by the kernel for many
  // rows; else one by the kernel for few.  At 16 rows that one takes 7.2 / 12.8 / 24 us for
  // 4096 x 4096, 4096 x 11008 and 32000 x 4096, the kernel for many rows 7.6 / 13.9 / 34 there and no
  // more at 17 to 32, where two passes of the other take about twice its time.
  // Where 9 to 16 rows of long inputs fit no CTA's shared memory (16 of 32768), the kernel for
  // many rows takes them too, 35 us for 4096 channels of 32768 and 65 of 65536, where two passes
  // of eight take 42 and 99; it has one cluster for 128 channels, and few of those leave SMs idle: 512
  // channels take it 27 and 51 us, the two passes 16 and 25 (2500 channels 34 and 65, 37 and 62).  Each of
  // its clusters reads the rows again, by elements where they are not aligned: 4096 channels of 39999
  // then take it 121 us, the two passes 82.
  constexpr int kManyChannels = 2560;
  int nt = rows > 8 ? 2 : 1, clusters = 0;
  int64_t pass = rows;
  // up to eight rows split the work alike, so that a row's sums have one order whatever
  // else is in the batch
  bool few = rows <= 16 && plan(p, nt, nt == 1 ? 8 : (int)rows);
  if (!few && rows <= 16 && (p.m < kManyChannels || !aligned(x, wide) || ldx * xb % (int64_t)wide != 0)) {
    nt = 1;
    pass = 8;
    few = plan(p, nt, 8);
  }
  if (few) {
    p.turns_of_row_inv = 1.f / (float)((p.per * 16 + 31) / 32);
    clusters = p.tiles < room(p.split) ? p.tiles : room(p.split);
  } else {
    const int64_t passes = (rows + 63) / 64;
    nt = 0;
    pass = (rows + passes - 1) / passes;
    plan_wide(p);
  }
  for (int64_t r0 = 0; r0 < rows; r0 += pass) {
    p.rows = (int)(rows - r0 < pass ? rows - r0 : pass);
    p.x = static_cast<const uint8_t*>(x) + r0 * ldx * xb;
    p.xs = x_scale ? x_scale + r0 : nullptr;
    p.y = static_cast<uint8_t*>(y) + r0 * ldy * yb;
    p.x_vec = aligned(p.x, wide) && (p.rows == 1 || ldx * xb % (int64_t)wide == 0);
    const cudaError_t e = gs == 1   ? launch_group32(p, bf, nt, clusters, s)
                          : gs == 2 ? launch_group64(p, bf, nt, clusters, s)
                                    : launch_group128(p, bf, nt, clusters, s);
    if (e != cudaSuccess || cudaGetLastError() != cudaSuccess) return KD_ERR_CUDA;
  }
  return KD_OK;
}
