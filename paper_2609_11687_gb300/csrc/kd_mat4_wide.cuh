// Products of 17 to 64 activation rows with 4-bit weights and group scales
// (kd_matmul_4bit), on the fifth-generation tensor cores.
//
// From 17 rows on mma.sync is what bounds the product of kd_mat4.cuh; here tcgen05.mma takes
// the decoded codes c - z (exact in 16 bits, see kd_mat4.cuh) as its A operand, 128 channels
// by 64 inputs at a time, the rows as B, and sums in tensor memory.  A goes through tensor
// memory too: a channel is a lane of it, so the thread that decodes a channel stores its own
// lane (through shared memory, which is then written and read once per stage by A's 32 KB,
// 32000 x 4096 at 64 rows took 51 us instead of 48 when this was changed).
//
// A CTA owns 128 channels and its share of the inputs, in chunks of 128; two CTAs share an
// SM, so that one computes while the other waits (one CTA of 256 channels and twice the warps:
// 24 us instead of 14 at 32 rows of 4096 x 11008).  Its eight warps all do the same: a thread has one
// channel (the warp's place among the lanes of tensor memory gives it) and one half of what
// belongs to that channel.  Per chunk it turns 64 codes into 32 columns of its lane of A and
// lays out its share of B; per group of inputs it reads its half of the group's sums from
// tensor memory, scales and adds them in fp32 registers, while the next group's form in the
// other of two accumulators.  One thread issues the products.  Codes and rows come through a
// ring (cp.async); the two warps of 32 channels copy their codes together, four lanes a
// channel: a lane for each channel's 64 bytes is 32 lines a load, and the lines a load touches
// are what it costs.
//
// Stages of A and B, and the accumulators, pass between threads and tensor cores by
// mbarriers.  B is K-major with 128-byte swizzle: 16-byte piece c of row r lies at
// c ^ (r % 8), chunks in two halves of 64 inputs.
//
// K order: a piece of eight inputs holds them as the codes of a word come out, (0 4 1 5 2 6
// 3 7), in A and B alike.
//
// No unit is saturated: 49 % of the issue slots are used (346 instructions a warp and chunk), the
// integer pipe is 32 % busy, the tensor pipe 18 %, DRAM 19 %; a warp waits longest for memory (the
// copies) and for shared and tensor memory, one step of a chunk after the other, and of 152 SMs 98 have two
// CTAs and the others one: 43.3 us for 64 rows of 32000 x 4096 in fp16 with groups of 128, floor
// 11.3.  Smaller groups drain the accumulators more often: 55 us at 64, 67 at 32.  Rows that are
// not aligned are read by elements, again by each CTA: 175 us for 64 rows of 32000 x 4095, 92 for
// 32, where the kernel for few rows takes 33 for each 16.
//
// Every wait is bounded (about a second); one that expires marks the CTA, whose waits then
// all return at once and whose outputs become NaN.  Before it gives back its memory such a CTA
// waits once more, bounded again, for the products that it has in flight.
#pragma once
#include "kd_bulk.cuh"
#include "kd_mat4.cuh"

namespace kd {
namespace mat4 {

constexpr int kWideChannels = 128;
constexpr int kWideThreads = 256;
constexpr int kWideWarps = kWideThreads / 32;
constexpr int kWideStages = 2;  // of A and B
template <int N>
constexpr int kWideRing = N == 64 ? 3 : 5;  // chunks of codes and rows as they come
template <int N>
constexpr int kWideUnits = N * 16 / kWideThreads;  // 16-byte pieces of B a thread lays out
template <int N>
constexpr int kWideStageBytes = N * 256;  // of B
template <int N>
constexpr int kWideRingBytes = (2 + kWideUnits<N>) * kWideThreads * 16;  // of a chunk
// The barriers (and what aligns B), B's stages, the ring; in the end the CTA's sums in their place.
template <int N>
constexpr size_t kWideSmem = 1024 + 1024 + kWideStages * kWideStageBytes<N> + kWideRing<N> * kWideRingBytes<N>;
static_assert(kWideSmem<64> <= 113 * 1024 && kWideSmem<32> <= 113 * 1024 &&
                  kWideSmem<32> >= 2048 + 32 * kWideChannels * 4 && kWideSmem<64> >= 2048 + 64 * kWideChannels * 4,
              "shared memory of two CTAs an SM");
// Columns of tensor memory: two accumulators of N columns, A's stages of 64.  Half of all 512.
constexpr int kTensorColumns = 256;
template <int N>
constexpr int kColumnsOfA = 2 * N;
static_assert(kColumnsOfA<64> + kWideStages * 64 <= kTensorColumns, "tensor memory");

struct WideBarriers {
  uint64_t full[kWideStages], empty[kWideStages];  // a stage of A and B is laid out; its products are done
  uint64_t sums[2], taken[2];  // an accumulator holds a group's sums; they have been read
  uint64_t drained;            // after an expired wait: no product is in flight
  uint32_t tmem;
  int failed;
};

__device__ __forceinline__ void barrier_arrive(uint64_t* b) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(b)) : "memory");
}
static __device__ __noinline__ void barrier_wait_long(uint64_t* b, uint32_t parity, volatile int* failed) {
  const long long start = clock64();
  while (!mbar_try_wait(b, parity)) {
    if (*failed) return;
    if (clock64() - start > kWaitCycles) *failed = 1;
  }
}
__device__ __forceinline__ void barrier_wait(uint64_t* b, uint32_t parity, int* failed) {
  if (!mbar_try_wait(b, parity)) barrier_wait_long(b, parity, failed);
}

// a 128-byte swizzled K-major operand: rows of 128 bytes, eight of them 1024 bytes apart
__device__ __forceinline__ uint64_t operand_descriptor(uint32_t address) {
  return (uint64_t)(address >> 4 & 0x3FFF) | (uint64_t)1 << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 |
         (uint64_t)2 << 61;
}
// One lane of a converged warp.  The products' operands want uniform registers: behind this
// instruction the compiler knows a single thread to run, behind a comparison of the lane's
// number it does not, and a product takes 57 cycles to issue (80 with a predicate in place of
// the branch) instead of the 31 that N = 64 takes to run.
__device__ __forceinline__ bool elect() {
  uint32_t one;
  asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(one));
  return one;
}
// D (+)= A B with A and D in tensor memory
__device__ __forceinline__ void tensor_mma(uint32_t d, uint32_t a, uint64_t b, uint32_t what, bool add) {
  asm volatile(
      "{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(d),
      "r"(a), "l"(b), "r"(what), "r"((uint32_t)add)
      : "memory");
}
// the arrival on a barrier once all products so far are done
__device__ __forceinline__ void tensor_commit(uint64_t* b) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(b))
               : "memory");
}
// 16 or 32 columns of this warp's 32 lanes
__device__ __forceinline__ void tensor_load(uint32_t address, float (&v)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, "
      "[%16];"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]),
        "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
      : "r"(address));
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tensor_load(uint32_t address, float (&v)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]),
        "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]),
        "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]),
        "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
      : "r"(address));
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

// 32 columns of this warp's 32 lanes, and until they are there
__device__ __forceinline__ void tensor_store(uint32_t address, const uint32_t (&v)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(address),
      "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
      "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]),
      "r"(v[19]), "r"(v[20]), "r"(v[21]), "r"(v[22]), "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]),
      "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31])
      : "memory");
}
__device__ __forceinline__ void tensor_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ void copy8(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(src) : "memory");
}

// BF: bf16 rows; GS: groups of 32 GS inputs; N: rows of a pass at most (32, 64); ZEROS: zero
// points by group.  Grid: one cluster of `split` CTAs for each 128 channels.
template <bool BF, int GS, int N, bool ZEROS>
__global__ void __launch_bounds__(kWideThreads, 2) mat4_wide_kernel(const __grid_constant__ Params p) {
  namespace cg = cooperative_groups;
  extern __shared__ uint4 smem_raw[];
  const uint32_t pad = -smem_u32(smem_raw) & 1023u;  // operands start on 1024 bytes
  uint8_t* smem = reinterpret_cast<uint8_t*>(smem_raw) + pad;
  WideBarriers& sh = *reinterpret_cast<WideBarriers*>(smem);
  uint8_t* stage_b = smem + 1024;
  uint4* ring = reinterpret_cast<uint4*>(stage_b + kWideStages * kWideStageBytes<N>) + threadIdx.x;
  // by shuffle: so the compiler knows a warp's role to be the same for all its lanes
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(~0u, tid >> 5, 0);
  const int rank = special<kRank>(), tile = special<kCluster>();
  const int c0 = rank * p.per, mine = max(0, min(p.per, p.chunks - c0));
  constexpr int kGroups = 4 / GS, kUnits = kWideUnits<N>, kHalf = N / 2, kRing = kWideRing<N>;

  if (tid == 32) {
    for (int s = 0; s < 2; ++s) {
      mbar_init(&sh.full[s], kWideWarps);
      mbar_init(&sh.empty[s], 1);
      mbar_init(&sh.sums[s], 1);
      mbar_init(&sh.taken[s], kWideWarps);
    }
    mbar_init(&sh.drained, 1);
    sh.failed = 0;
    mbar_init_fence();
  }
  wait_for_last();
  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem)),
                 "r"(kTensorColumns)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  let_next_start();

  // this thread's lane of tensor memory, channel, and half: inputs 64 part .. + 63 of a
  // chunk, rows kHalf part .. of the sums
  const int part = warp >> 2, of_tile = (warp & 3) * 32 + lane;
  const uint32_t tensor = __shfl_sync(~0u, sh.tmem, 0), lanes = tensor + ((uint32_t)(warp & 3) << 21);
  const int ch = min(tile * kWideChannels + of_tile, p.m - 1);

  // Codes: pieces idx % 4 of channel idx / 4 of the 32 that this warp shares with the one
  // four further, idx = 32 part + lane (+ 64); piece c of channel r lies at c ^ (r / 2 % 4).
  // Rows: 8 inputs of row u / 16, u = tid + 256 i, for this thread alone.  In place of
  // rows past the batch its first ones come again: a column of B meets one column of the sums.
  // (The last one in all these places is the same few lines for all CTAs: 32000 x 4096 took 40 us
  // at 17 rows, 65 at 33, instead of 34 and 43.  Copying no rows there cost more at full tiles,
  // 47 us instead of 43 at 64 rows, than it saved at others.)
  const int idx = 32 * part + lane, base = tile * kWideChannels + (warp & 3) * 32;
  uint4* pair_ring = reinterpret_cast<uint4*>(stage_b + kWideStages * kWideStageBytes<N>) + (warp & 3) * 128;
  const uint4* codes[2];
  int code_at[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = (idx + 64 * i) >> 2, c = idx & 3;
    codes[i] = reinterpret_cast<const uint4*>(p.codes + (int64_t)min(base + r, p.m - 1) * p.pieces * 16);
    code_at[i] = r * 4 + (c ^ (r >> 1 & 3));
  }
  const uint8_t* x[kUnits];
#pragma unroll
  for (int i = 0; i < kUnits; ++i)
    x[i] = p.x + ((int64_t)(((tid + kWideThreads * i) >> 4) % p.rows) * p.ldx + c0 * kChunk + 8 * (tid & 15)) *
                     (p.e4m3 ? 1 : 2);
  const int whole = p.x_vec ? (p.n - c0 * kChunk) / kChunk : 0;  // chunks without a row's end
  int to_slot = 0;
  auto fetch = [&](int l) {
    if (l < mine) {
      const int slot_at = to_slot * (kWideRingBytes<N> / 16);
      to_slot = to_slot + 1 == kRing ? 0 : to_slot + 1;
      const int piece = min(4 * (c0 + l) + (idx & 3), p.pieces - 1);
#pragma unroll
      for (int i = 0; i < 2; ++i) copy16(smem_u32(pair_ring + slot_at + code_at[i]), codes[i] + piece);
      if (l < whole) {
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
          const uint32_t slot = smem_u32(ring + slot_at + (2 + i) * kWideThreads);
          if (p.e4m3) copy8(slot, x[i] + l * kChunk);
          else copy16(slot, x[i] + l * (2 * kChunk));
        }
      } else {
        const int have = p.n - (c0 + l) * kChunk - 8 * (tid & 15);  // inputs from this piece on
#pragma unroll 1
        for (int i = 0; i < kUnits; ++i)
          ring[slot_at + (2 + i) * kWideThreads] =
              have > 0 ? load_inputs_one_by_one(x[i], p.e4m3, l * kChunk, have) : make_uint4(0, 0, 0, 0);
      }
    }
    commit();
  };
  for (int l = 0; l < kRing - 1; ++l) fetch(l);

  // scales, and zero points of this thread's inputs, of a chunk's groups
  uint32_t scale[kGroups], zero[GS == 1 ? 2 : 1];
  const uint16_t* scales = p.scales + (int64_t)c0 * kGroups * p.m + ch;
  auto fetch_scales = [&](int l) {
#pragma unroll
    for (int k = 0; k < kGroups; ++k)
      scale[k] = scales[(int64_t)(GS == 4 ? l : min(l * kGroups + k, p.groups - 1 - c0 * kGroups)) * p.m];
    if constexpr (ZEROS) {
#pragma unroll
      for (int k = 0; k < (GS == 1 ? 2 : 1); ++k)
        zero[k] = p.zeros[(int64_t)min((4 * (c0 + l) + 2 * part + k) / GS, p.groups - 1) * p.m + ch];
    }
  };
  if (mine) fetch_scales(0);

  // warp 0: the products of group k, of chunk l
  auto issue = [&](int l, int k) {
    // fp32 sums of fp16 or bf16 products, M = 128, N, B K-major
    constexpr uint32_t kWhat = 1u << 4 | (BF ? 1u : 0u) << 7 | (BF ? 1u : 0u) << 10 | (N / 8) << 17 | (128 / 16) << 24;
    const int group = l * kGroups + k, stage = l & 1;
    if (group >= 2) barrier_wait(&sh.taken[group & 1], (group >> 1) - 1 & 1, &sh.failed);
    if (k == 0) barrier_wait(&sh.full[stage], l >> 1 & 1, &sh.failed);
    __syncwarp();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t to = tensor + (group & 1) * N, a = tensor + kColumnsOfA<N> + stage * 64 + k * (16 * GS);
    const uint64_t b = operand_descriptor(smem_u32(stage_b) + stage * kWideStageBytes<N>);
    if (elect()) {
#pragma unroll
      for (int i = 0; i < 2 * GS; ++i) {  // 16 inputs each: 32 bytes further along the rows
        const int q = 2 * GS * k + i;
        const uint64_t bq = b + (q >> 2) * (N * 128 / 16) + 2 * (q & 3);
        tensor_mma(to, a + 8 * i, bq, kWhat, i > 0);
      }
      if (k == kGroups - 1) tensor_commit(&sh.empty[stage]);
      tensor_commit(&sh.sums[group & 1]);
    }
    __syncwarp();
  };
  float acc[kHalf];
#pragma unroll
  for (int j = 0; j < kHalf; ++j) acc[j] = 0.f;
  // this thread's sums of a group, scaled and added
  auto take = [&](int group, uint32_t raw) {
    const float s = p.scale_bf16 ? __uint_as_float(raw << 16) : __half2float(__ushort_as_half((unsigned short)raw));
    barrier_wait(&sh.sums[group & 1], group >> 1 & 1, &sh.failed);
    __syncwarp();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    float v[kHalf];
    tensor_load(lanes + (group & 1) * N + part * kHalf, v);
#pragma unroll
    for (int j = 0; j < kHalf; ++j) acc[j] = __fmaf_rn(s, v[j], acc[j]);
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncwarp();
    if (lane == 0) barrier_arrive(&sh.taken[group & 1]);
  };

  const Magic<BF> magic;
  uint32_t last = 0;  // the scale of the group before
  int from_slot = 0;
  for (int l = 0; l < mine; ++l) {
    const int stage = l & 1;
    uint32_t now[kGroups];
#pragma unroll
    for (int k = 0; k < kGroups; ++k) now[k] = scale[k];
    wait_group<kRing - 2>();
    // both warps' copies are there, and both have read the chunk before, whose place is next
    asm volatile("barrier.sync %0, 64;" ::"r"(1 + (warp & 3)) : "memory");
    fetch(l + kRing - 1);
    const int slot_at = from_slot * (kWideRingBytes<N> / 16);
    from_slot = from_slot + 1 == kRing ? 0 : from_slot + 1;
    const uint4* raw = ring + slot_at;
    uint4 word[2];
#pragma unroll
    for (int c = 0; c < 2; ++c) word[c] = pair_ring[slot_at + lane * 4 + ((2 * part + c) ^ (lane >> 1 & 3))];
    uint32_t a[32];
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      const uint4 v = word[c / 4];
      const uint32_t w = c % 4 == 0 ? v.x : c % 4 == 1 ? v.y : c % 4 == 2 ? v.z : v.w;
      const uint2 z = zero_words<BF>(ZEROS ? zero[GS == 1 ? c / 4 : 0] : 8u);
      const uint2 lo = code_pairs<BF>(w, 0, magic, z), hi = code_pairs<BF>(w, 1, magic, z);
      a[4 * c] = lo.x; a[4 * c + 1] = lo.y; a[4 * c + 2] = hi.x; a[4 * c + 3] = hi.y;
    }
    if (l + 1 < mine) fetch_scales(l + 1);
    if (l >= kWideStages) barrier_wait(&sh.empty[stage], (l >> 1) - 1 & 1, &sh.failed);
    __syncwarp();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    tensor_store(lanes + kColumnsOfA<N> + stage * 64 + part * 32, a);
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      const int u = tid + kWideThreads * i, r = u >> 4, c = u & 15;
      const uint4 v = raw[(2 + i) * kWideThreads], h = p.e4m3 ? bytes_to_half(v) : v;
      *reinterpret_cast<uint4*>(stage_b + stage * kWideStageBytes<N> + (c >> 3) * (N * 128) + r * 128 +
                                (((c ^ r) & 7) << 4)) =
          make_uint4(__byte_perm(h.x, h.z, 0x5410), __byte_perm(h.x, h.z, 0x7632), __byte_perm(h.y, h.w, 0x5410),
                     __byte_perm(h.y, h.w, 0x7632));
    }
    fence_proxy_async_smem();
    tensor_store_wait();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncwarp();
    if (lane == 0) barrier_arrive(&sh.full[stage]);
#pragma unroll
    for (int k = 0; k < kGroups; ++k) {
      if (warp == 0) issue(l, k);
      if (l * kGroups + k > 0) take(l * kGroups + k - 1, k ? now[k - 1] : last);
    }
    last = now[kGroups - 1];
  }
  if (mine) {
    take(mine * kGroups - 1, last);
    // nothing of this CTA is in flight when it ends
    barrier_wait(&sh.empty[(mine - 1) & 1], (mine - 1) >> 1 & 1, &sh.failed);
  }
  wait_group<0>();
  __syncthreads();  // every wait is over: `failed` is final, and stages and ring are free
  const bool failed = *static_cast<volatile int*>(&sh.failed);
  if (failed) {
    // The stages' barriers are out of step with the products by now; this one is new.  Every
    // product has been issued, by the lane that commits here.
    if (warp == 0 && elect()) tensor_commit(&sh.drained);
    mbar_wait_bounded(&sh.drained, 0);
  }

  auto finish = [&](int r, int c, float v) {
    const int j = tile * kWideChannels + c;
    if (j >= p.m) return;
    if (p.xs) v *= p.xs[r];
    store1_any(p.y, p.ydtype, (int64_t)r * p.ldy + j, v);
  };
  if (failed) {
#pragma unroll
    for (int j = 0; j < kHalf; ++j) acc[j] = __int_as_float(0x7FC00000);
  }
  if (p.split == 1) {
#pragma unroll
    for (int j = 0; j < kHalf; ++j)
      if (part * kHalf + j < p.rows) finish(part * kHalf + j, of_tile, acc[j]);
  } else {
    cg::cluster_group cl = cg::this_cluster();
    float* sums = reinterpret_cast<float*>(stage_b);
#pragma unroll
    for (int j = 0; j < kHalf; ++j)
      if (part * kHalf + j < p.rows) sums[(part * kHalf + j) * kWideChannels + of_tile] = acc[j];
    cl.sync();
    for (int o = rank * kWideThreads + tid; o < p.rows * kWideChannels; o += p.split * kWideThreads) {
      float v = 0.f;
      for (int k = 0; k < p.split; ++k) v += cl.map_shared_rank(sums, k)[o];
      finish(o / kWideChannels, o % kWideChannels, v);
    }
    cl.sync();  // no CTA leaves while its sums are read
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  if (warp == 0)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(sh.tmem), "r"(kTensorColumns));
}

template <bool BF, int GS, int N, bool ZEROS>
cudaError_t launch_wide_one(const Params& p, cudaStream_t s) {
  auto kernel = mat4_wide_kernel<BF, GS, N, ZEROS>;
  static std::atomic<uint64_t> ready{0};
  const cudaError_t e = allow_shared_memory(kernel, ready);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(p.tiles * p.split));
  cfg.blockDim = dim3(kWideThreads);
  cfg.dynamicSmemBytes = kWideSmem<N>;
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
cudaError_t launch_wide(const Params& p, cudaStream_t s) {
  if (p.rows <= 32) return p.zeros ? launch_wide_one<BF, GS, 32, true>(p, s) : launch_wide_one<BF, GS, 32, false>(p, s);
  return p.zeros ? launch_wide_one<BF, GS, 64, true>(p, s) : launch_wide_one<BF, GS, 64, false>(p, s);
}

}  // namespace mat4
}  // namespace kd
