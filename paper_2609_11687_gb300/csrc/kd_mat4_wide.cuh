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
// Roles in a CTA, which owns 256 channels (two A tiles for each B tile, which halves the
// traffic of the rows) and its share of the inputs:
//   warps 0-7   a thread a channel: after each group of inputs its sums are read from tensor
//               memory, scaled and added in fp32 registers, while the next group's form in
//               the other of two accumulators; one thread of warp 0 issues the products;
//   warps 8-15  a thread a channel: 64 codes a stage become 32 columns of its lane of A, two
//               inputs each; the same threads lay out B in shared memory.  Codes and rows come
//               through a ring that each thread fills and reads for itself (cp.async).
// Stages of A and B, and the accumulators, pass between them by mbarriers.  B is K-major
// with 128-byte swizzle: 16-byte piece c of row r lies at c ^ (r % 8).
//
// K order: a piece of eight inputs holds them as the codes of a word come out, (0 4 1 5 2 6
// 3 7), in A and B alike.
//
// Every wait is bounded (about a second); one that expires marks the CTA, whose waits then
// all return at once and whose outputs become NaN.
#pragma once
#include "kd_bulk.cuh"
#include "kd_mat4.cuh"

namespace kd {
namespace mat4 {

constexpr int kWideChannels = 256;
constexpr int kWideThreads = 512;
constexpr int kWideStages = 4;  // of A and B
constexpr int kWideRing = 7;    // of codes and rows as they come
constexpr int kStageInputs = 64;
template <int N>
constexpr int kWideStageBytes = N * 128;  // of B
// B's stages, or in the end the CTA's sums; the barriers; the ring of raw codes and rows;
// room to align
template <int N>
constexpr size_t kWideSums = (size_t)N * kWideChannels * 4;
template <int N>
constexpr size_t kWideSmem = kWideSums<N> + 256 + (size_t)kWideRing * (2 + N / 32) * 256 * 16 + 1024;
// Columns of tensor memory, all 512 taken (one CTA an SM): two accumulators of two times 128
// channels, N columns each; A's stages, 32 columns for each 128 channels.
constexpr int kTensorColumns = 512;
template <int N>
constexpr int kColumnsOfA = 4 * N;
static_assert(kColumnsOfA<64> + kWideStages * 64 <= kTensorColumns, "tensor memory");

struct WideBarriers {
  uint64_t full[kWideStages], empty[kWideStages];
  uint64_t sums[2], taken[2];  // an accumulator holds a group's sums; they have been read
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
// 32 columns of this warp's 32 lanes
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
// points by group.  Grid: one cluster of `split` CTAs for each 256 channels.
template <bool BF, int GS, int N, bool ZEROS>
__global__ void __launch_bounds__(kWideThreads, 1) mat4_wide_kernel(const __grid_constant__ Params p) {
  namespace cg = cooperative_groups;
  extern __shared__ uint4 smem_raw[];
  const uint32_t pad = -smem_u32(smem_raw) & 1023u;  // operands start on 1024 bytes
  uint8_t* smem = reinterpret_cast<uint8_t*>(smem_raw) + pad;
  WideBarriers& sh = *reinterpret_cast<WideBarriers*>(smem + kWideSums<N>);
  // by shuffle: so the compiler knows a warp's role to be the same for all its lanes
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(~0u, tid >> 5, 0);
  const int rank = special<kRank>(), tile = special<kCluster>();
  const int c0 = rank * p.per, mine = max(0, min(p.per, p.chunks - c0));
  const int stages = 2 * mine, groups = mine * (4 / GS);

  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem)),
                 "r"(kTensorColumns)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (tid == 32) {
    for (int s = 0; s < kWideStages; ++s) {
      mbar_init(&sh.full[s], 8);
      mbar_init(&sh.empty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&sh.sums[b], 1);
      mbar_init(&sh.taken[b], 8);
    }
    sh.failed = 0;
    mbar_init_fence();
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  constexpr uint32_t tmem = 0;  // all of it
  depend_on_last();

  const float nan = __int_as_float(0x7FC00000);
  float* sums = reinterpret_cast<float*>(smem);  // of the CTA, in the end
  auto finish = [&](int r, int c, float v) {
    const int ch = tile * kWideChannels + c;
    if (ch >= p.m) return;
    if (p.xs) v *= p.xs[r];
    store1_any(p.y, p.ydtype, (int64_t)r * p.ldy + ch, v);
  };
  if (warp < 8) {
    // scale and add: thread tid is channel tid of the tile
    const int ch = min(tile * kWideChannels + tid, p.m - 1);
    const uint32_t from = tmem + ((uint32_t)(warp & 3) << 21) + (warp >> 2) * N;
    auto fetch = [&](int k) { return p.scales[(int64_t)min(c0 * (4 / GS) + k, p.groups - 1) * p.m + ch]; };
    // warp 0: the products of group k
    auto issue = [&](int k) {
      // fp32 sums of fp16 or bf16 products, M = 128, N, B K-major
      constexpr uint32_t kWhat = 1u << 4 | (BF ? 1u : 0u) << 7 | (BF ? 1u : 0u) << 10 | (N / 8) << 17 | (128 / 16) << 24;
      if (k >= 2) {
        barrier_wait(&sh.taken[k & 1], (k >> 1) - 1 & 1, &sh.failed);
        __syncwarp();
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      }
      const uint32_t to = tmem + (k & 1) * 2 * N;
#pragma unroll
      for (int i = 0; i < 2 * GS; ++i) {  // 16 inputs each: 32 bytes further along the rows
        const int s = (2 * GS * k + i) / 4, slot = s % kWideStages, q = (GS == 1 ? 2 * (k & 1) : 0) + i % 4;
        if (q == 0) {
          barrier_wait(&sh.full[slot], s / kWideStages & 1, &sh.failed);
          __syncwarp();
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        }
        const uint32_t a = tmem + kColumnsOfA<N> + slot * 64 + 8 * q;
        const uint64_t b = operand_descriptor(smem_u32(smem) + slot * kWideStageBytes<N>) + 2 * q;
        if (elect()) {
          tensor_mma(to, a, b, kWhat, i > 0);
          tensor_mma(to + N, a + 32, b, kWhat, i > 0);
          if (q == 3) tensor_commit(&sh.empty[slot]);
          if (i == 2 * GS - 1) tensor_commit(&sh.sums[k & 1]);
        }
        __syncwarp();
      }
    };
    float acc[N];
#pragma unroll
    for (int j = 0; j < N; ++j) acc[j] = 0.f;
    uint16_t next = groups ? fetch(0) : 0;
    if (warp == 0 && groups) issue(0);
    for (int k = 0; k < groups; ++k) {
      const uint16_t raw = next;
      if (k + 1 < groups) next = fetch(k + 1);
      if (warp == 0 && k + 1 < groups) issue(k + 1);
      __syncwarp();
      const float s = p.scale_bf16 ? __uint_as_float((uint32_t)raw << 16) : __half2float(__ushort_as_half(raw));
      barrier_wait(&sh.sums[k & 1], k >> 1 & 1, &sh.failed);
      __syncwarp();
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
      for (int h = 0; h < N / 32; ++h) {
        float v[32];
        tensor_load(from + (k & 1) * 2 * N + 32 * h, v);
#pragma unroll
        for (int j = 0; j < 32; ++j) acc[32 * h + j] = __fmaf_rn(s, v[j], acc[32 * h + j]);
      }
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0) barrier_arrive(&sh.taken[k & 1]);
    }
    // the last sums are here, so no product runs any more and the stages' memory is free;
    // nothing of this CTA is in flight when it ends
    if (stages) barrier_wait(&sh.empty[(stages - 1) % kWideStages], (stages - 1) / kWideStages & 1, &sh.failed);
    const bool failed = *static_cast<volatile int*>(&sh.failed);
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (j < p.rows) {
        const float v = failed ? nan : acc[j];
        if (p.split == 1) finish(j, tid, v);
        else sums[j * kWideChannels + tid] = v;
      }
  } else {
    // decode: thread d is channel d of the tile; and lay out the rows
    const int d = tid - 256, ch = min(tile * kWideChannels + d, p.m - 1);
    const uint4* codes = reinterpret_cast<const uint4*>(p.codes + (int64_t)ch * p.pieces * 16);
    const uint32_t lanes = tmem + ((uint32_t)(warp & 3) << 21) + kColumnsOfA<N> + (d >> 7) * 32;
    const Magic<BF> magic;
    constexpr int kUnits = N * 8 / 256;  // 16-byte pieces of B a thread lays out
    // This thread's own places in the ring of raw stages: two pieces of codes, then its
    // pieces of the rows (8 inputs of row u / 8, u = d + 256 i).  Rows past the batch repeat
    // its last one: a column of B meets one column of the sums.
    uint4* ring = reinterpret_cast<uint4*>(smem + kWideSums<N> + 256) + d;
    const uint8_t* x[kUnits];
#pragma unroll
    for (int i = 0; i < kUnits; ++i)
      x[i] = p.x + ((int64_t)min((d + 256 * i) >> 3, p.rows - 1) * p.ldx + c0 * kChunk + 8 * (d & 7)) * (p.e4m3 ? 1 : 2);
    auto fetch = [&](int s) {
      if (s < stages) {
        uint4* to = ring + s % kWideRing * (2 + kUnits) * 256;
        const int piece = 4 * c0 + 2 * s;
        copy16(smem_u32(to), codes + min(piece, p.pieces - 1));
        copy16(smem_u32(to + 256), codes + min(piece + 1, p.pieces - 1));
        const int have = p.n - c0 * kChunk - s * kStageInputs - 8 * (d & 7);  // inputs from this piece on
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
          uint4* slot = to + (2 + i) * 256;
          if (p.x_vec && have >= 8) {
            if (p.e4m3) copy8(smem_u32(slot), x[i] + s * kStageInputs);
            else copy16(smem_u32(slot), x[i] + s * (2 * kStageInputs));
          } else {
            *slot = have > 0 ? load_inputs_one_by_one(x[i], p.e4m3, s * kStageInputs, have) : make_uint4(0, 0, 0, 0);
          }
        }
      }
      commit();
    };
    uint32_t zero = 0;
    for (int s = 0; s < kWideRing - 1; ++s) fetch(s);
    for (int s = 0; s < stages; ++s) {
      const int slot = s % kWideStages;
      if constexpr (ZEROS) {
        // the group of the stage's first and second 32 inputs
        const int g0 = (4 * c0 + 2 * s) / GS;
        zero = p.zeros[(int64_t)min(g0, p.groups - 1) * p.m + ch];
        if constexpr (GS == 1) zero |= (uint32_t)p.zeros[(int64_t)min(g0 + 1, p.groups - 1) * p.m + ch] << 8;
        else zero *= 0x101u;
      }
      fetch(s + kWideRing - 1);
      wait_group<kWideRing - 1>();  // this thread's own copies: nobody else reads them
      const uint4* raw = ring + s % kWideRing * (2 + kUnits) * 256;
      uint32_t a[32];
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const uint4 v = raw[c / 4 * 256];
        const uint32_t w = c % 4 == 0 ? v.x : c % 4 == 1 ? v.y : c % 4 == 2 ? v.z : v.w;
        const uint2 z = zero_words<BF>(ZEROS ? zero >> (8 * (c / 4)) & 255u : 8u);
        const uint2 lo = code_pairs<BF>(w, 0, magic, z), hi = code_pairs<BF>(w, 1, magic, z);
        a[4 * c] = lo.x; a[4 * c + 1] = lo.y; a[4 * c + 2] = hi.x; a[4 * c + 3] = hi.y;
      }
      if (s >= kWideStages) {
        barrier_wait(&sh.empty[slot], s / kWideStages - 1 & 1, &sh.failed);
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      }
      __syncwarp();
      tensor_store(lanes + slot * 64, a);
      uint8_t* b = smem + slot * kWideStageBytes<N>;
#pragma unroll
      for (int i = 0; i < kUnits; ++i) {
        const int u = d + 256 * i, r = u >> 3, c = u & 7;
        const uint4 v = raw[(2 + i) * 256], h = p.e4m3 ? bytes_to_half(v) : v;
        *reinterpret_cast<uint4*>(b + r * 128 + ((c ^ (r & 7)) << 4)) =
            make_uint4(__byte_perm(h.x, h.z, 0x5410), __byte_perm(h.x, h.z, 0x7632), __byte_perm(h.y, h.w, 0x5410),
                       __byte_perm(h.y, h.w, 0x7632));
      }
      fence_proxy_async_smem();
      tensor_store_wait();
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0) barrier_arrive(&sh.full[slot]);
    }
    wait_group<0>();
  }
  __syncwarp();
  if (p.split > 1) {
    cg::cluster_group cl = cg::this_cluster();
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
