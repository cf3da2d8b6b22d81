// The paged 4-bit cache of keys and values and the sequences of a call, as the kernels that
// write, read and attend to it see them (kd_cache4.cu, kd_attn4*.cu).
#pragma once
#include "kd_serve.cuh"

namespace kd {
namespace cache4 {

using namespace serve;

constexpr int64_t kMaxD = 256, kMaxSeqs = (int64_t)1 << 30;

// host checks, in parts: those of sizes, and of pointers that a call with work to do needs
inline bool cache_sizes_ok(const kd_cache4* c) {
  return c && c->pages >= 0 && c->pages <= INT32_MAX && c->heads >= 1 && c->heads <= 65535 && c->page >= 16 &&
         c->page <= 65536 && c->page % 16 == 0 && (c->group == 32 || c->group == 64 || c->group == 128);
}
inline bool cache_pointers_ok(const kd_cache4* c) {
  return c->k_codes && c->k_scales && c->v_codes && c->v_scales && aligned(c->k_codes, 16) && aligned(c->k_scales, 16) &&
         aligned(c->v_codes, 16) && aligned(c->v_scales, 16) && c->pages > 0;
}
inline bool sequences_sizes_ok(const kd_sequences* s) {
  return s && s->seqs >= 0 && s->seqs <= kMaxSeqs && s->wide >= 0 && s->wide <= INT32_MAX && s->ld_table >= s->wide &&
         s->most >= 0 && s->most <= INT32_MAX && s->longest >= 0;
}
inline bool sequences_pointers_ok(const kd_sequences* s) {
  return s->table && s->lengths && aligned(s->table, 4) && aligned(s->lengths, 4) && aligned(s->starts, 4) && s->wide > 0;
}

// rows of `heads` x `tokens` vectors of d elements do not overlap
inline bool rows_apart(int64_t tokens, int64_t heads, int64_t d, int64_t token, int64_t head) {
  if (tokens > 1 && heads > 1)
    return (head >= d && token >= d && (token - d) / head >= heads - 1) ||
           (token >= d && head >= d && (head - d) / token >= tokens - 1);
  return (tokens <= 1 || token >= d) && (heads <= 1 || head >= d);
}

// what the device needs of both
struct Pages {
  uint32_t* codes[2];   // keys, values
  uint32_t* scales[2];  // (step, low) pairs as words
  const int32_t* table;
  const int32_t* lengths;
  const int32_t* starts;
  int64_t ld_table;
  int seqs, wide, most;
  int pages, heads, page;
  int page_log;                  // of page, where it is a power of two, else -1
  int d, group, groups, chunks;  // of a row: channels, of one scale, scales, 32-channel pieces of codes
};
inline Pages pages_of(const kd_cache4* c, const kd_sequences* s) {
  Pages p{};
  p.codes[0] = c->k_codes;
  p.codes[1] = c->v_codes;
  p.scales[0] = reinterpret_cast<uint32_t*>(c->k_scales);
  p.scales[1] = reinterpret_cast<uint32_t*>(c->v_scales);
  p.table = s->table;
  p.lengths = s->lengths;
  p.starts = s->starts;
  p.ld_table = s->ld_table;
  p.seqs = (int)s->seqs;
  p.wide = (int)s->wide;
  p.most = (int)s->most;
  p.pages = (int)c->pages;
  p.heads = (int)c->heads;
  p.page = (int)c->page;
  p.page_log = -1;
  for (int log = 4; log <= 16; ++log)
    if (c->page == (int64_t)1 << log) p.page_log = log;
  p.d = (int)c->d;
  p.group = (int)c->group;
  p.groups = (int)((c->d + c->group - 1) / c->group);
  p.chunks = (int)((c->d + 31) / 32);
  return p;
}

// The first key head's row at a position of sequence s, -1 on a bad page.  Rows are counted in 64 bits: a cache may
// have more than 2^31.
__device__ __forceinline__ int64_t row_of(const Pages& p, int s, int position) {
  const unsigned nth = p.page_log >= 0 ? (unsigned)position >> p.page_log : (unsigned)position / (unsigned)p.page;
  if (nth >= (unsigned)p.wide) return -1;
  const int page = p.table[s * p.ld_table + nth];
  if ((unsigned)page >= (unsigned)p.pages) return -1;
  return (int64_t)page * p.heads * p.page + (int)((unsigned)position - nth * (unsigned)p.page);
}

// Row t's sequence, -1 for none, found by the whole warp: the last s with starts[s] <= t, 32 ways
// at a time (two rounds of loads for a thousand sequences).  before: rows of the sequence from t
// on, which place it before the sequence's end.
__device__ __forceinline__ int sequence_of(const Pages& p, int t, int& before) {
  const int lane = threadIdx.x & 31;
  if (!p.starts) {
    const int s = p.most > 0 ? t / p.most : p.seqs;
    before = p.most - (t - s * p.most);
    return s < p.seqs ? s : -1;
  }
  int lo = 0, hi = p.seqs + 1;
  for (;;) {
    const int stride = (hi - lo + 31) / 32;
    const int64_t at = lo + (int64_t)lane * stride;
    const int start = at < hi ? p.starts[at] : 0;
    const int found = __popc(__ballot_sync(~0u, at < hi && start <= t));
    if (found == 0) return -1;
    lo += (found - 1) * stride;
    if (stride == 1) {
      if (lo >= p.seqs) return -1;
      // the sequence's start and end are what these lanes have, but for the end in the last one
      const int64_t first = __shfl_sync(~0u, start, found - 1);
      int64_t end = __shfl_sync(~0u, start, found & 31);
      if (lo + 1 >= hi) end = p.starts[lo + 1];
      if (t < first || t >= end || t - first >= p.most) return -1;  // starts that decrease, rows past `most`
      before = (int)(end - t);
      return lo;
    }
    hi = (int)min((int64_t)lo + stride, (int64_t)hi);
  }
}

}  // namespace cache4
}  // namespace kd
