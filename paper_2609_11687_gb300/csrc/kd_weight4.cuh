// Argument checks of a kd_weight4 shared by its producer (kd_weight4.cu) and the
// product (kd_mat4.cu).
#pragma once
#include "kd_serve.cuh"

namespace kd {
namespace serve {

inline bool weight4_sizes_ok(const kd_weight4* w) {
  return w && w->n >= 1 && w->n <= INT32_MAX && w->m >= 0 && w->m <= INT32_MAX &&
         (w->group == 32 || w->group == 64 || w->group == 128) &&
         (w->scale_dtype == KD_F16 || w->scale_dtype == KD_BF16);
}
inline bool weight4_pointers_ok(const kd_weight4* w) {
  return w->codes && w->scales && aligned(w->codes, 16) && aligned(w->scales, 2);
}
inline int64_t weight4_words(int64_t n) { return (n + 31) / 32 * 4; }

}  // namespace serve
}  // namespace kd
