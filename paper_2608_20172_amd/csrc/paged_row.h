// Rows over a paged cache: where an entry stands, and how Exchange states join
// (eq. 11). Args names a kernel's arguments: a paged cache c with its table [B, W].
#pragma once

#include "common.h"

namespace rel {

// Merges state (mo, lo, zo) into (m, l, z); an empty state has m = -inf, l = 0. A NaN in l stays.
template <int VEC>
__device__ __forceinline__ void merge_into(float& m, float& l, float (&z)[VEC], float mo, float lo,
                                           const float (&zo)[VEC]) {
  const float mn = fmaxf(m, mo);
  const float a = m == kNegInf ? 0.0f : fast_exp2(m - mn);
  const float b = mo == kNegInf ? 0.0f : fast_exp2(mo - mn);
  l = l * a + lo * b;
#pragma unroll
  for (int e = 0; e < VEC; ++e) z[e] = z[e] * a + zo[e] * b;
  m = mn;
}

// Element offset of the request's entry j (0-based) at head h; false if its page is not one of the pool's.
template <typename Args>
__device__ __forceinline__ bool entry_offset(const Args& a, int b, int h, int j, int64_t& off) {
  const int id = a.table[(int64_t)b * a.W + (j >> a.c.shift)];
  const bool ok = id >= 0 && id < a.c.num_pages;
  off = (int64_t)(ok ? id : 0) * a.c.sp + (int64_t)h * a.c.sh + (int64_t)(j & ((1 << a.c.shift) - 1)) * a.c.st;
  return ok;
}

}  // namespace rel
