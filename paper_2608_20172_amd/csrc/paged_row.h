// One new row over a paged cache by one wave: its Self entry, Exchange states and
// how they join (eqs. 11-13). Args names a kernel's arguments: a paged cache c with
// its table [B, W], q, k, v, out, row_stat, G queries a key head, lambda, scale
// and inv_tau.
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

// The Self entry's reads of one wave, of row `row` of q (query head hq of request b) at position len (one-based):
// lane holds channels lane and lane + 64.
struct SelfEntry {
  float dot, v0, v1;  // q . k over the lane's channels; the own value
  bool ok;
};
template <typename TI, typename Args>
__device__ __forceinline__ SelfEntry read_self(const Args& a, int b, int64_t row, int hq, int len, int lane) {
  SelfEntry s{0.0f, 0.0f, 0.0f, false};
  if (len < 1) return s;
  int64_t off;
  s.ok = entry_offset(a, b, hq / a.G, len - 1, off);
  if (!s.ok) return s;
  const TI* q = (const TI*)a.q + row * a.c.D;
  const TI *k = (const TI*)a.k + off, *v = (const TI*)a.v + off;
  if (lane < a.c.D) {
    s.dot = Elem<TI>::load(q + lane) * Elem<TI>::load(k + lane);
    s.v0 = Elem<TI>::load(v + lane);
  }
  if (lane + 64 < a.c.D) {
    s.dot += Elem<TI>::load(q + lane + 64) * Elem<TI>::load(k + lane + 64);
    s.v1 = Elem<TI>::load(v + lane + 64);
  }
  return s;
}

// Eqs. 12-13 of a row at position len by one wave: state (m, l) with z0, z1 at channels lane, lane + 64.
template <typename TI, typename Args>
__device__ __forceinline__ void finish_row(const Args& a, int64_t row, int len, int lane, SelfEntry s, float m, float l,
                                           float z0, float z1) {
  float d = s.dot;
  for (int o = 32; o >= 1; o >>= 1) d += __shfl_xor(d, o, 64);
  const float S = 1.0f / (1.0f + expf(-d * a.scale * a.inv_tau));
  const float ln_i = logf((float)len);
  const float lam = *a.lambda;
  float g = 0.0f, omg = 1.0f, zr0 = 0.0f, zr1 = 0.0f, lnZ = S;
  if (!(l == 0.0f)) {                               // some history (or a NaN in it)
    const float A = m * kLn2 + logf(l) - lam * ln_i;       // A_i = L^E_i - lambda ln i (eq. 5)
    g = 1.0f / (1.0f + expf(S - A));                // g = sigmoid(A - S)
    omg = 1.0f / (1.0f + expf(A - S));              // 1 - g = sigmoid(S - A)
    const float il = 1.0f / l;
    zr0 = z0 * il;
    zr1 = z1 * il;
    lnZ = fmaxf(S, A) + log1pf(expf(-fabsf(S - A)));
  }
  // a length outside 1 .. max_len or a page outside the pool: NaN, so that the error is seen
  const float nan = __builtin_nanf("");
  TI* o = (TI*)a.out + row * a.c.D;
  if (lane < a.c.D) Elem<TI>::store(o + lane, s.ok ? omg * s.v0 + g * zr0 : nan);
  if (lane + 64 < a.c.D) Elem<TI>::store(o + lane + 64, s.ok ? omg * s.v1 + g * zr1 : nan);
  if (lane == 0 && a.row_stat) a.row_stat[row] = s.ok ? lnZ + lam * ln_i : nan;
}

}  // namespace rel
