// The Exchange scan of 32 query rows by one wave, as the fused forward kernels and
// the chunk kernel over pages run it: evidence of 32-key blocks in transposed
// 32x32 MFMA blocks, the weights, the value sums, and the row epilogue.
#pragma once

#include "common.h"

namespace rel {

constexpr float kRescale = 8.0f;
constexpr float kSpecMax = 18446744073709551616.0f;  // 2^64

constexpr int kIlValu = 28;  // vector instructions scheduled after each matrix instruction in full tiles

// How the query operand carries c = scale log2(e):
//   0 (bf16): raw q; each evidence entry is multiplied by c in fp32
//   1 (fp32): q c in the operand
template <class P, int D>
constexpr int qmode() {
  return sizeof(typename P::T) == 4 ? 1 : 0;
}

// Exchange logits of one 32x32 block, in place: s[r] (U log2 e, or raw q.k in
// mode 0) becomes E log2(e) - m; in a block that meets the diagonal (DIAG) the
// entries from key `self` on, the lane's own position counted from the block's
// first key, get -inf. mx tracks the lane's largest value.
template <bool DIAG, int QM, bool TRACK = true>
__device__ __forceinline__ void exchange_logits(floatx16& s, const Lane& L, int self, float c, float m, float& mx) {
  // passes over groups of 4 independent entries: consecutive instructions do
  // not wait on a transcendental result, and few temporaries are live
#pragma unroll
  for (int r0 = 0; r0 < 16; r0 += 4) {
    float up[4], t[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) up[r] = QM == 0 ? s[r0 + r] * c : s[r0 + r];   // U log2(e)
#pragma unroll
    for (int r = 0; r < 4; ++r) t[r] = fast_exp2(-up[r]);
#pragma unroll
    for (int r = 0; r < 4; ++r) t[r] = fast_rcp(1.0f + t[r]);                  // sigmoid(U)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float e = __builtin_fmaf(up[r], t[r], -m);                               // SiLU(U) log2(e) - m
      if (DIAG && acc_row(r0 + r, L.g) >= self) e = kNegInf;                    // strictly historical: j < i
      s[r0 + r] = e;
    }
    if (TRACK) mx = fmaxf(mx, fmaxf(fmaxf(s[r0], s[r0 + 1]), fmaxf(s[r0 + 2], s[r0 + 3])));
  }
}

// Whether this lane holds the evidence of key `self` of a block, the Self evidence of its row.
__device__ __forceinline__ bool holds_self(int self, int g) { return (unsigned)self < 32u && holds_row(self, g); }

// An operand with 0 in the place of what is not finite.
__device__ __forceinline__ bf16x8 finite_part(const bf16x8& x) {
  uintx4 u = __builtin_bit_cast(uintx4, x);
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    if ((u[t] & 0x7f80u) == 0x7f80u) u[t] &= 0xffff0000u;
    if ((u[t] & 0x7f800000u) == 0x7f800000u) u[t] &= 0xffffu;
  }
  return __builtin_bit_cast(bf16x8, u);
}
__device__ __forceinline__ floatx8 finite_part(floatx8 x) {
#pragma unroll
  for (int t = 0; t < 8; ++t) x[t] = fabsf(x[t]) < __builtin_inff() ? x[t] : 0.0f;
  return x;
}

// What the rounding of the weights p to the operand hi leaves of them, as an operand: bf16 weights of two parts
// have 16 significant bits.
template <class P>
__device__ __forceinline__ typename P::Op rest_of(const float (&p)[8], const typename P::Op& hi) {
  static_assert(sizeof(typename P::T) == 2, "fp32 weights have no rest");
  const uintx4 u = __builtin_bit_cast(uintx4, hi);
  float r[8];
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    r[2 * t] = p[2 * t] - bf16_lo(u[t]);
    r[2 * t + 1] = p[2 * t + 1] - bf16_hi(u[t]);
  }
  return P::pack(r);
}

// One 32-key block of the scan for this wave's 32 rows: s holds the block's
// evidence (layout of a 32x32 accumulator, keys on rows, queries on lanes);
// Vs is the V tile and vslice the index of the block's first 16-key slice. CLEAN:
// values that are not finite count as 0. TWO: bf16 weights in two parts.
template <class P, int D, int QM, bool DIAG, bool CLEAN = false, bool TWO = false>
__device__ __forceinline__ void scan_block(floatx16 s, floatx16 (&oacc)[D / 32], float& m, float& l,
                                           float& uii, const unsigned char* Vs, int vslice,
                                           const Lane& L, int self, float c) {
  constexpr int DB = D / 32;
  using Op = typename P::Op;
  if (DIAG && holds_self(self, L.g)) uii = pick(s, row_reg(self));
  float mx = kNegInf;
  exchange_logits<DIAG, QM>(s, L, self, c, m, mx);
  if (wave_any(mx > kRescale)) {
    const float d = fmaxf(fmaxf(mx, xor32(mx)), 0.0f);  // row max over both halves
    m += d;
    const float al = fast_exp2(-d);
    l *= al;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) oacc[db][r] *= al;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] -= d;
  }
  // l sums the fp32 p (not the bf16-rounded MFMA operand), so that L^E and the
  // saved statistic M carry no operand rounding
#pragma unroll
  for (int hh = 0; hh < 2; ++hh) {
    float p[8];
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      p[t] = fast_exp2(s[8 * hh + t]);
      l += p[t];
    }
    const Op pop = P::pack(p);
    Op rest;
    if constexpr (TWO) rest = rest_of<P>(p, pop);
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      Op vop = P::col_op(Vs, vslice + hh, 32 * db, L);
      if (CLEAN) vop = finite_part(vop);
      oacc[db] = P::mma(vop, pop, oacc[db]);
      if constexpr (TWO) oacc[db] = P::mma(vop, rest, oacc[db]);
    }
  }
}

// Evidence block: keys krow0 .. krow0+31 of the K tile against this lane's row.
template <class P, int KS>
__device__ __forceinline__ floatx16 evidence(const unsigned char* Ks, int krow0, const typename P::Op (&qop)[KS],
                                             const Lane& L) {
  floatx16 s = {};
#pragma unroll
  for (int k0 = 0; k0 < KS; k0 += 2) {  // operands two slices at a time
    typename P::Op ka[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) ka[j] = P::row_op(Ks, krow0 + L.n, k0 + j, L);
#pragma unroll
    for (int j = 0; j < 2; ++j) s = P::mma(ka[j], qop[k0 + j], s);
  }
  return s;
}

// A block of the scan with the reference m held fixed: the logits of the block,
// the packed weights P of its two 16-key halves and their sum into l; with TWO
// the rest of the bf16 weights as well.
template <class P, int D, int QM, bool DIAG, bool TWO = false>
__device__ __forceinline__ void fast_block(floatx16 s, float m, float& l, float& uii, typename P::Op (&pop)[2],
                                           const Lane& L, int self, float c, typename P::Op* rest = nullptr) {
  if (DIAG && holds_self(self, L.g)) uii = pick(s, row_reg(self));
  float mx = kNegInf;
  exchange_logits<DIAG, QM, false>(s, L, self, c, m, mx);
  // l sums the fp32 p (not the bf16-rounded MFMA operand), so that L^E and the
  // saved statistic M carry no operand rounding
#pragma unroll
  for (int hh = 0; hh < 2; ++hh) {
    float p[8];
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      p[t] = fast_exp2(s[8 * hh + t]);
      l += p[t];
    }
    pop[hh] = P::pack(p);
    if constexpr (TWO) rest[hh] = rest_of<P>(p, pop[hh]);
  }
}

// The weights of one block into the value sums: b counts the blocks of the tile from V's row krow0.
template <class P, int D>
__device__ __forceinline__ void add_values(const unsigned char* Vs, int krow0, int b, const typename P::Op (&pop)[2],
                                           floatx16 (&oacc)[D / 32], const Lane& L) {
#pragma unroll
  for (int hh = 0; hh < 2; ++hh)
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
      oacc[db] = P::mma(P::col_op(Vs, krow0 / 16 + 2 * b + hh, 32 * db, L), pop[hh], oacc[db]);
}
// The same of weights in two parts.
template <class P, int D>
__device__ __forceinline__ void add_values(const unsigned char* Vs, int krow0, int b, const typename P::Op (&pop)[2],
                                           const typename P::Op (&rest)[2], floatx16 (&oacc)[D / 32], const Lane& L) {
#pragma unroll
  for (int hh = 0; hh < 2; ++hh)
#pragma unroll
    for (int db = 0; db < D / 32; ++db) {
      const typename P::Op vop = P::col_op(Vs, krow0 / 16 + 2 * b + hh, 32 * db, L);
      oacc[db] = P::mma(vop, pop[hh], oacc[db]);
      oacc[db] = P::mma(vop, rest[hh], oacc[db]);
    }
}

// The 64 keys krow0 .. krow0+63 of a tile, all before every row of the wave, with the reference held fixed.
template <class P, int D, int QM>
__device__ __forceinline__ void full_keys64(const unsigned char* Ks, const unsigned char* Vs, int krow0,
                                            const typename P::Op (&qop)[D / 16], floatx16 (&oacc)[D / 32], float m,
                                            float& l, float& uii, const Lane& L, float c) {
  constexpr int KS = D / 16, DB = D / 32;
  using Op = typename P::Op;
  Op p0[2] = {Op{}, Op{}}, p1[2] = {Op{}, Op{}};
  floatx16 s1;
  // one basic block: the evidence of block 1 under the vector work of block
  // 0, the P V products of block 0 under that of block 1
  const floatx16 s0 = evidence<P, KS>(Ks, krow0, qop, L);
  __builtin_amdgcn_sched_barrier(0);
  s1 = evidence<P, KS>(Ks, krow0 + 32, qop, L);
  fast_block<P, D, QM, false>(s0, m, l, uii, p0, L, 0, c);
  __builtin_amdgcn_sched_group_barrier(0x100, 64, 0);
#pragma unroll
  for (int i = 0; i < KS; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x002, kIlValu, 0);
  }
  __builtin_amdgcn_sched_barrier(0);
  add_values<P, D>(Vs, krow0, 0, p0, oacc, L);
  fast_block<P, D, QM, false>(s1, m, l, uii, p1, L, 0, c);
  __builtin_amdgcn_sched_group_barrier(0x100, 64, 1);
#pragma unroll
  for (int i = 0; i < 2 * DB; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 1);
    __builtin_amdgcn_sched_group_barrier(0x002, kIlValu, 1);
  }
  __builtin_amdgcn_sched_barrier(0);
  add_values<P, D>(Vs, krow0, 1, p1, oacc, L);
}

struct RowEpilogue {
  float g, omg, inv_l, LE, lnZ, S;
};

// Completes row i from the terminal scan state (eqs. 12-13):
// L^E = m + ln l, A = L^E - lambda ln i, g = sigmoid(A - S), 1-g = sigmoid(S - A).
// uii2 = U_ii log2(e).
__device__ __forceinline__ RowEpilogue row_epilogue(float m_log2, float l, float uii2, float inv_tau,
                                                    float lam, float ln_i) {
  RowEpilogue e;
  e.S = 1.0f / (1.0f + exp2f(-uii2 * inv_tau));
  if (l > 0.0f) {
    e.LE = (m_log2 + log2f(l)) * kLn2;
    const float A = e.LE - lam * ln_i;
    const float d = A - e.S;
    e.g = 1.0f / (1.0f + expf(-d));
    e.omg = 1.0f / (1.0f + expf(d));
    e.lnZ = fmaxf(e.S, A) + log1pf(expf(-fabsf(d)));
    e.inv_l = e.g / l;
  } else {  // empty history (row 1): g = 0, y = v (App. A.1.8)
    e.LE = kNegInf;
    e.g = 0.0f;
    e.omg = 1.0f;
    e.lnZ = e.S;
    e.inv_l = 0.0f;
  }
  return e;
}

}  // namespace rel
