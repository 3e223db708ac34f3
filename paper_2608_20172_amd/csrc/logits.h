// Rows of logits in registers: loads of 16 bytes on any element boundary, NaN as
// -inf, the order of the numbers as bits, and reductions over a wave.
#pragma once

#include "common.h"

namespace rel {

__device__ __forceinline__ float no_nan(float x) { return x == x ? x : kNegInf; }

// Loads of 16 bytes, on any element boundary: raw first, so that a run of them is in flight together.
template <typename TI>
struct Logits;
template <>
struct Logits<float> {
  static constexpr int VE = 4;
  typedef float V __attribute__((ext_vector_type(4), aligned(4)));
  static __device__ __forceinline__ void values(const V& u, float (&x)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = no_nan(u[e]);
  }
};
template <>
struct Logits<bf16> {
  static constexpr int VE = 8;
  typedef unsigned int V __attribute__((ext_vector_type(4), aligned(2)));
  static __device__ __forceinline__ void values(const V& u, float (&x)[8]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[2 * e] = no_nan(bf16_lo(u[e]));
      x[2 * e + 1] = no_nan(bf16_hi(u[e]));
    }
  }
};
__device__ __forceinline__ float element(const Logits<float>::V& u, int e) { return u[e]; }
__device__ __forceinline__ float element(const Logits<bf16>::V& u, int e) {
  return e & 1 ? bf16_hi(u[e >> 1]) : bf16_lo(u[e >> 1]);
}
__device__ __forceinline__ void set_lowest(Logits<float>::V& u, int e) { u[e] = kNegInf; }
__device__ __forceinline__ void set_lowest(Logits<bf16>::V& u, int e) {
  u[e >> 1] = e & 1 ? (u[e >> 1] & 0xffffu) | 0xff800000u : (u[e >> 1] & 0xffff0000u) | 0xff80u;
}

// N runs of VE elements of a row of V: run s is wanted from at[s] on. Where it
// would pass the row's end it is the row's last VE elements (at[s] becomes their
// first), and those before the wanted ones, which another run has, are -inf.
template <typename TI, int N>
__device__ __forceinline__ void load_runs(const TI* row, int V, int (&at)[N], float (&x)[N][Logits<TI>::VE]) {
  constexpr int VE = Logits<TI>::VE;
  if (V >= VE) {
    typename Logits<TI>::V raw[N];
    int want[N];
#pragma unroll
    for (int s = 0; s < N; ++s) {
      want[s] = at[s];
      at[s] = min(at[s], V - VE);
      raw[s] = *reinterpret_cast<const typename Logits<TI>::V*>(row + at[s]);
    }
#pragma unroll
    for (int s = 0; s < N; ++s) {
      Logits<TI>::values(raw[s], x[s]);
      if (__any(want[s] != at[s])) {
#pragma unroll
        for (int e = 0; e < VE; ++e)
          if (at[s] + e < want[s]) x[s][e] = kNegInf;
      }
    }
  } else {
#pragma unroll
    for (int s = 0; s < N; ++s) {
#pragma unroll
      for (int e = 0; e < VE; ++e) x[s][e] = at[s] + e < V ? no_nan((float)row[at[s] + e]) : kNegInf;
    }
  }
}
// Makes the compiler take the values as new: what it derived from them in one pass
// over the registers (an index or an unpacked number for each) is derived again in
// the next, not kept in registers, and not in scratch memory.
template <int N>
__device__ __forceinline__ void derive_again(int (&at)[N]) {
#pragma unroll
  for (int s = 0; s < N; ++s) asm volatile("" : "+v"(at[s]));
}

// Bits in the order of the numbers, and back.
__device__ __forceinline__ unsigned ordered(float x) {
  const unsigned u = __builtin_bit_cast(unsigned, x);
  return u ^ ((unsigned)((int)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unordered(unsigned u) {
  return __builtin_bit_cast(float, u & 0x80000000u ? u ^ 0x80000000u : ~u);
}

// Reductions over a wave whose result every lane has: lane moves inside rows of
// 16 on the vector unit, then two exchanges across the rows.
template <int CTRL>
__device__ __forceinline__ int dpp_word(int x) {
  return __builtin_amdgcn_update_dpp(0, x, CTRL, 0xF, 0xF, false);
}
template <typename T, typename M>
__device__ __forceinline__ T moved(T x, M move) {
  static_assert(sizeof(T) % 4 == 0, "whole words");
  struct Words {
    int w[sizeof(T) / 4];
  } u = __builtin_bit_cast(Words, x);
#pragma unroll
  for (unsigned k = 0; k < sizeof(T) / 4; ++k) u.w[k] = move(u.w[k]);
  return __builtin_bit_cast(T, u);
}
// Over aligned groups of G lanes, 4 to 16.
template <int G, typename T, typename F>
__device__ __forceinline__ T group_reduce(T x, F join) {
  x = join(x, moved(x, [](int y) { return dpp_word<0xB1>(y); }));                      // lane ^ 1
  x = join(x, moved(x, [](int y) { return dpp_word<0x4E>(y); }));                      // lane ^ 2
  if constexpr (G >= 8) x = join(x, moved(x, [](int y) { return dpp_word<0x141>(y); }));   // lane i <-> 7 - i of its 8
  if constexpr (G >= 16) x = join(x, moved(x, [](int y) { return dpp_word<0x140>(y); }));  // lane i <-> 15 - i of its 16
  return x;
}
template <typename T, typename F>
__device__ __forceinline__ T wave_reduce(T x, F join) {
  x = group_reduce<16>(x, join);
  x = join(x, moved(x, [](int y) { return __shfl_xor(y, 16, 64); }));
  return join(x, moved(x, [](int y) { return __shfl_xor(y, 32, 64); }));
}
__device__ __forceinline__ float wave_max(float x) {
  return wave_reduce(x, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float wave_sum(float x) {
  return wave_reduce(x, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ int wave_sum(int x) {
  return wave_reduce(x, [](int a, int b) { return a + b; });
}

}  // namespace rel
