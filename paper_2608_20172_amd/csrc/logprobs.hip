// Log-probabilities of given tokens, with entropy, rank and the likeliest
// alternatives, and the gradient by the logits.
//
// With m = max x, w_i = exp(x_i - m), Z = sum w, T = sum w_i (x_i - m):
//   log p_t = x_t - m - ln Z,  entropy = ln Z - T / Z,
//   rank = how many x_i are over x_t, or equal to it at a lower index.
// All four come from one pass over the row: a thread holds S pieces of 16 bytes in
// registers, takes its own maximum, sums against it, and states (m_k, Z_k, T_k) join as
//   m = max m_k, Z = sum a_k Z_k, T = sum a_k (T_k + (m_k - m) Z_k), a_k = exp(m_k - m).
// A row is cut into chunks of 256 S such pieces, a workgroup each; a second kernel
// joins the chunks of rows that have several.
// Alternatives: K thread maxima, the 4th part of them in each wave or all in one, bound
// the K-th largest logit from below; what is over the bound (some more than K) is
// listed in LDS, and an entry's place is the number of entries over it. Where a list
// overflows (ties at the bound: flat rows) the K-th largest is found by bisection, and
// of its equals the lowest indices. In the sub-chunks after a workgroup's first the
// K-th so far is the bound.
// Bounds: the read of the logits (4000 x 57344 in bf16, 459 MB: 82 us, 5.6 TB/s), with
// the rank 85; with 20 alternatives and the rank 4000 x 50257 131 us, 3.1 TB/s: six waves
// a SIMD of vector work and three barriers a sub-chunk, between which nobody loads. The
// backward pass reads and writes once: 4096 x 131072 in bf16 400 us, 5.4 TB/s.
// Pieces a thread: 4, 6 and 8 of them took 89, 81 and 102 us for 4000 x 50257 (8 leave
// five waves a SIMD, and half of the last sub-chunk empty), 208, 226 and 236 for 4096 x
// 131072. Numbers unpacked once and kept: one wave a SIMD, 234 us for 1000 x 50257 with 20
// alternatives, against 44.
#include <algorithm>
#include <type_traits>

#include "logits.h"
#include "tokens.h"

namespace rel {

namespace {

constexpr int kT = 256;
constexpr int kNW = kT / 64;
constexpr int kCap = 256;        // listed logits of a wave's share of a chunk
constexpr int kMaxS = 6;         // pieces of 16 bytes that a thread holds
constexpr int kMaxSubs = 64;     // sub-chunks of a workgroup
constexpr float kFar = 65536.0f;  // a row whose maximum is beyond takes differences before it multiplies by log2 e
constexpr int kFillGroups = 1024;  // workgroups that fill the chip
constexpr int kMaxKeys = 512;    // keys of a row's parts
constexpr unsigned kOrderedNegInf = 0x007fffffu;  // ordered(-inf)

// Low bits of the ordered logit that a cut leaves out: all that bf16 has not, some of fp32's.
template <typename TI>
constexpr int kCutBits = sizeof(TI) == 2 ? 16 : 12;

// What a workgroup leaves of its part of a row.
struct State {
  float m, z, t;  // maximum, sum of w, sum of w (x - m); m = -inf: nothing above it
  int before;     // logits before the given token
};
// State (m, z, t) against the maximum top of those that it is joined with: then z and t add up.
__device__ __forceinline__ State against(State s, float top) {
  // 0, not NaN, for what lies infinitely below, and for equal infinities
  const float d = s.m == top ? 0.0f : fmaxf(s.m - top, -1000.0f), w = fast_exp2(d * kLog2e);
  return State{top, s.z * w, w * __builtin_fmaf(d, s.z, s.t), s.before};
}
__device__ __forceinline__ State join4(State a, State b, State c, State d) {
  const float top = fmaxf(fmaxf(a.m, b.m), fmaxf(c.m, d.m));
  a = against(a, top);
  b = against(b, top);
  c = against(c, top);
  d = against(d, top);
  return State{top, (a.z + b.z) + (c.z + d.z), (a.t + b.t) + (c.t + d.t), (a.before + b.before) + (c.before + d.before)};
}
__device__ __forceinline__ State wave_join(State s) {
  s = against(s, wave_max(s.m));
  return State{s.m, wave_sum(s.z), wave_sum(s.t), s.before};
}

// The states of n sub-chunks as one, by every wave alike.
template <typename F>
__device__ __forceinline__ State fold(F of_sub, int n) {
  if (n == 1) return of_sub(0);
  State s{kNegInf, 0.0f, 0.0f, 0};
  for (int i = threadIdx.x & 63; i < n; i += 64) {
    const State o = of_sub(i);
    const float top = fmaxf(s.m, o.m);
    const State x = against(s, top), y = against(o, top);
    s = State{top, x.z + y.z, x.t + y.t, x.before + y.before};
  }
  s = wave_join(s);
  s.before = wave_sum(s.before);
  return s;
}

// An entry of the order: larger first, equal ones by the lower index. Unlike any other.
typedef unsigned long long Key;
__device__ __forceinline__ Key key_of(float x, int i) {
  return ((Key)ordered(no_nan(x) + 0.0f) << 32) | (unsigned)~i;  // + 0: -0 and 0 are equal
}
__device__ __forceinline__ float key_value(Key k) { return unordered((unsigned)(k >> 32)); }
__device__ __forceinline__ int key_index(Key k) { return (int)~(unsigned)k; }

// Outputs of one row from its state and, for K > 0, its K first keys in LDS.
__device__ __forceinline__ void finish(const LogprobArgs& a, int n, State s, float xt, const Key* first) {
  const float nan = __builtin_nanf("");
  const int64_t t = a.tokens[n];
  const bool none = s.m == kNegInf;  // nothing above -inf
  const float ln_z = none ? nan : logf(s.z), H = none ? nan : ln_z - s.t / s.z;
  const int tid = threadIdx.x;
  if (tid == 0) {
    xt = no_nan(xt);
    const float lp = t < 0 ? 0.0f : none || t >= a.V ? nan : (xt == s.m ? 0.0f : xt - s.m) - ln_z;
    if (a.logprob) a.logprob[n] = lp;
    if (a.entropy) a.entropy[n] = H;
    if (a.rank) a.rank[n] = none || t < 0 || t >= a.V ? -1 : s.before;
    if (a.stats) *reinterpret_cast<float4*>(a.stats + 4 * (int64_t)n) = float4{s.m, none ? nan : 1.0f / s.z, ln_z, H};
  }
  if (tid < a.K) {
    const Key k = first[tid];
    const float x = key_value(k);
    a.top_tokens[(int64_t)n * a.K + tid] = none ? -1 : key_index(k);
    a.top_logprobs[(int64_t)n * a.K + tid] = none ? nan : (x == s.m ? 0.0f : x - s.m) - ln_z;
  }
}

// The number below x: a > number_below(x) is a >= x (below 0 and -0: past both).
__device__ __forceinline__ float number_below(float x) { return unordered(ordered(x + 0.0f) - (x == 0.0f ? 2 : 1)); }

// Lists of keys in LDS: one of each wave, and the K first so far.
struct Lists {
  Key wave[kNW][kCap];
  Key held[kLogprobMaxK];
  unsigned cut[2][kNW];
  int count[kNW];
  int total;
};

// How many keys of list are over mine.
__device__ __forceinline__ int keys_over(const Key* list, int n, Key mine) {
  int place = 0, j = 0;
  for (; j + 4 <= n; j += 4) {  // four reads in flight
    Key k[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) k[u] = list[j + u];
#pragma unroll
    for (int u = 0; u < 4; ++u) place += k[u] > mine;
  }
  for (; j < n; ++j) place += list[j] > mine;
  return place;
}
// The K first of all lists into out, in order: an entry's place is the number of entries over it, counted by four lanes,
// each over one wave's list. Every place of the first min(K, n) gets its entry because no two keys are alike: a logit is
// listed by the one thread whose piece it is (real()), in the sub-chunk that has it. Places from n on are left as they
// were; the lists of a row have K entries in all, as K is at most V.
__device__ __forceinline__ void first_keys(const Lists& l, int held, int K, Key* out) {
  const int sub = threadIdx.x & 3;
  int n = held, count[kNW];
#pragma unroll
  for (int w = 0; w < kNW; ++w) n += count[w] = l.count[w];
  const int own = l.count[sub];
  for (int i = threadIdx.x >> 2; i < (n + 63) / 64 * 64; i += kT / 4) {  // whole waves reach the lane moves
    int at = min(i, n - 1), list = 0;
#pragma unroll
    for (int w = 0; w < kNW; ++w)
      if (list == w && at >= count[w]) {
        at -= count[w];
        ++list;
      }
    const Key mine = list < kNW ? l.wave[list][at] : l.held[at];
    int place = keys_over(l.wave[sub], own, mine);
    if (sub == 0) place += keys_over(l.held, held, mine);
    place += moved(place, [](int y) { return dpp_word<0xB1>(y); });
    place += moved(place, [](int y) { return dpp_word<0x4E>(y); });
    if (i < n && place < K && sub == 0) out[place] = mine;
  }
}

// The largest of three numbers, none of them NaN: one instruction (fmaxf quiets its operands first).
__device__ __forceinline__ float max3(float a, float b, float c) {
  float m;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(m) : "v"(a), "v"(b), "v"(c));
  return m;
}

// Pieces of 16 bytes of a row in registers, as they were read but for NaN (-inf) and for what is not this thread's
// (nothing(), below every other): piece s is wanted from want(s) on, and where it would pass the row's end it is the
// row's last VE logits, the first of which another piece has. Numbers are unpacked where they are used: kept unpacked,
// they would take twice the registers, and half of the waves.
constexpr float kWild = 0x1p119f;  // logits of this size or more, and NaN, are looked after; others are tame
template <typename TI, int S>
struct Pieces {
  static constexpr int VE = Logits<TI>::VE;
  typename Logits<TI>::V raw[S];
  int V, first;  // the row's length; want(0)
  int used;      // pieces of which the wave has a part (scalar)
  bool tame;     // all of the wave's logits are
  __device__ __forceinline__ int want(int s) const { return first + s * kT * VE; }
  __device__ __forceinline__ int at(int s) const { return V >= VE ? min(want(s), V - VE) : want(s); }
  __device__ __forceinline__ float x(int s, int e) const { return element(raw[s], e); }
  // whether element e of piece s is a logit of the row, and this piece's
  __device__ __forceinline__ bool real(int s, int e) const {
    const int i = at(s) + e;
    return i >= want(s) && i < V;
  }
  __device__ __forceinline__ void load(const TI* row) {
    used = __builtin_amdgcn_readfirstlane(min(S, max(0, (V - first + kT * VE - 1) / (kT * VE))));
    if (V >= VE) {
#pragma unroll
      for (int s = 0; s < S; ++s) raw[s] = *reinterpret_cast<const typename Logits<TI>::V*>(row + at(s));
    } else {
#pragma unroll
      for (int s = 0; s < S; ++s)
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          set_lowest(raw[s], e);
          if (want(s) + e < V) set_element(raw[s], e, row[want(s) + e]);
        }
    }
    tame = !__any(wild(raw));
    if (!tame) clean(raw);
    if (V >= VE && want(S - 1) > V - VE) {
#pragma unroll
      for (int s = 0; s < S; ++s) leave_out(raw[s], want(s) - at(s), tame ? -kWild : kNegInf);
    }
  }
  // The first n elements of a piece become x.
  static __device__ __forceinline__ void leave_out(Logits<float>::V& u, int n, float x) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < n) u[e] = x;
  }
  static __device__ __forceinline__ void leave_out(Logits<bf16>::V& u, int n, float x) {
    const unsigned hi = __builtin_bit_cast(unsigned, x), lo = hi >> 16;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      if (2 * t < n) u[t] = (u[t] & 0xffff0000u) | lo;
      if (2 * t + 1 < n) u[t] = lo | hi;
    }
  }
  static __device__ __forceinline__ bool wild(const Logits<float>::V (&u)[S]) {
    bool some = false;
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int e = 0; e < 4; ++e) some |= !(fabsf(u[s][e]) < kWild);
    return some;
  }
  // kWild is 0x7b00: sizes from there on carry into the sign's place.
  static __device__ __forceinline__ bool wild(const Logits<bf16>::V (&u)[S]) {
    unsigned some = 0;
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int t = 0; t < 4; ++t) some |= (u[s][t] & 0x7fff7fffu) + 0x05000500u;
    return (some & 0x80008000u) != 0;
  }
  static __device__ __forceinline__ void set_element(Logits<float>::V& u, int e, float x) { u[e] = x; }
  static __device__ __forceinline__ void set_element(Logits<bf16>::V& u, int e, bf16 x) {
    const unsigned b = __builtin_bit_cast(unsigned short, x);
    u[e >> 1] = e & 1 ? (u[e >> 1] & 0xffffu) | b << 16 : (u[e >> 1] & 0xffff0000u) | b;
  }
  // NaN becomes -inf.
  static __device__ __forceinline__ void clean(Logits<float>::V (&u)[S]) {
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int e = 0; e < 4; ++e) u[s][e] = no_nan(u[s][e]);
  }
  static __device__ __forceinline__ void clean(Logits<bf16>::V (&u)[S]) {
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        if ((u[s][t] & 0x7fffu) > 0x7f80u) u[s][t] = (u[s][t] & 0xffff0000u) | 0xff80u;
        if ((u[s][t] & 0x7fff0000u) > 0x7f800000u) u[s][t] = (u[s][t] & 0xffffu) | 0xff800000u;
      }
  }
  // The largest of the pieces' logits (of which none is NaN).
  __device__ __forceinline__ float largest() const { return tame ? largest(raw, 0xffffffffu) : largest(raw, 0xffff0000u); }
  static __device__ __forceinline__ float largest(const Logits<float>::V (&u)[S], unsigned) {
    float m = kNegInf;
#pragma unroll
    for (int s = 0; s < S; ++s) m = max3(max3(m, u[s][0], u[s][1]), u[s][2], u[s][3]);
    return m;
  }
  // A word's number is its high logit's with more bits behind, which the order of the high logits does not see; but
  // behind an infinity they would make a NaN, and are left out.
  static __device__ __forceinline__ float largest(const Logits<bf16>::V (&u)[S], unsigned bits) {
    float hi = kNegInf, lo = kNegInf;
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int t = 0; t < 4; t += 2) {
        hi = max3(hi, __builtin_bit_cast(float, u[s][t] & bits), __builtin_bit_cast(float, u[s][t + 1] & bits));
        lo = max3(lo, bf16_lo(u[s][t]), bf16_lo(u[s][t + 1]));
      }
    return max3(lo, lo, bf16_hi(__builtin_bit_cast(unsigned, hi)));
  }
  // What a pass has unpacked is not kept for the next.
  __device__ __forceinline__ void unpack_again() {
    asm volatile("" : "+v"(first));
#pragma unroll
    for (int s = 0; s < S; ++s) asm volatile("" : "+v"(raw[s]));
  }
};
// Part blockIdx.x % parts of row blockIdx.x / parts: sub-chunks of kT S pieces, one after another.
template <typename TI, int S, bool RANK, bool TOP>
__global__ __launch_bounds__(kT, TOP ? 6 : 1) void logprobs_kernel(LogprobArgs a, int parts, int subs, State* states, Key* keys) {
  constexpr int VE = Logits<TI>::VE, CH = kT * S * VE;
  __shared__ State joined[kMaxSubs][kNW];
  __shared__ Lists sh;                   // TOP
  __shared__ Key first[kLogprobMaxK];    // TOP: the K first so far
  const int part = blockIdx.x % parts, n = blockIdx.x / parts;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const TI* row = (const TI*)a.logits + (int64_t)n * a.sl;
  const int64_t t64 = a.tokens[n];
  const bool given = t64 >= 0 && t64 < a.V;
  const int t = given ? (int)t64 : -1;
  float xt = kNegInf;
  if (given) xt = no_nan((float)row[t]);
  // x is before t: x > xt, or x >= xt at a lower index; x >= xt is x > the number below xt
  float below = xt;
  if (RANK && given && xt > kNegInf) below = number_below(xt);
  int held = 0;    // keys in first
  const int all = (a.V + CH - 1) / CH, sub0 = part * subs, nsub = min(subs, all - sub0);
  for (int sub = 0; sub < nsub; ++sub) {
    const int base = (sub0 + sub) * CH;
    int before = 0;  // of the whole wave
    Pieces<TI, S> p;
    p.V = a.V;
    p.first = base + tid * VE;
    p.load(row);
    const bool has = p.first < a.V;  // this thread has a part of the row
    const float m = has ? p.largest() : kNegInf;
    p.unpack_again();
    float z = 0.0f, tt = 0.0f;
    if (__any(fabsf(m) > kFar && m > kNegInf)) {  // far from 0: differences first; +inf weighs 1, all below it nothing
#pragma unroll
      for (int s = 0; s < S; ++s)
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          const float d = p.x(s, e) == m ? 0.0f : fmaxf(p.x(s, e) - m, -1000.0f), y = fast_exp2(d * kLog2e);
          z += y;
          tt = __builtin_fmaf(y, d, tt);
        }
    } else {
      // w = 2^(x log2 e - c) with c the rounded m log2 e: one instruction, rounded once. What c is off by is taken out of
      // the sums.
      const float c = m * kLog2e;
      auto sum = [&](auto clamped) __attribute__((always_inline)) {
#pragma unroll
        for (int s = 0; s < S; ++s) {
          if (s >= p.used) break;
#pragma unroll
          for (int e = 0; e < VE; ++e) {
            float d = __builtin_fmaf(p.x(s, e), kLog2e, -c);
            if (decltype(clamped)::value) d = fmaxf(d, -1000.0f);  // -inf: w = 0
            const float y = fast_exp2(d);
            z += y;
            tt = __builtin_fmaf(y, d, tt);
          }
        }
      };
      if (p.tame)
        sum(std::false_type{});
      else
        sum(std::true_type{});
      const float off = __builtin_fmaf(m, kLog2e, -c), f = fast_exp2(-off);
      tt = f * kLn2 * (tt - off * z);
      z *= f;
    }
    if (m == kNegInf) z = tt = 0.0f;
    if (RANK && given && __any(m >= xt)) {  // else no logit of this wave is before t
      p.unpack_again();
#pragma unroll
      for (int s = 0; s < S; ++s) {
        if (s >= p.used) break;
        const int at = p.at(s);
        const float over = at + VE <= t ? below : xt;
        if (!__any((t >= at && t < at + VE) || at < p.want(s) || p.want(s) + VE > a.V || xt == kNegInf)) {
#pragma unroll
          for (int e = 0; e < VE; ++e) before += __popcll(__ballot(p.x(s, e) > over));
        } else {  // one by one
#pragma unroll
          for (int e = 0; e < VE; ++e)
            before += __popcll(__ballot(p.real(s, e) && (p.x(s, e) > xt || (p.x(s, e) == xt && at + e < t))));
        }
      }
    }

    const State wave = wave_join(State{m, z, tt, before});
    if (lane == 0) joined[sub][w] = wave;

    if constexpr (TOP) {
      const int K = a.K;
      float over = 0.0f;  // logits over it are listed
      bool few = false;   // -inf may be among the first K
      unsigned cut = 0;
      if (held == K) {  // those of the sub-chunks before stand before their equals here
        over = key_value(first[K - 1]);
      } else {
        // K logits at or above the cut: ceil(K / 4) thread maxima in each wave, or K in one
        const unsigned mine = has ? ordered(m + 0.0f) : 0u;  // 0: nothing
        const int r4 = (K + kNW - 1) / kNW;
        unsigned c4 = 0, cK = 0;  // the r4-th and the K-th largest of the wave's, cut to the high bits
#pragma unroll 1
        for (unsigned bit = 1u << 31; bit >= 1u << kCutBits<TI>; bit >>= 1) {
          if (__popcll(__ballot(mine >= (c4 | bit))) >= r4) c4 |= bit;
          if (__popcll(__ballot(mine >= (cK | bit))) >= K) cK |= bit;
        }
        if (lane == 0) {
          sh.cut[0][w] = c4;
          sh.cut[1][w] = cK;
        }
        __syncthreads();
        unsigned low = 0xffffffffu, high = 0;
#pragma unroll
        for (int k = 0; k < kNW; ++k) {
          low = min(low, sh.cut[0][k]);
          high = max(high, sh.cut[1][k]);
        }
        cut = max(low, high);
        few = cut <= kOrderedNegInf;
        if (!few) over = number_below(unordered(cut));
      }
      p.unpack_again();
      int listed = 0;  // of this wave
      auto list = [&](bool take, float v, int i) __attribute__((always_inline)) {
        const unsigned long long who = __ballot(take);
        if (who) {
          const int at = listed + (int)__builtin_amdgcn_mbcnt_hi((unsigned)(who >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)who, 0));
          if (take && at < kCap) sh.wave[w][at] = key_of(v, i);
          listed += __popcll(who);
        }
      };
      // Places left out are -kWild in a tame wave, -inf in others: under the bound, but where a mask of a finite value is
      // the bound (-2^119 and less) or -inf may be listed.
      if (few || (p.tame && over < -kWild)) {
        const unsigned least = few ? cut : 0u;  // a tame wave's logits are all over such a bound
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
          for (int e = 0; e < VE; ++e)
            list(p.real(s, e) && ordered(p.x(s, e) + 0.0f) >= least, p.x(s, e), p.at(s) + e);
      } else if (__any(m > over)) {
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
          for (int e = 0; e < VE; ++e) list(p.x(s, e) > over, p.x(s, e), p.at(s) + e);
      }
      if (lane == 0) sh.count[w] = listed;
      if (tid < held) sh.held[tid] = first[tid];
      __syncthreads();
      bool full = false;
      int count = 0;
#pragma unroll
      for (int k = 0; k < kNW; ++k) {
        full |= sh.count[k] > kCap;
        count += sh.count[k];
      }
      if (full) {
        // Too many. The K-th largest value v: bisection of its bits. Then those over it, and of its equals the lowest
        // indices that make K: bisection of an index. Uniform in the workgroup.
        unsigned v = 0;
        int last = 0;  // with the equals before it there are fewer than K, with itself K
        auto taken = [&](int s, int e, unsigned over, unsigned equal, int end) __attribute__((always_inline)) {
          const unsigned o = ordered(p.x(s, e) + 0.0f);
          return p.real(s, e) && (o > over || (o == equal && p.at(s) + e < end));
        };
#pragma unroll 1
        for (int turn = 31; turn >= -22; --turn) {
          // at or over the trial value is over its predecessor, and no equals; then the trial index
          const unsigned trial = turn >= 0 ? v | 1u << turn : v;
          const int end = turn >= 0 ? 0 : last + (1 << (22 + turn));
          p.unpack_again();
          int c = 0;
#pragma unroll
          for (int s = 0; s < S; ++s) {
#pragma unroll
            for (int e = 0; e < VE; ++e) c += __popcll(__ballot(taken(s, e, turn >= 0 ? trial - 1 : v, v, end)));
          }
          __syncthreads();  // total and the counts are read
          if (tid == 0) sh.total = 0;
          __syncthreads();
          if (lane == 0) atomicAdd(&sh.total, c);
          __syncthreads();
          if (turn >= 0) {
            if (sh.total >= K) v = trial;
          } else if (sh.total < K) {
            last = end;
          }
        }
        listed = 0;
#pragma unroll
        for (int s = 0; s < S; ++s) {
#pragma unroll
          for (int e = 0; e < VE; ++e) list(taken(s, e, v, v, last + 1), p.x(s, e), p.at(s) + e);
        }
        if (lane == 0) sh.count[w] = listed;
        count = K;
        __syncthreads();
      }
      if (count) {  // else the K first stay
        first_keys(sh, held, K, first);
        held = min(K, count + held);
      }
      __syncthreads();
    }
  }
  __syncthreads();
  // states of sub-chunks are joined in an order of their own, whoever had them: a row's numbers do not depend on how many
  // rows the call has
  auto of_sub = [&](int i) __attribute__((always_inline)) {
    return join4(joined[i][0], joined[i][1], joined[i][2], joined[i][3]);
  };
  if (parts == 1) {
    if (w > 0) return;
    const State s = fold(of_sub, nsub);
    finish(a, n, s, xt, TOP ? first : nullptr);
    return;
  }
  if (tid < nsub) states[(int64_t)n * all + sub0 + tid] = of_sub(tid);
  if (TOP && tid < a.K) keys[((int64_t)n * parts + part) * a.K + tid] = tid < held ? first[tid] : 0;
}

// One workgroup a row: joins its parts.
template <typename TI>
__global__ __launch_bounds__(kT) void logprobs_join_kernel(LogprobArgs a, int parts, int all, const State* states, const Key* keys) {
  __shared__ Key list[kMaxKeys];
  __shared__ Key first[kLogprobMaxK];
  const int n = blockIdx.x, tid = threadIdx.x;
  const int64_t t = a.tokens[n];
  float xt = kNegInf;
  if (t >= 0 && t < a.V) xt = (float)((const TI*)a.logits)[(int64_t)n * a.sl + t];
  const State s = fold([&](int i) { return states[(int64_t)n * all + i]; }, all);
  if (a.K > 0) {
    const int count = parts * a.K;  // at most kMaxKeys; 0 where a part had fewer, below every key
    for (int i = tid; i < count; i += kT) list[i] = keys[(int64_t)n * count + i];
    __syncthreads();
    const int sub = tid & 3, per = (count + 3) / 4;
    for (int i = tid >> 2; i < (count + 63) / 64 * 64; i += kT / 4) {
      const Key mine = list[min(i, count - 1)];
      int place = keys_over(list + min(sub * per, count), min(per, max(0, count - sub * per)), mine);
      place += moved(place, [](int y) { return dpp_word<0xB1>(y); });
      place += moved(place, [](int y) { return dpp_word<0x4E>(y); });
      if (i < count && sub == 0 && mine && place < a.K) first[place] = mine;
    }
    __syncthreads();
  }
  finish(a, n, s, xt, first);
}

// dlogits of one piece of a row a thread. Rows without a token and an entropy gradient are 0, whatever they
// hold. (To find that out before the row is read costs all others a wait: 623 us for 4096 x 131072 forward and back, 600.)
template <typename TI>
__global__ __launch_bounds__(kT) void logprobs_bwd_kernel(LogprobGradArgs a, int per_row, int slab) {
  constexpr int VE = Logits<TI>::VE;
  const int n = blockIdx.y * slab + blockIdx.x / per_row, c = blockIdx.x % per_row;
  if (n >= a.N) return;
  const TI* row = (const TI*)a.logits + (int64_t)n * a.sl;
  TI* out = (TI*)a.dlogits + (int64_t)n * a.sg;
  const float4 st = *reinterpret_cast<const float4*>(a.stats + 4 * (int64_t)n);
  const float m = st.x, inv_z = st.y, ln_z = st.z, H = st.w;
  const int64_t t = a.tokens[n];
  float g = a.dlogprob && t >= 0 ? a.dlogprob[n] : 0.0f;
  if (t >= a.V) g = __builtin_nanf("");
  const float h = a.dentropy ? a.dentropy[n] : 0.0f;
  const bool top_inf = m == __builtin_inff();
  auto grad = [&](float x, int i) __attribute__((always_inline)) {
    float d = fmaxf(x - m, -1000.0f);  // NaN counts as -inf: weight 0
    if (top_inf) d = x == m ? 0.0f : -1000.0f;
    const float p = fast_exp2(d * kLog2e) * inv_z;
    const float y = -p * __builtin_fmaf(h, d - ln_z + H, g);
    return i == t ? y + g : y;
  };
  const bool nothing = t < 0 && h == 0.0f;
  const int at = (c * kT + threadIdx.x) * VE;
  if (at >= a.V) return;
  if (a.V >= VE) {
    const int i0 = min(at, a.V - VE);  // the last piece ends with the row: what it shares with the one before is the same
    typename Logits<TI>::V raw = *reinterpret_cast<const typename Logits<TI>::V*>(row + i0);
    asm volatile("" : "+v"(raw));  // read before the branch
    if (nothing) {
      *reinterpret_cast<typename Logits<TI>::V*>(out + i0) = typename Logits<TI>::V{};
      return;
    }
    float x[VE];
    Logits<TI>::values(raw, x);
#pragma unroll
    for (int e = 0; e < VE; ++e) x[e] = grad(x[e], i0 + e);
    if constexpr (sizeof(TI) == 4) {
      *reinterpret_cast<typename Logits<TI>::V*>(out + i0) = typename Logits<TI>::V{x[0], x[1], x[2], x[3]};
    } else {
      bf16x8 o;
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = (bf16)x[e];
      *reinterpret_cast<typename Logits<TI>::V*>(out + i0) = __builtin_bit_cast(uintx4, o);
    }
  } else {
    for (int e = at; e < min(at + VE, a.V); ++e) out[e] = (TI)(nothing ? 0.0f : grad(no_nan((float)row[e]), e));
  }
}

// How a row is cut: S pieces of 16 bytes a thread in a sub-chunk, `all` sub-chunks, `subs` of them a workgroup, `parts`
// workgroups.
// With alternatives the first sub-chunk of a workgroup costs most (its bound is found, and the lists are long), so that
// rows enough to fill the chip are not split.
struct Cut {
  int S, all, subs, parts;
};
Cut cut_of(int64_t N, int64_t V, int64_t K, int dtype) {
  const int64_t piece = (int64_t)kT * (dtype == 1 ? 8 : 4);
  const int64_t pieces = (V + piece - 1) / piece;
  Cut c;
  const int64_t n = (pieces + kMaxS - 1) / kMaxS;  // sub-chunks, all of the same size
  c.S = (int)((pieces + n - 1) / n);
  int64_t most = n;
  if (K > 0) most = std::max<int64_t>(1, std::min<int64_t>({n, kMaxKeys / K, kFillGroups / N}));
  c.all = (int)n;
  c.subs = (int)std::min<int64_t>((n + most - 1) / most, kMaxSubs);
  c.parts = (int)((n + c.subs - 1) / c.subs);  // n is at most 683; with K > 0 parts K is at most kMaxKeys
  return c;
}

template <typename TI, int S>
void launch_s(const LogprobArgs& a, const Cut& c, State* states, Key* keys, hipStream_t stream) {
  const dim3 grid((unsigned)((int64_t)a.N * c.parts));
  if (a.K > 0 && a.rank)
    hipLaunchKernelGGL((logprobs_kernel<TI, S, true, true>), grid, dim3(kT), 0, stream, a, c.parts, c.subs, states, keys);
  else if (a.K > 0)
    hipLaunchKernelGGL((logprobs_kernel<TI, S, false, true>), grid, dim3(kT), 0, stream, a, c.parts, c.subs, states, keys);
  else if (a.rank)
    hipLaunchKernelGGL((logprobs_kernel<TI, S, true, false>), grid, dim3(kT), 0, stream, a, c.parts, c.subs, states, keys);
  else
    hipLaunchKernelGGL((logprobs_kernel<TI, S, false, false>), grid, dim3(kT), 0, stream, a, c.parts, c.subs, states, keys);
}
template <typename TI>
hipError_t launch_t(const LogprobArgs& a, const Cut& c, hipStream_t stream) {
  State* states = (State*)a.ws;
  Key* keys = (Key*)(states + (int64_t)a.N * c.all);
  switch (c.S) {
    case 1: launch_s<TI, 1>(a, c, states, keys, stream); break;
    case 2: launch_s<TI, 2>(a, c, states, keys, stream); break;
    case 3: launch_s<TI, 3>(a, c, states, keys, stream); break;
    case 4: launch_s<TI, 4>(a, c, states, keys, stream); break;
    case 5: launch_s<TI, 5>(a, c, states, keys, stream); break;
    default: launch_s<TI, 6>(a, c, states, keys, stream); break;
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || c.parts == 1) return e;
  hipLaunchKernelGGL((logprobs_join_kernel<TI>), dim3((unsigned)a.N), dim3(kT), 0, stream, a, c.parts, c.all, states, keys);
  return hipGetLastError();
}

}  // namespace

size_t logprobs_scratch_bytes(int64_t N, int64_t V, int64_t K, int dtype) {
  const Cut c = cut_of(N, V, K, dtype);
  return c.parts == 1 ? 0 : (size_t)N * ((size_t)c.all * sizeof(State) + (size_t)c.parts * (size_t)K * sizeof(Key));
}
// Fewer rows may be cut into more parts each: enough for any number of rows up to N.
size_t logprobs_workspace_bytes(int64_t N, int64_t V, int64_t K, int dtype) {
  const Cut one = cut_of(1, V, K, dtype), c = cut_of(N, V, K, dtype);
  if (one.parts == 1) return 0;
  const int64_t rows = c.parts == 1 ? std::min<int64_t>(N, kFillGroups) : N;  // more are not split
  return (size_t)rows * ((size_t)one.all * sizeof(State) + (size_t)one.parts * (size_t)K * sizeof(Key));
}

hipError_t launch_logprobs_fwd(const LogprobArgs& a, int dtype, hipStream_t stream) {
  const Cut c = cut_of(a.N, a.V, a.K, dtype);
  return dtype == 1 ? launch_t<bf16>(a, c, stream) : launch_t<float>(a, c, stream);
}

hipError_t launch_logprobs_bwd(const LogprobGradArgs& a, int dtype, hipStream_t stream) {
  const int piece = kT * (dtype == 1 ? 8 : 4), per_row = (a.V + piece - 1) / piece;
  const int slab = std::min(a.N, (1 << 23) / per_row);  // rows: a grid is under 2^32 threads along x
  const dim3 grid((unsigned)(slab * per_row), (unsigned)((a.N + slab - 1) / slab));
  if (dtype == 1)
    hipLaunchKernelGGL((logprobs_bwd_kernel<bf16>), grid, dim3(kT), 0, stream, a, per_row, slab);
  else
    hipLaunchKernelGGL((logprobs_bwd_kernel<float>), grid, dim3(kT), 0, stream, a, per_row, slab);
  return hipGetLastError();
}

}  // namespace rel
