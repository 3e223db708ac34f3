// One token of each row of logits: temperature, top-k, top-p and min-p, drawn by
// given exponential variates.
//
// With d_i = (x_i - max x) / T, w_i = exp(d_i) and Z their sum, tokens stand in the
// order of falling x, equal ones by their index. All three filters keep a prefix
// of that order, so the kept set is a prefix too, and whether token i is in it
// needs no sort: i is kept if it is the first, or if fewer than k tokens stand
// before it, they weigh less than top_p Z, and w_i >= min_p. The token drawn is
// the kept one with the largest w_i / r_i (r_i exponential: a race that token i
// wins with probability w_i / sum of the kept w). So the race is run over all
// tokens, its winner is looked up in the order by one sum, and if it is not kept,
// nothing after it is either, and the race is run again over the tokens before
// it. Over a list the sum and the next race are one pass.
//
// Short rows (8192 fp32 logits, 16384 bf16) are held by one workgroup each, in one
// launch. Longer ones are read once, by many workgroups a row (scan): each holds its
// chunk in registers, and leaves the chunk's maximum, its sum of exponentials, and
// for a row without filters the winner of its race. For a row with filters it lists
// its largest logits: all at or above a bound tau that about kTarget tokens of the
// row pass. One workgroup a row (pick) then joins the chunks; the tokens at or above
// the largest tau are all in the lists, and where the filters' bound is reached
// among them, the rounds run over the lists in registers, with r read for those
// tokens alone. Otherwise (flat rows, many equal logits) they run over the row.
// Sums are in fp32 and in an order that the sizes alone give.
//
// Bounds: the reads of the logits for large batches (scan of 256 rows of 131072 in
// fp32, 168 MB with the random numbers of its rows without filters: 51 us, 3.3 TB/s,
// the vector unit busy for 26 of them at some 30 instructions a logit); latency for
// small ones (1 row of 32000: scan 5 us, pick 8: the chunks' summaries, then the
// lists' random numbers, then two to four rounds of 1 us); and for flat rows the one
// workgroup that places a token among 131072 (17 us a time, vector unit). A top_k
// past the lists is such a row, and its chunks have not raced in the scan either:
// top_k 20000 of 1 row of 131072 235 us, top_k 5000 of 32000 70.
#include "kernels.h"
#include "logits.h"
#include "serve.h"

namespace rel {

namespace {

constexpr int kScanT = 256, kPickT = 512;
constexpr int kListCap = 512;  // listed tokens of a chunk
constexpr int kTarget = 2048;  // listed tokens of a row, about
constexpr int kHeld = 12;      // listed tokens that a thread of pick holds
constexpr int kCutBits = 12;   // low bits of the ordered logit that the bound tau leaves out
constexpr float kTiny = 1.17549435e-38f;  // random numbers count as at least 2^-126
constexpr float kFltMax = 3.402823466e+38f;

// What the scan leaves of a chunk.
struct Part {
  float m;       // largest logit, and the first token that has it
  int mi;
  float z;       // sum of exp((x - m) / T)
  float tau;     // all tokens at or above are listed
  int n;         // listed tokens; -1: no list
  int wi;        // winner of the chunk's race (0x7fffffff: not run), its logit and random number
  float wx, wr;
};

struct RowParams {
  float T, top_p, min_p;
  int k;          // V where the filter is off
  bool greedy;    // the first token
  bool bad;       // a parameter outside its range: token -1
  bool filtered;  // some filter may leave tokens out
};
__device__ __forceinline__ RowParams row_params(const SampleArgs& a, int b) {
  RowParams p;
  p.T = a.temperature ? a.temperature[b] : 1.0f;
  p.k = a.top_k ? a.top_k[b] : 0;
  p.top_p = a.top_p ? a.top_p[b] : 1.0f;
  p.min_p = a.min_p ? a.min_p[b] : 0.0f;
  p.bad = !(p.T >= 0.0f) || p.top_p != p.top_p || p.min_p != p.min_p;
  if (p.k <= 0 || p.k > a.V) p.k = a.V;
  p.greedy = p.T == 0.0f || p.k == 1;
  if (p.T == 0.0f) p.T = 1.0f;
  p.filtered = p.k < a.V || p.top_p < 1.0f || p.min_p > 0.0f;
  return p;
}

// The random numbers of such runs; 1 past the end of a row shorter than one.
template <int N, int VE>
__device__ __forceinline__ void load_noise(const float* row, int V, const int (&at)[N], float (&r)[N][VE]) {
  typedef float F4 __attribute__((ext_vector_type(4), aligned(4)));
  if (V >= VE) {
#pragma unroll
    for (int s = 0; s < N; ++s) {
#pragma unroll
      for (int q = 0; q < VE / 4; ++q) {
        const F4 u = *reinterpret_cast<const F4*>(row + at[s] + 4 * q);
#pragma unroll
        for (int e = 0; e < 4; ++e) r[s][4 * q + e] = u[e];
      }
    }
  } else {
#pragma unroll
    for (int s = 0; s < N; ++s) {
#pragma unroll
      for (int e = 0; e < VE; ++e) r[s][e] = at[s] + e < V ? row[at[s] + e] : 1.0f;
    }
  }
}

// exp((x - top) / T) with log2(e) / T as pre (hi + lo), so that the exponent keeps its fp32 accuracy however large.
// pre is 1, or 2^24 for a T under 2^-126 whose log2(e) / T is past fp32.
struct Scale {
  float hi, lo, pre;
};
// A value that all lanes have, in a scalar register.
__device__ __forceinline__ int scalar(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ float scalar(float x) {
  return __builtin_bit_cast(float, scalar(__builtin_bit_cast(int, x)));
}
__device__ __forceinline__ Scale scale_of(float T) {
  const double c = 1.4426950408889634074 / (double)T;
  const double d = c > 1.0e38 ? c * 0x1p-24 : c;
  const float hi = (float)d;
  return Scale{scalar(hi), scalar((float)(d - (double)hi)), scalar(c > 1.0e38 ? 0x1p24f : 1.0f)};
}
// (x - top) pre: with pre = 1 the difference, rounded once. From |top| = 2^100 on pre is left out, since top pre would
// overflow: numbers there differ by 2^76 or not at all, and with such a T the exponent of a difference is out of range
// either way.
__device__ __forceinline__ float below_top(float x, float top, Scale s) {
  const float pre = fabsf(top) < 0x1p100f ? s.pre : 1.0f;
  return __builtin_fmaf(x, pre, -(top * pre));
}
__device__ __forceinline__ float weight(float x, float top, Scale s) {
  const float t = below_top(x, top, s), y = t * s.hi;
  const float e = __builtin_fmaf(t, s.hi, -y) + t * s.lo, p = fast_exp2(y);
  // 1 for the largest, also where that is infinite; 0 for -inf, and where the exponent is past fp32's
  return x == top ? 1.0f : y > -150.0f ? __builtin_fmaf(p, e * kLn2, p) : 0.0f;
}
// The same to the rounding of the exponent (2^-23 of it, either way): for sums of
// many. min and max pass over the NaN of inf - inf (1) and of inf - inf or 0 inf in the exponent (0: x is -inf or
// below +inf).
__device__ __forceinline__ float weight_fast(float x, float top, Scale s) {
  const float t = fminf(below_top(x, top, s), 0.0f);
  return fast_exp2(fmaxf(__builtin_fmaf(t, s.lo, t * s.hi), -1000.0f));
}
__device__ __forceinline__ float race(float w, float r) { return w / fmaxf(r, kTiny); }

constexpr unsigned kLowest = 0x00800000u;  // ordered(-FLT_MAX)

// A token in a race: the larger v wins, equal ones by the lower index. x: its logit.
struct Best {
  float v;
  int i;
  float x;
};
constexpr Best kNobody = {-1.0f, 0x7fffffff, kNegInf};
__device__ __forceinline__ Best better(Best a, Best b) { return b.v > a.v || (b.v == a.v && b.i < a.i) ? b : a; }

__device__ __forceinline__ Best wave_best(Best x) {
  return wave_reduce(x, [](Best a, Best b) { return better(a, b); });
}
// First logit of run v of chunk c of nch: the chunk has every nch-th piece of 128
// bytes (8 runs of 16 bytes), so that tokens that stand together in the
// vocabulary (often those of like frequency) are spread over the chunks.
template <int VE>
__device__ __forceinline__ int run_start(int v, int c, int nch) {
  return (((v >> 3) * nch + c) * 8 + (v & 7)) * VE;
}

// One chunk of one row: S loads of 16 bytes a thread, S * 4 KB in all. Every
// fourth piece goes to a wave, for the same spread.
// The bound tau is the least of the waves' rank-th largest thread maxima (64 a
// wave), so that about 4 rank tokens pass it; where more do than the list holds
// (several large ones in a thread), rank is cut to a quarter and again. A chunk
// whose list weighs less than top_p of it belongs, most likely, to a row whose
// kept tokens are too many for lists: it runs its race here as well, with the
// whole chip, and spares the one workgroup of pick that.
template <typename TI, int S>
__global__ __launch_bounds__(kScanT, 4) void sample_scan_kernel(SampleArgs a, int nch, int rank, int cap, Part* parts,
                                                                float2* lists) {
  constexpr int VE = Logits<TI>::VE, NW = kScanT / 64;
  __shared__ float tops[NW], zs[2][NW], vs[NW];
  __shared__ unsigned cut[2][NW];
  __shared__ int cnt[2][NW];
  __shared__ int first;
  __shared__ unsigned long long winner;
  const int c = blockIdx.x % nch, b = blockIdx.x / nch;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const TI* row = (const TI*)a.logits + (int64_t)b * a.sl;
  const float* noise = a.noise + (int64_t)b * a.sn;
  const RowParams p = row_params(a, b);
  const bool listed = !p.greedy && p.filtered && !p.bad;
  float x[S][VE];
  int at[S];
#pragma unroll
  for (int s = 0; s < S; ++s)
    at[s] = run_start<VE>(s * kScanT + (((lane >> 3) * NW + w) << 3) + (lane & 7), c, nch);
  load_runs<TI, S>(row, a.V, at, x);
  float own = kNegInf;
#pragma unroll
  for (int s = 0; s < S; ++s)
#pragma unroll
    for (int e = 0; e < VE; ++e) own = fmaxf(own, x[s][e]);
  const unsigned mine = ordered(own);
  // the rank-th largest of the wave's maxima, cut to its high bits
  auto wave_cut = [&](int r) __attribute__((always_inline)) {
    unsigned t = 0;
#pragma unroll 1
    for (unsigned bit = 1u << 31; bit >= 1u << kCutBits; bit >>= 1) {
      if (__popcll(__ballot(mine >= (t | bit))) >= r) t |= bit;
    }
    return t;
  };
  const float wtop = wave_max(own);
  const unsigned c0 = listed ? wave_cut(rank) : 0;
  if (lane == 0) {
    tops[w] = wtop;
    cut[0][w] = c0;
  }
  if (tid == 0) {
    first = 0x7fffffff;
    winner = 0;
  }
  __syncthreads();
  float top = tops[0];
#pragma unroll
  for (int k = 1; k < NW; ++k) top = fmaxf(top, tops[k]);
  const Scale sc = scale_of(p.T);
  derive_again(at);
  if (own == top && top > kNegInf) {  // the first token that has it: the least index, whatever the order of arrival
    int i = 0x7fffffff;
#pragma unroll
    for (int s = S - 1; s >= 0; --s)
#pragma unroll
      for (int e = VE - 1; e >= 0; --e)
        if (x[s][e] == top) i = at[s] + e;
    atomicMin(&first, i);
  }
  float tau = 0.0f;
  int total = 0;
  if (listed) {
    int turn = 0;
    for (int r = rank;;) {
      // a wave without so many numbers above -inf has no say; where none has one, all are listed
      unsigned t = 0xffffffffu;
#pragma unroll
      for (int k = 0; k < NW; ++k) t = min(t, cut[turn][k] < kLowest ? 0xffffffffu : cut[turn][k]);
      tau = t == 0xffffffffu ? -kFltMax : unordered(t);
      int n = 0;
#pragma unroll
      for (int s = 0; s < S; ++s)
#pragma unroll
        for (int e = 0; e < VE; ++e) n += x[s][e] >= tau;
      int incl = n;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(incl, o, 64);
        if (lane >= o) incl += y;
      }
      if (lane == 63) cnt[turn][w] = incl;
      __syncthreads();
      total = 0;
      int before = incl - n;
#pragma unroll
      for (int k = 0; k < NW; ++k) {
        if (k < w) before += cnt[turn][k];
        total += cnt[turn][k];
      }
      derive_again(at);
      if (total <= cap) {  // places in the order of (wave, lane, own): the list is the same in every run
        if (n) {
          float2* list = lists + ((int64_t)b * nch + c) * kListCap;
#pragma unroll
          for (int s = 0; s < S; ++s)
#pragma unroll
            for (int e = 0; e < VE; ++e)
              if (x[s][e] >= tau) list[before++] = float2{x[s][e], __builtin_bit_cast(float, at[s] + e)};
        }
        break;
      }
      if (r == 1) {
        total = -1;
        tau = __builtin_inff();
        break;
      }
      r = max(1, r >> 2);
      turn ^= 1;
      const unsigned cn = wave_cut(r);
      if (lane == 0) cut[turn][w] = cn;
      __syncthreads();
    }
  }
  derive_again(at);
  float z = 0.0f, zl = 0.0f;  // the chunk's weight, and that of its listed tokens
#pragma unroll
  for (int s = 0; s < S; ++s)
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      const float wt = weight_fast(x[s][e], top, sc);
      z += wt;
      if (listed) zl += x[s][e] >= tau ? wt : 0.0f;
    }
  z = wave_sum(z);
  zl = wave_sum(zl);
  if (lane == 0) {
    zs[0][w] = z;
    zs[1][w] = zl;
  }
  __syncthreads();
  z = zl = 0.0f;
#pragma unroll
  for (int k = 0; k < NW; ++k) {
    z += zs[0][k];
    zl += zs[1][k];
  }
  const bool open = p.k >= a.V && !(p.top_p < 1.0f && zl >= p.top_p * z) && !(p.min_p > 0.0f && weight(tau, top, sc) < p.min_p);
  const bool racing = top > kNegInf && !p.greedy && !p.bad && (!p.filtered || open);
  if (racing) {
    float v[S][VE], vmax = -1.0f;
    load_noise<S, VE>(noise, a.V, at, v);
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int e = 0; e < VE; ++e) asm volatile("" : "+v"(x[s][e]));
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        v[s][e] = weight_fast(x[s][e], top, sc) * fast_rcp(fmaxf(v[s][e], kTiny));
        vmax = fmaxf(vmax, v[s][e]);
      }
    const float wmax = wave_max(vmax);
    if (lane == 0) vs[w] = wmax;
    __syncthreads();
    float near = vs[0];
#pragma unroll
    for (int k = 1; k < NW; ++k) near = fmaxf(near, vs[k]);
    near *= 1.0f - 3.0e-5f;
    derive_again(at);
    if (vmax >= near) {  // the few that come near the best are compared without the approximations
#pragma unroll
      for (int s = 0; s < S; ++s)
#pragma unroll
        for (int e = 0; e < VE; ++e)
          if (v[s][e] >= near && x[s][e] > kNegInf) {
            const unsigned long long bits = __builtin_bit_cast(unsigned, race(weight(x[s][e], top, sc), noise[at[s] + e]));
            atomicMax(&winner, bits << 32 | (unsigned)(0x7fffffff - (at[s] + e)));
          }
    }
    __syncthreads();
  }
  if (tid == 0) {
    Part part{top, first, z, tau, total, 0x7fffffff, kNegInf, 1.0f};
    if (racing) {
      part.wi = 0x7fffffff - (int)(winner & 0x7fffffff);
      part.wx = no_nan((float)row[part.wi]);
      part.wr = noise[part.wi];
    }
    parts[(int64_t)b * nch + c] = part;
  }
}

// One round over some tokens: how many stand before the pivot, their weight, and the winner of the race among them.
struct Round {
  Best win;
  int n;
  float mass;
  float z;  // a part of Z, where it is still summed
};

// Reductions over a workgroup of NW waves; the two sets of LDS are taken in turn: one barrier each.
template <int NW>
struct Reducer {
  Round (*lds)[NW];
  int lane, w, turn;
  __device__ __forceinline__ Round operator()(Round r) {
    r.win = wave_best(r.win);
    r.n = wave_sum(r.n);
    r.mass = wave_sum(r.mass);
    r.z = wave_sum(r.z);
    if (lane == 0) lds[turn][w] = r;
    __syncthreads();
    r = lds[turn][lane % NW];  // then over the waves, NW lanes to one
    turn ^= 1;
    r.win = group_reduce<NW>(r.win, [](Best a, Best b) { return better(a, b); });
    r.n = group_reduce<NW>(r.n, [](int a, int b) { return a + b; });
    r.mass = group_reduce<NW>(r.mass, [](float a, float b) { return a + b; });
    r.z = group_reduce<NW>(r.z, [](float a, float b) { return a + b; });
    return r;
  }
};

// What the filters of a row come to once its first token and Z are known.
struct Filters {
  Best top;
  float Z, bound, min_p;  // bound: top_p Z
  bool by_p;
  int k;
  // whether a token is kept by those before it (min_p apart); the first token is in any case
  __device__ __forceinline__ bool within(const Round& before) const {
    return before.n < k && (!by_p || before.mass < bound);
  }
  __device__ __forceinline__ bool kept(int i, const Round& before) const { return i == top.i || within(before); }
};
__device__ __forceinline__ Filters filters_of(const RowParams& p, Best top, float Z) {
  return Filters{top, Z, p.top_p * Z, p.min_p, p.top_p < 1.0f, p.k};
}
__device__ __forceinline__ bool stands_before(float x, int i, const Best& pivot) {
  return x > pivot.x || (x == pivot.x && i < pivot.i);
}

// The rounds over listed tokens, H a thread: logits x (-inf: none), indexes, random
// numbers v. All tokens at or above tau are among them. The first round sums Z
// from the threads' parts z as well. False where the kept set may reach past the
// list; else the token.
template <int H, int NW>
__device__ __forceinline__ bool race_listed(const float (&x)[H], const int (&id)[H], float (&v)[H], float tau, float z,
                                            const RowParams& p, Best top, Scale sc, Reducer<NW>& reduce, Filters& f,
                                            Best& token) {
  float wt[H];
#pragma unroll
  for (int k = 0; k < H; ++k) {
    const bool in = x[k] > kNegInf;
    wt[k] = in ? weight(x[k], top.v, sc) : 0.0f;
    v[k] = in && (wt[k] >= p.min_p || id[k] == top.i) ? race(wt[k], v[k]) : -1.0f;
  }
  Best pivot = kNobody;  // only tokens before it are still in the race; at first all
  for (bool all = true;; all = false) {
    Round r{kNobody, 0, 0.0f, all ? z : 0.0f};
#pragma unroll
    for (int k = 0; k < H; ++k) {
      if (x[k] > kNegInf && (all || stands_before(x[k], id[k], pivot))) {
        ++r.n;
        r.mass += wt[k];
        r.win = better(r.win, Best{v[k], id[k], x[k]});
      }
    }
    r = reduce(r);
    if (all) {
      f = filters_of(p, top, r.z);
      // the tokens that are not among these stand after all of them, and weigh less than the bound: do they all fail a
      // filter?
      const bool within = tau <= -kFltMax || r.n >= f.k || (f.by_p && r.mass >= f.bound) ||
                          (f.min_p > 0.0f && weight(tau, top.v, sc) < f.min_p);
      if (!within || r.win.v < 0.0f) return false;
    } else if (f.kept(pivot.i, r)) {
      break;
    }
    pivot = r.win;
    if (pivot.i == top.i) break;
  }
  token = pivot;
  return true;
}

__device__ __forceinline__ void store_token(const SampleArgs& a, int b, const RowParams& p, Best token, float top, float Z) {
  a.tokens[b] = token.i;
  if (a.logprob) a.logprob[b] = (token.x == top ? 0.0f : (token.x - top) / p.T) - logf(Z);
}
__device__ __forceinline__ void store_nothing(const SampleArgs& a, int b) {
  a.tokens[b] = -1;
  if (a.logprob) a.logprob[b] = __builtin_nanf("");
}

// A thread's part of the tokens before the pivot, the whole row being read by
// kPickT threads: one workgroup, so the vector unit bounds it, and the pass is kept
// to what it needs (NaN and -inf compare false, the rare equal ones apart).
template <typename TI>
__device__ __forceinline__ Round place_in_row(const TI* row, int V, int tid, const Best& pivot, float top, Scale sc) {
  constexpr int VE = Logits<TI>::VE, kAhead = 64 / VE, kBlock = kPickT * VE * kAhead;
  Round r{kNobody, 0, 0.0f, 0.0f};
  const float wp = weight_fast(pivot.x, top, sc);
  int i0 = 0;
  for (; i0 + kBlock <= V; i0 += kBlock) {
    typename Logits<TI>::V u[kAhead];
#pragma unroll
    for (int s = 0; s < kAhead; ++s)
      u[s] = *reinterpret_cast<const typename Logits<TI>::V*>(row + i0 + (s * kPickT + tid) * VE);
    bool equal = false;
#pragma unroll
    for (int s = 0; s < kAhead; ++s) {
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        const float y = element(u[s], e), t = fminf(below_top(y, top, sc), 0.0f),
                    w = fast_exp2(__builtin_fmaf(t, sc.lo, t * sc.hi));
        const bool in = y > pivot.x;
        r.n += in;
        r.mass += in ? w : 0.0f;
        equal = equal || y == pivot.x;
      }
    }
    if (equal) {
#pragma unroll
      for (int s = 0; s < kAhead; ++s) {
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          if (element(u[s], e) == pivot.x && i0 + (s * kPickT + tid) * VE + e < pivot.i) {
            ++r.n;
            r.mass += wp;
          }
        }
      }
    }
  }
  if (i0 < V) {
    float y[kAhead][VE];
    int at[kAhead];
#pragma unroll
    for (int s = 0; s < kAhead; ++s) at[s] = i0 + (s * kPickT + tid) * VE;
    load_runs<TI, kAhead>(row, V, at, y);
#pragma unroll
    for (int s = 0; s < kAhead; ++s) {
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        const bool in = stands_before(y[s][e], at[s] + e, pivot);
        r.n += in;
        r.mass += in ? weight_fast(y[s][e], top, sc) : 0.0f;
      }
    }
  }
  return r;
}

// Rounds over a row before the filters' bound itself is looked for. Random numbers that know nothing of the
// logits halve the tokens left in a round, about, and come to the end in a dozen; numbers that fall along the logits'
// order take one token out a round, and there may be 2^22.
constexpr int kRowRounds = 48;

// The winner among the kept tokens, given one that is not: the first place of the order whose token is not kept is found
// by bisection, of the logit (its ordered bits, up to the first token's: is a token kept that has none of its equals
// before it?), then of the index among equals. At most 55 passes over the row.
template <typename TI, int NW>  // NW waves
__device__ __forceinline__ Best race_bounded(const TI* row, const float* noise, int V, int tid, Best out, const RowParams& p,
                                             Scale sc, const Filters& f, Reducer<NW>& reduce) {
  unsigned lo = ordered(out.x), hi = ordered(f.top.v);
  int i0 = 0, i1 = V;
  if (!f.within(Round{kNobody, 0, 0.0f, 0.0f}) || p.min_p > 1.0f) return f.top;  // no other is kept
  for (;;) {
    const bool by_logit = lo < hi, found = !by_logit && i0 >= i1;
    const unsigned u = lo + (hi - lo) / 2;
    const int i = i0 + (i1 - i0) / 2;
    const Best at{0.0f, by_logit ? 0 : found ? i1 : i, unordered(u)};
    Round r{kNobody, 0, 0.0f, 0.0f};
#pragma unroll 8
    for (int j = tid; j < V; j += NW * 64) {
      const float y = no_nan((float)row[j]);
      if (!stands_before(y, j, at)) continue;
      ++r.n;
      r.mass += weight_fast(y, f.top.v, sc);
      if (found) r.win = better(r.win, Best{race(weight(y, f.top.v, sc), noise[j]), j, y});
    }
    r = reduce(r);
    if (found) return r.win;
    const bool in = f.within(r) && weight(at.x, f.top.v, sc) >= p.min_p;
    if (by_logit) {
      if (in)
        hi = u;
      else
        lo = u + 1;
    } else if (in) {
      i0 = i + 1;
    } else {
      i1 = i;
    }
  }
}

// Joins a row's chunks, at most one a thread. `group` threads (a power of two) load a chunk's list,
// kHeld tokens each at most, before it is known how long it is.
template <typename TI>
__global__ __launch_bounds__(kPickT) void sample_pick_kernel(SampleArgs a, int nch, int group, const Part* parts,
                                                             const float2* lists) {
  constexpr int NW = kPickT / 64, VE = Logits<TI>::VE;
  constexpr int kAhead = 32 / VE;  // loads of 16 bytes in flight where the row is read
  __shared__ Round rounds[2][NW];
  __shared__ float taus[NW];
  __shared__ unsigned char stale[kPickT];  // of a chunk: its race is to be run (again)
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const TI* row = (const TI*)a.logits + (int64_t)b * a.sl;
  const float* noise = a.noise + (int64_t)b * a.sn;
  parts += (int64_t)b * nch;
  lists += (int64_t)b * nch * kListCap;
  const int lc = min(tid / group, nch - 1), j0 = tid % group;
  const Part mine = parts[min(tid, nch - 1)];
  const int ln = tid / group < nch ? parts[lc].n : 0;
  const RowParams p = row_params(a, b);
  const bool choose = !p.greedy && p.filtered;
  float x[kHeld];
  int id[kHeld];
  if (choose) {
#pragma unroll
    for (int k = 0; k < kHeld; ++k) {
      const float2 e = lists[(int64_t)lc * kListCap + min(j0 + k * group, kListCap - 1)];
      x[k] = e.x;
      id[k] = __builtin_bit_cast(int, e.y);
    }
  }
  const Scale sc = scale_of(p.T);

  Reducer<NW> reduce{rounds, lane, w, 0};

  // the row's first token, the bound above which all tokens are listed, and whether a chunk has no list (n)
  Round r0{{mine.m, mine.mi, mine.m}, mine.n < 0, 0.0f, 0.0f};
  float tau = mine.tau;
  tau = wave_max(tau);
  if (lane == 0) taus[w] = tau;
  r0 = reduce(r0);
#pragma unroll
  for (int k = 0; k < NW; ++k) tau = fmaxf(tau, taus[k]);
  const Best top = r0.win;
  if (p.bad || top.v == kNegInf) {  // nothing to choose from
    if (tid == 0) store_nothing(a, b);
    return;
  }
  // Z, and the winner of a race over all tokens
  Round r1{kNobody, 0, 0.0f, 0.0f};
  const bool race_all = !p.greedy && !p.filtered;
  if (tid < nch && mine.m > kNegInf) {
    r1.z = mine.z * weight(mine.m, top.v, sc);
    if (race_all && mine.wi != 0x7fffffff) r1.win = Best{race(weight(mine.wx, top.v, sc), mine.wr), mine.wi, mine.wx};
  }
  // the listed tokens that belong to the whole bound
  float v[kHeld];
  if (choose) {
#pragma unroll
    for (int k = 0; k < kHeld; ++k)
      if (j0 + k * group >= ln || !(x[k] >= tau)) x[k] = kNegInf;
#pragma unroll
    for (int k = 0; k < kHeld; ++k) v[k] = x[k] > kNegInf ? noise[id[k]] : 1.0f;
  }
  Best token = top;
  Filters f;
  bool done = false;
  if (choose && r0.n == 0) {
    done = race_listed(x, id, v, tau, r1.z, p, top, sc, reduce, f, token);
  } else {
    r1 = reduce(r1);
    f = filters_of(p, top, r1.z);
    if (race_all) token = r1.win;
  }
  if (choose) {
    if (!done) {
      // The same over the row. A chunk's winner stands until the pivot comes before it: only such chunks race again.
      if (tid < nch) stale[tid] = mine.wi == 0x7fffffff;
      Best champion = kNobody;  // thread c: of chunk c
      if (tid < nch && mine.wi != 0x7fffffff)
        champion = Best{race(weight(mine.wx, top.v, sc), mine.wr), mine.wi, mine.wx};
      Best pivot = kNobody;
      for (int round = 0;; ++round) {
        const bool all = round == 0;
        __syncthreads();
        for (int c = 0; c < nch; ++c) {
          if (!stale[c]) continue;
          Round r{kNobody, 0, 0.0f, 0.0f};
          for (int v0 = 0; run_start<VE>(v0, c, nch) < a.V; v0 += kPickT * kAhead) {
            float y[kAhead][VE], q[kAhead][VE];
            int at[kAhead];
#pragma unroll
            for (int s = 0; s < kAhead; ++s) at[s] = run_start<VE>(v0 + s * kPickT + tid, c, nch);
            load_runs<TI, kAhead>(row, a.V, at, y);
            load_noise<kAhead, VE>(noise, a.V, at, q);
#pragma unroll
            for (int s = 0; s < kAhead; ++s) {
#pragma unroll
              for (int e = 0; e < VE; ++e) {
                const int i = at[s] + e;
                if (y[s][e] > kNegInf && (all || stands_before(y[s][e], i, pivot)))
                  r.win = better(r.win, Best{race(weight(y[s][e], top.v, sc), q[s][e]), i, y[s][e]});
              }
            }
          }
          r = reduce(r);
          if (tid == c) champion = r.win;
        }
        Round r{champion, 0, 0.0f, 0.0f};
        pivot = reduce(r).win;
        if (pivot.i == top.i) break;
        r = place_in_row<TI>(row, a.V, tid, pivot, top.v, sc);
        r = reduce(r);
        if (f.kept(pivot.i, r) && weight(pivot.x, top.v, sc) >= p.min_p) break;
        if (round == kRowRounds) {
          pivot = race_bounded<TI>(row, noise, a.V, tid, pivot, p, sc, f, reduce);
          break;
        }
        if (tid < nch) stale[tid] = champion.i != 0x7fffffff && !stands_before(champion.x, champion.i, pivot);
      }
      token = pivot;
    }
  }
  if (tid == 0) store_token(a, b, p, token, top.v, f.Z);
}

// ---------------------------------------------------------------------------
// A row in one workgroup: up to kRuns runs of 16 bytes a thread, held as they came.
// The same steps as scan and pick, with the list in LDS and no second launch; the
// rounds that a list does not hold run over the registers. Bound by latency: 1 row of
// 8192 in fp32 12 us, 1000 7.7; 256 rows, a quarter of them with top-p alone and half of
// those past the list, 31.
// ---------------------------------------------------------------------------
constexpr int kRowT = 256, kRuns = 8;

template <typename TI>
__global__ __launch_bounds__(kRowT) void sample_row_kernel(SampleArgs a, int rank) {
  constexpr int NT = kRowT, VE = Logits<TI>::VE, NW = NT / 64, H = 8, kCap = NT * H;
  constexpr int kBatch = 32 / VE;  // runs of random numbers in flight
  typedef typename Logits<TI>::V Raw;
  __shared__ Round rounds[2][NW];
  __shared__ unsigned cut[NW];
  __shared__ int cnt[NW];
  __shared__ float2 list[kCap];
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const TI* row = (const TI*)a.logits + (int64_t)b * a.sl;
  const float* noise = a.noise + (int64_t)b * a.sn;
  Reducer<NW> reduce{rounds, lane, w, 0};
  // pieces of 128 bytes to the waves in turn, as in the scan; runs past the row's end are -inf
  Raw x[kRuns];
  int at[kRuns];
#pragma unroll
  for (int s = 0; s < kRuns; ++s) at[s] = (s * NT + (((lane >> 3) * NW + w) << 3) + (lane & 7)) * VE;
  const int nrun = (a.V + NT * VE - 1) / (NT * VE);  // runs that a thread has, at most
  if (a.V >= VE) {
    int want[kRuns];
#pragma unroll
    for (int s = 0; s < kRuns; ++s) {
      want[s] = at[s];
      at[s] = min(at[s], a.V - VE);
      if (s < nrun) x[s] = *reinterpret_cast<const Raw*>(row + at[s]);
    }
#pragma unroll
    for (int s = 0; s < kRuns; ++s) {
#pragma unroll
      for (int e = 0; e < VE; ++e)
        if (s >= nrun || at[s] + e < want[s] || element(x[s], e) != element(x[s], e)) set_lowest(x[s], e);
    }
  } else {
#pragma unroll
    for (int s = 0; s < kRuns; ++s) {
      x[s] = Raw{};
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        set_lowest(x[s], e);
        if (at[s] + e < a.V && row[at[s] + e] == row[at[s] + e]) {
          const float f = (float)row[at[s] + e];
          if constexpr (sizeof(TI) == 4)
            x[s][e] = f;
          else
            x[s][e >> 1] = e & 1 ? (x[s][e >> 1] & 0xffffu) | __builtin_bit_cast(unsigned, f)
                                 : (x[s][e >> 1] & 0xffff0000u) | (__builtin_bit_cast(unsigned, f) >> 16);
        }
      }
    }
  }
  const RowParams p = row_params(a, b);
  const Scale sc = scale_of(p.T);
  const bool choose = !p.greedy && p.filtered;
  auto again = [&]() __attribute__((always_inline)) {
    derive_again(at);
#pragma unroll
    for (int s = 0; s < kRuns; ++s) asm volatile("" : "+v"(x[s]));
  };
  again();
  Round r0{{kNegInf, 0x7fffffff, kNegInf}, 0, 0.0f, 0.0f};
#pragma unroll
  for (int s = 0; s < kRuns; ++s) {
    if (s < nrun) {
#pragma unroll
      for (int e = 0; e < VE; ++e)
        if (element(x[s], e) > r0.win.v) r0.win = Best{element(x[s], e), at[s] + e, element(x[s], e)};
    }
  }
  const unsigned mine = ordered(r0.win.v);
  auto wave_cut = [&](int r) __attribute__((always_inline)) {
    unsigned t = 0;
#pragma unroll 1
    for (unsigned bit = 1u << 31; bit >= 1u << kCutBits; bit >>= 1) {
      if (__popcll(__ballot(mine >= (t | bit))) >= r) t |= bit;
    }
    return t;
  };
  if (choose) {
    const unsigned t = wave_cut(rank);
    if (lane == 0) cut[w] = t;
  }
  const Best top = reduce(r0).win;
  if (p.bad || top.v == kNegInf) {  // nothing to choose from
    if (tid == 0) store_nothing(a, b);
    return;
  }
  again();
  float z = 0.0f;
#pragma unroll
  for (int s = 0; s < kRuns; ++s) {
    if (s < nrun) {
#pragma unroll
      for (int e = 0; e < VE; ++e) z += weight_fast(element(x[s], e), top.v, sc);
    }
  }
  Best token = top;
  Filters f;
  bool done = false, summed = false;
  {
    if (choose) {
      float tau;
      int total;
      for (int r = rank;;) {  // the list, as in the scan
        unsigned t = 0xffffffffu;
#pragma unroll
        for (int k = 0; k < NW; ++k) t = min(t, cut[k] < kLowest ? 0xffffffffu : cut[k]);
        tau = t == 0xffffffffu ? -kFltMax : unordered(t);
        again();
        int n = 0;
#pragma unroll
        for (int s = 0; s < kRuns; ++s) {
          if (s < nrun) {
#pragma unroll
            for (int e = 0; e < VE; ++e) n += element(x[s], e) >= tau;
          }
        }
        int incl = n;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
          const int y = __shfl_up(incl, o, 64);
          if (lane >= o) incl += y;
        }
        if (lane == 63) cnt[w] = incl;
        __syncthreads();
        total = 0;
        int before = incl - n;
#pragma unroll
        for (int k = 0; k < NW; ++k) {
          if (k < w) before += cnt[k];
          total += cnt[k];
        }
        if (total <= kCap) {
          again();
          if (n) {
#pragma unroll
            for (int s = 0; s < kRuns; ++s) {
              if (s < nrun) {
#pragma unroll
                for (int e = 0; e < VE; ++e)
                  if (element(x[s], e) >= tau) list[before++] = float2{element(x[s], e), __builtin_bit_cast(float, at[s] + e)};
              }
            }
          }
          break;
        }
        if (r == 1) break;
        r = max(1, r >> 2);
        const unsigned cn = wave_cut(r);
        if (lane == 0) cut[w] = cn;
        __syncthreads();
      }
      __syncthreads();
      if (total <= kCap) {
        float lx[H], lv[H];
        int id[H];
#pragma unroll
        for (int k = 0; k < H; ++k) {
          const int j = tid + k * NT;
          lx[k] = kNegInf;
          id[k] = 0;
          lv[k] = 1.0f;
          if (j < total) {
            const float2 e = list[j];
            lx[k] = e.x;
            id[k] = __builtin_bit_cast(int, e.y);
            lv[k] = noise[id[k]];
          }
        }
        done = race_listed(lx, id, lv, tau, z, p, top, sc, reduce, f, token);
        summed = true;
      }
    }
    if (!summed) f = filters_of(p, top, reduce(Round{kNobody, 0, 0.0f, z}).z);
    Best pivot = kNobody;
    for (int round = 0; !p.greedy && !done; ++round) {
      const bool all = round == 0;
      Round r{kNobody, 0, 0.0f, 0.0f};
      float near = -1.0f;  // what the approximations put below this does not win
      again();
#pragma unroll
      for (int s0 = 0; s0 < kRuns; s0 += kBatch) {
        if (s0 >= nrun) break;
        int some[kBatch];
        float q[kBatch][VE];
#pragma unroll
        for (int s = 0; s < kBatch; ++s) some[s] = at[s0 + s];
        load_noise<kBatch, VE>(noise, a.V, some, q);
#pragma unroll
        for (int s = 0; s < kBatch; ++s) {
#pragma unroll
          for (int e = 0; e < VE; ++e) {
            const float y = element(x[s0 + s], e), g = weight_fast(y, top.v, sc) * fast_rcp(fmaxf(q[s][e], kTiny));
            if (g >= near && y > kNegInf && (all || stands_before(y, some[s] + e, pivot))) {
              const float wi = weight(y, top.v, sc);
              if (wi >= p.min_p || some[s] + e == top.i) {
                r.win = better(r.win, Best{race(wi, q[s][e]), some[s] + e, y});
                near = fmaxf(near, g * (1.0f - 3.0e-5f));
              }
            }
          }
        }
      }
      pivot = token = reduce(r).win;
      if (!p.filtered || pivot.i == top.i) break;
      again();
      r = Round{kNobody, 0, 0.0f, 0.0f};
#pragma unroll
      for (int s = 0; s < kRuns; ++s) {
        if (s < nrun) {
#pragma unroll
          for (int e = 0; e < VE; ++e) {
            const bool in = stands_before(element(x[s], e), at[s] + e, pivot);
            r.n += in;
            r.mass += in ? weight_fast(element(x[s], e), top.v, sc) : 0.0f;
          }
        }
      }
      if (f.kept(pivot.i, reduce(r))) break;
      if (round == kRowRounds) {
        token = race_bounded<TI>(row, noise, a.V, tid, pivot, p, sc, f, reduce);
        break;
      }
    }
  }
  if (tid == 0) store_token(a, b, p, token, top.v, f.Z);
}

// How a batch is cut: chunks of 8192 logits (32 a thread of the scan); 2048 where
// these would be few, so that more of the chip reads (scan and pick together, fp32:
// 1 row of 131072 15.7 us in 16 chunks, 13.5 in 64; 24 rows 18.6 and 18.0; 64 rows of
// 32000, 256 chunks, 15.4 and 16.1).
constexpr int kChunk = 8192, kFineChunk = 2048;
static_assert(kSampleMaxV / kChunk <= kPickT, "a chunk a thread of pick");
struct Cut {
  bool fine;
  int nch, rank, group, cap;
};
Cut cut_of(int64_t B, int64_t V) {
  Cut c;
  const int64_t big = (V + kChunk - 1) / kChunk;
  c.fine = B * big < 256 && V <= kFineChunk * 256;
  c.nch = (int)(c.fine ? (V + kFineChunk - 1) / kFineChunk : big);
  c.rank = kTarget / (4 * c.nch);
  c.rank = c.rank < 1 ? 1 : c.rank > 40 ? 40 : c.rank;
  int pow2 = 1;
  while (pow2 < c.nch) pow2 *= 2;
  c.group = kPickT / pow2;
  c.cap = c.group * kHeld < kListCap ? c.group * kHeld : kListCap;
  return c;
}

// The largest row that one workgroup takes: kRowT threads of kRuns runs. (Four times that, with 1024 threads, is
// slower than scan and pick: 17.6 against 14.7 us for 32000 logits in fp32, 33 against 24 for 64 rows of 50257 in bf16.)
int64_t row_limit(int dtype) { return (int64_t)kRowT * kRuns * (dtype == 1 ? 8 : 4); }

template <typename TI>
hipError_t launch_row(const SampleArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL((sample_row_kernel<TI>), dim3((unsigned)a.B), dim3(kRowT), 0, stream, a, 40);
  return hipGetLastError();
}

template <typename TI>
hipError_t launch_t(const SampleArgs& a, hipStream_t stream) {
  const Cut c = cut_of(a.B, a.V);
  Part* parts = (Part*)a.ws;
  float2* lists = (float2*)(parts + (((int64_t)a.B * c.nch + 7) & ~7LL));
  const dim3 grid((unsigned)((int64_t)a.B * c.nch));
  constexpr int full = 32 / Logits<TI>::VE, quarter = 8 / Logits<TI>::VE;
  if (c.fine)
    hipLaunchKernelGGL((sample_scan_kernel<TI, quarter>), grid, dim3(kScanT), 0, stream, a, c.nch, c.rank, c.cap, parts, lists);
  else
    hipLaunchKernelGGL((sample_scan_kernel<TI, full>), grid, dim3(kScanT), 0, stream, a, c.nch, c.rank, c.cap, parts, lists);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((sample_pick_kernel<TI>), dim3((unsigned)a.B), dim3(kPickT), 0, stream, a, c.nch, c.group, parts, lists);
  return hipGetLastError();
}

}  // namespace

size_t sample_workspace_bytes(int64_t B, int64_t V, int dtype) {
  if (V <= row_limit(dtype)) return 0;
  const Cut c = cut_of(B, V);
  const size_t n = (size_t)B * (size_t)c.nch;
  return ((n + 7) & ~(size_t)7) * sizeof(Part) + n * kListCap * sizeof(float2);
}

hipError_t launch_sample(const SampleArgs& a, int dtype, hipStream_t stream) {
  if (a.V <= row_limit(dtype)) return dtype == 1 ? launch_row<bf16>(a, stream) : launch_row<float>(a, stream);
  return dtype == 1 ? launch_t<bf16>(a, stream) : launch_t<float>(a, stream);
}

}  // namespace rel
