// Log-probabilities of given tokens, with entropy, rank and the likeliest
// alternatives, and the gradient by the logits.
//
// With m = max x, w_i = exp(x_i - m), Z = sum w, T = sum w_i (x_i - m):
//   log p_t = x_t - m - ln Z,  entropy = ln Z - T / Z,
//   rank = how many x_i are over x_t, or equal to it at a lower index.
// All four come from one pass over the row: a thread holds S pieces of 16 bytes in
// registers, takes its own maximum, sums against it, and states (m, Z, T) join as
//   m = max, Z = Z_1 a_1 + Z_2 a_2, T = a_1 (T_1 + (m_1 - m) Z_1) + ..., a = exp(m_1 - m).
// A row is cut into chunks of 256 S such pieces, a workgroup each; a second kernel
// joins the chunks of rows that have several.
// Alternatives: a bound tau that at least K of a chunk's logits reach comes from the
// threads' maxima; what reaches it (some more than K) is listed in LDS, and an
// entry's place is the number of entries before it. Ties at the bound may be many
// (flat rows, bf16): then those of the lowest indices are found by bisection.
// Bounds: the read of the logits, and close to it the vector unit (10 instructions a
// logit). The backward pass reads and writes once: memory.
#include <algorithm>

#include "logits.h"
#include "tokens.h"

namespace rel {

namespace {

constexpr int kT = 256;
constexpr int kNW = kT / 64;
constexpr int kCap = 2048;       // listed logits of a chunk
constexpr int kMaxParts = 64;    // workgroups of a row
constexpr int kMaxKeys = 512;    // keys of a row's parts
constexpr unsigned kOrderedNegInf = 0x007fffffu;  // ordered(-inf)

// What a workgroup leaves of its part of a row.
struct State {
  float m, z, t;  // maximum, sum of w, sum of w (x - m); m = -inf: nothing above it
  int before;     // logits before the given token
};
__device__ __forceinline__ State join(State a, State b) {
  const float m = fmaxf(a.m, b.m);
  // 0, not NaN, for what lies infinitely below, and for equal infinities
  const float da = a.m == m ? 0.0f : fmaxf(a.m - m, -1000.0f), db = b.m == m ? 0.0f : fmaxf(b.m - m, -1000.0f);
  const float wa = fast_exp2(da * kLog2e), wb = fast_exp2(db * kLog2e);
  return State{m, a.z * wa + b.z * wb, wa * (a.t + da * a.z) + wb * (b.t + db * b.z), a.before + b.before};
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
    const float lp = none || t >= a.V ? nan : t < 0 ? 0.0f : (xt == s.m ? 0.0f : xt - s.m) - ln_z;
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

// The K largest of the n keys in list into out, in order. n >= K.
__device__ __forceinline__ void first_keys(const Key* list, int n, int K, Key* out) {
  for (int i = threadIdx.x; i < n; i += kT) {
    const Key mine = list[i];
    int place = 0;
    for (int j = 0; j < n; ++j) place += list[j] > mine;
    if (place < K) out[place] = mine;
  }
}

struct TopShared {
  Key list[kCap + kLogprobMaxK];
  unsigned cut[2][kNW];
  int count, total;
};

// Part blockIdx.x % parts of row blockIdx.x / parts: sub-chunks of kT S pieces, one after another.
template <typename TI, int S, bool RANK, bool TOP>
__global__ __launch_bounds__(kT) void logprobs_kernel(LogprobArgs a, int parts, int subs, State* states, Key* keys) {
  constexpr int VE = Logits<TI>::VE, CH = kT * S * VE;
  __shared__ State joined[kNW];
  __shared__ TopShared sh;               // TOP
  __shared__ Key first[kLogprobMaxK];    // TOP: the K first so far
  const int part = blockIdx.x % parts, n = blockIdx.x / parts;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const TI* row = (const TI*)a.logits + (int64_t)n * a.sl;
  const int64_t t64 = a.tokens[n];
  const bool given = t64 >= 0 && t64 < a.V;
  const int t = given ? (int)t64 : -1;
  float xt = kNegInf;
  if (given) xt = no_nan((float)row[t]);
  // x is before t: x > xt, or x >= xt at a lower index; x >= xt is x > the number below xt (below 0: past -0)
  float below = xt;
  if (RANK && given && xt > kNegInf) below = unordered(ordered(xt + 0.0f) - (xt == 0.0f ? 2 : 1));
  State own{kNegInf, 0.0f, 0.0f, 0};
  int held = 0;  // keys in first
  const int c0 = part * subs * CH, c1 = min(c0 + subs * CH, (a.V + CH - 1) / CH * CH);
  for (int base = c0; base < c1; base += CH) {
    float x[S][VE];
    int at[S];
#pragma unroll
    for (int s = 0; s < S; ++s) at[s] = base + (s * kT + tid) * VE;
    load_runs<TI, S>(row, a.V, at, x);
    float m = kNegInf;
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int e = 0; e < VE; ++e) m = fmaxf(m, x[s][e]);
    State st{m, 0.0f, 0.0f, 0};
    if (__any(m == __builtin_inff())) {  // +inf weighs 1, all below it nothing
#pragma unroll
      for (int s = 0; s < S; ++s)
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          const float d = x[s][e] == m ? 0.0f : fmaxf(x[s][e] - m, -1000.0f), y = fast_exp2(d * kLog2e);
          if (m > kNegInf) {
            st.z += y;
            st.t = __builtin_fmaf(y, d, st.t);
          }
        }
    } else {
#pragma unroll
      for (int s = 0; s < S; ++s)
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          const float d = fmaxf(x[s][e] - m, -1000.0f), y = fast_exp2(d * kLog2e);  // -inf, and NaN of -inf - -inf: 0
          st.z += y;
          st.t = __builtin_fmaf(y, d, st.t);
        }
    }
    if (RANK && given) {
#pragma unroll
      for (int s = 0; s < S; ++s) {
        const int want = base + (s * kT + tid) * VE;
        const bool meets = t >= at[s] && t < at[s] + VE;
        const float over = at[s] + VE <= t ? below : xt;
        int c = 0;
#pragma unroll
        for (int e = 0; e < VE; ++e) c += x[s][e] > over;
        if (__any(meets || (at[s] < want) || xt == kNegInf)) {  // one by one
          c = 0;
#pragma unroll
          for (int e = 0; e < VE; ++e) {
            const int i = at[s] + e;
            c += i >= want && i < a.V && (x[s][e] > xt || (x[s][e] == xt && i < t));
          }
        }
        st.before += c;
      }
    }
    own = join(own, st);

    if constexpr (TOP) {
      const int K = a.K;
      // logits that exist: those of a piece that was moved back to the row's end belong to another one
      auto real = [&](int s, int e) __attribute__((always_inline)) {
        const int i = at[s] + e;
        return i >= base + (s * kT + tid) * VE && i < a.V;
      };
      const bool any_real = base + tid * VE < a.V;
      const unsigned mine = any_real ? ordered(m + 0.0f) : 0u;  // 0: this thread has none
      auto wave_cut = [&](int r) __attribute__((always_inline)) {  // the r-th largest of the wave's, cut to high bits
        unsigned c = 0;
#pragma unroll 1
        for (unsigned bit = 1u << 31; bit >= 1u << 12; bit >>= 1)
          if (__popcll(__ballot(mine >= (c | bit))) >= r) c |= bit;
        return c;
      };
      // K logits at or above it: ceil(K / 4) in each wave, or K in one
      const unsigned c4 = wave_cut((K + kNW - 1) / kNW), cK = wave_cut(K);
      if (lane == 0) {
        sh.cut[0][w] = c4;
        sh.cut[1][w] = cK;
      }
      if (tid == 0) sh.count = 0;
      __syncthreads();
      unsigned low = 0xffffffffu, high = 0;
#pragma unroll
      for (int k = 0; k < kNW; ++k) {
        low = min(low, sh.cut[0][k]);
        high = max(high, sh.cut[1][k]);
      }
      const unsigned cut = max(low, high);
      auto listed = [&](float v) __attribute__((always_inline)) { return ordered(v + 0.0f) >= cut; };
      auto add = [&](float v, int i) __attribute__((always_inline)) {
        const int p = atomicAdd(&sh.count, 1);
        if (p < kCap) sh.list[p] = key_of(v, i);
      };
      if (cut > kOrderedNegInf) {
        const float tau = unordered(cut);
        if (m >= tau) {
#pragma unroll
          for (int s = 0; s < S; ++s)
#pragma unroll
            for (int e = 0; e < VE; ++e)
              if (x[s][e] >= tau) add(x[s][e], at[s] + e);
        }
      } else {  // few above -inf: -inf may be among the first K
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
          for (int e = 0; e < VE; ++e)
            if (real(s, e) && listed(x[s][e])) add(x[s][e], at[s] + e);
      }
      __syncthreads();
      int count = sh.count;
      if (count > kCap) {
        // Too many. The K-th largest value v: bisection of its bits. Then those over it, and of its equals the lowest
        // indices that make K: bisection of an index. Uniform in the workgroup.
        auto counted = [&](auto pred) __attribute__((always_inline)) {
          int c = 0;
#pragma unroll
          for (int s = 0; s < S; ++s)
#pragma unroll
            for (int e = 0; e < VE; ++e) c += real(s, e) && pred(ordered(x[s][e] + 0.0f), at[s] + e);
          c = wave_sum(c);
          __syncthreads();  // total is read
          if (tid == 0) sh.total = 0;
          __syncthreads();
          if (lane == 0) atomicAdd(&sh.total, c);
          __syncthreads();
          return sh.total;
        };
        unsigned v = 0;
#pragma unroll 1
        for (unsigned bit = 1u << 31; bit; bit >>= 1)
          if (counted([&](unsigned o, int) { return o >= (v | bit); }) >= K) v |= bit;
        int last = 0;  // with the equals before it there are fewer than K, with itself K
#pragma unroll 1
        for (int bit = 1 << 21; bit; bit >>= 1)
          if (counted([&](unsigned o, int i) { return o > v || (o == v && i < last + bit); }) < K) last += bit;
        if (tid == 0) sh.count = 0;
        __syncthreads();
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
          for (int e = 0; e < VE; ++e) {
            const unsigned o = ordered(x[s][e] + 0.0f);
            if (real(s, e) && (o > v || (o == v && at[s] + e <= last))) add(x[s][e], at[s] + e);
          }
        __syncthreads();
        count = min(sh.count, kCap);
      }
      if (tid < held) sh.list[count + tid] = first[tid];
      __syncthreads();
      count += held;
      held = min(K, count);
      first_keys(sh.list, count, held, first);
      __syncthreads();
    }
  }
  const State wave = wave_reduce(own, [](State x, State y) { return join(x, y); });
  if (lane == 0) joined[w] = wave;
  __syncthreads();
  State s = joined[0];
#pragma unroll
  for (int k = 1; k < kNW; ++k) s = join(s, joined[k]);
  if (parts == 1) {
    finish(a, n, s, xt, TOP ? first : nullptr);
    return;
  }
  if (tid == 0) states[(int64_t)n * parts + part] = s;
  if (TOP && tid < a.K) keys[((int64_t)n * parts + part) * a.K + tid] = tid < held ? first[tid] : 0;
}

// One workgroup a row: joins its parts.
template <typename TI>
__global__ __launch_bounds__(kT) void logprobs_join_kernel(LogprobArgs a, int parts, const State* states, const Key* keys) {
  __shared__ Key list[kMaxKeys];
  __shared__ Key first[kLogprobMaxK];
  const int n = blockIdx.x, tid = threadIdx.x;
  const int64_t t = a.tokens[n];
  float xt = kNegInf;
  if (t >= 0 && t < a.V) xt = (float)((const TI*)a.logits)[(int64_t)n * a.sl + t];
  State s{kNegInf, 0.0f, 0.0f, 0};
  for (int p = 0; p < parts; ++p) s = join(s, states[(int64_t)n * parts + p]);
  if (a.K > 0) {
    const int count = parts * a.K;  // at most kMaxKeys; 0 where a part had fewer, below every key
    for (int i = tid; i < count; i += kT) list[i] = keys[(int64_t)n * count + i];
    __syncthreads();
    for (int i = tid; i < count; i += kT) {
      const Key mine = list[i];
      int place = 0;
      for (int j = 0; j < count; ++j) place += list[j] > mine;
      if (mine && place < a.K) first[place] = mine;
    }
    __syncthreads();
  }
  finish(a, n, s, xt, first);
}

// dlogits of one piece of a row a thread and turn.
template <typename TI>
__global__ __launch_bounds__(kT) void logprobs_bwd_kernel(LogprobGradArgs a, int per_row) {
  constexpr int VE = Logits<TI>::VE;
  const int n = blockIdx.x / per_row, c = blockIdx.x % per_row;
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
  const int at = (c * kT + threadIdx.x) * VE;
  if (at >= a.V) return;
  if (a.V >= VE) {
    const int i0 = min(at, a.V - VE);  // the last piece ends with the row: what it shares with the one before is the same
    const typename Logits<TI>::V raw = *reinterpret_cast<const typename Logits<TI>::V*>(row + i0);
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
    for (int e = at; e < min(at + VE, a.V); ++e) out[e] = (TI)grad(no_nan((float)row[e]), e);
  }
}

// How a row is cut: S pieces of 16 bytes a thread in a sub-chunk, `subs` sub-chunks a workgroup, `parts` workgroups.
struct Cut {
  int S, subs, parts;
};
Cut cut_of(int64_t V, int64_t K, int dtype) {
  const int64_t piece = (int64_t)kT * (dtype == 1 ? 8 : 4);
  const int64_t pieces = (V + piece - 1) / piece;
  Cut c;
  c.S = pieces <= 1 ? 1 : pieces <= 2 ? 2 : pieces <= 4 ? 4 : 8;
  const int64_t n = (pieces + c.S - 1) / c.S;
  const int64_t most = K > 0 ? std::min<int64_t>(kMaxParts, std::max<int64_t>(1, kMaxKeys / K)) : kMaxParts;
  c.subs = (int)((n + most - 1) / most);
  c.parts = (int)((n + c.subs - 1) / c.subs);
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
  Key* keys = (Key*)(states + (int64_t)a.N * c.parts);
  if (c.S == 1) launch_s<TI, 1>(a, c, states, keys, stream);
  else if (c.S == 2) launch_s<TI, 2>(a, c, states, keys, stream);
  else if (c.S == 4) launch_s<TI, 4>(a, c, states, keys, stream);
  else launch_s<TI, 8>(a, c, states, keys, stream);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || c.parts == 1) return e;
  hipLaunchKernelGGL((logprobs_join_kernel<TI>), dim3((unsigned)a.N), dim3(kT), 0, stream, a, c.parts, states, keys);
  return hipGetLastError();
}

}  // namespace

size_t logprobs_workspace_bytes(int64_t N, int64_t V, int64_t K, int dtype) {
  const Cut c = cut_of(V, K, dtype);
  return c.parts == 1 ? 0 : (size_t)N * c.parts * (sizeof(State) + (size_t)K * sizeof(Key));
}

hipError_t launch_logprobs_fwd(const LogprobArgs& a, int dtype, hipStream_t stream) {
  const Cut c = cut_of(a.V, a.K, dtype);
  return dtype == 1 ? launch_t<bf16>(a, c, stream) : launch_t<float>(a, c, stream);
}

hipError_t launch_logprobs_bwd(const LogprobGradArgs& a, int dtype, hipStream_t stream) {
  const int piece = kT * (dtype == 1 ? 8 : 4), per_row = (a.V + piece - 1) / piece;
  const dim3 grid((unsigned)((int64_t)a.N * per_row));
  if (dtype == 1)
    hipLaunchKernelGGL((logprobs_bwd_kernel<bf16>), grid, dim3(kT), 0, stream, a, per_row);
  else
    hipLaunchKernelGGL((logprobs_bwd_kernel<float>), grid, dim3(kT), 0, stream, a, per_row);
  return hipGetLastError();
}

}  // namespace rel
