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
// tokens, its winner is looked up in the order by one sum over the row, and if it
// is not kept, nothing after it is either, and the race is run again over the
// tokens before it. The sum and the next race are one pass.
#include "kernels.h"
#include "serve.h"

namespace rel {

namespace {

constexpr int kSampleT = 1024;
constexpr float kTiny = 1.17549435e-38f;  // random numbers count as at least 2^-126

struct RowParams {
  float T, top_p, min_p;
  int k;        // V where the filter is off
  bool greedy;  // the first token
  bool bad;     // a parameter outside its range: token -1
};
__device__ __forceinline__ RowParams row_params(const SampleArgs& a, int b) {
  RowParams p;
  p.T = a.temperature ? a.temperature[b] : 1.0f;
  p.k = a.top_k ? a.top_k[b] : 0;
  p.top_p = a.top_p ? a.top_p[b] : 1.0f;
  p.min_p = a.min_p ? a.min_p[b] : 0.0f;
  p.bad = !(p.T >= 0.0f) || p.top_p != p.top_p || p.min_p != p.min_p;
  p.greedy = p.T == 0.0f;
  if (p.greedy) p.T = 1.0f;
  if (p.k <= 0 || p.k > a.V) p.k = a.V;
  return p;
}

__device__ __forceinline__ float logit(const bf16* p, int64_t i) { return (float)p[i]; }
__device__ __forceinline__ float logit(const float* p, int64_t i) { return p[i]; }
__device__ __forceinline__ float no_nan(float x) { return x == x ? x : kNegInf; }

// w of logit x: 1 for the largest, also where that is infinite
__device__ __forceinline__ float exponent(float x, float top, float T) { return x == top ? 0.0f : (x - top) / T; }

// The larger of two (value, index) pairs; equal values: the lower index.
struct Best {
  float v;
  int i;
};
__device__ __forceinline__ Best better(Best a, Best b) {
  return b.v > a.v || (b.v == a.v && b.i < a.i) ? b : a;
}
__device__ __forceinline__ Best wave_best(Best x) {
  for (int o = 32; o >= 1; o >>= 1) x = better(x, Best{__shfl_xor(x.v, o, 64), __shfl_xor(x.i, o, 64)});
  return x;
}

template <typename TI>
__global__ __launch_bounds__(kSampleT) void sample_rows_kernel(SampleArgs a) {
  constexpr int NW = kSampleT / 64;
  __shared__ float sv[NW], sm[NW];
  __shared__ int si[NW], sc[NW];
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const TI* x = (const TI*)a.logits + (int64_t)b * a.sl;
  const float* r = a.noise + (int64_t)b * a.sn;
  const RowParams p = row_params(a, b);

  auto block_best = [&](Best v) __attribute__((always_inline)) {
    v = wave_best(v);
    __syncthreads();
    if (lane == 0) {
      sv[w] = v.v;
      si[w] = v.i;
    }
    __syncthreads();
    Best all{sv[0], si[0]};
#pragma unroll
    for (int k = 1; k < NW; ++k) all = better(all, Best{sv[k], si[k]});
    return all;
  };
  auto block_sum = [&](float v) __attribute__((always_inline)) {
    for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
    __syncthreads();
    if (lane == 0) sm[w] = v;
    __syncthreads();
    float s = 0.0f;
#pragma unroll
    for (int k = 0; k < NW; ++k) s += sm[k];
    return s;
  };
  auto block_count = [&](int v) __attribute__((always_inline)) {
    for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
    __syncthreads();
    if (lane == 0) sc[w] = v;
    __syncthreads();
    int s = 0;
#pragma unroll
    for (int k = 0; k < NW; ++k) s += sc[k];
    return s;
  };

  Best top{kNegInf, 0x7fffffff};
  for (int i = tid; i < a.V; i += kSampleT) top = better(top, Best{no_nan(logit(x, i)), i});
  top = block_best(top);
  if (p.bad || top.v == kNegInf) {  // uniform: nothing to choose from
    if (tid == 0) {
      a.tokens[b] = -1;
      if (a.logprob) a.logprob[b] = __builtin_nanf("");
    }
    return;
  }
  float z = 0.0f;
  for (int i = tid; i < a.V; i += kSampleT) z += expf(exponent(no_nan(logit(x, i)), top.v, p.T));
  z = block_sum(z);
  int token = top.i;
  float xt = top.v;
  if (!p.greedy && p.k > 1) {
    const bool all = p.k >= a.V && p.top_p >= 1.0f && p.min_p <= 0.0f;
    float px = kNegInf;   // the pivot: tokens before it are still in the race
    int pi = 0x7fffffff;
    for (;;) {  // ends: every round leaves fewer tokens before the pivot, and the first is always kept
      Best win{-1.0f, 0x7fffffff};
      int n = 0;
      float mass = 0.0f;
      for (int i = tid; i < a.V; i += kSampleT) {
        const float v = no_nan(logit(x, i));
        if (v > px || (v == px && i < pi)) {
          const float wt = expf(exponent(v, top.v, p.T));
          ++n;
          mass += wt;
          if (wt >= p.min_p || i == top.i) win = better(win, Best{wt / fmaxf(r[i], kTiny), i});
        }
      }
      n = block_count(n);
      mass = block_sum(mass);
      win = block_best(win);
      const bool pivot_kept = pi != 0x7fffffff && (pi == top.i || (n < p.k && (p.top_p >= 1.0f || mass < p.top_p * z)));
      if (pivot_kept) {
        token = pi;
        xt = px;
        break;
      }
      pi = win.i;
      px = no_nan(logit(x, pi));
      if (all || pi == top.i) {
        token = pi;
        xt = px;
        break;
      }
    }
  }
  if (tid == 0) {
    a.tokens[b] = token;
    if (a.logprob) a.logprob[b] = exponent(xt, top.v, p.T) - logf(z);
  }
}

}  // namespace

size_t sample_workspace_bytes(int64_t B, int64_t V) { return 0; }

hipError_t launch_sample(const SampleArgs& a, int dtype, hipStream_t stream) {
  if (dtype == 1)
    hipLaunchKernelGGL((sample_rows_kernel<bf16>), dim3((unsigned)a.B), dim3(kSampleT), 0, stream, a);
  else
    hipLaunchKernelGGL((sample_rows_kernel<float>), dim3((unsigned)a.B), dim3(kSampleT), 0, stream, a);
  return hipGetLastError();
}

}  // namespace rel
