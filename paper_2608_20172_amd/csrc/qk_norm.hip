// RMS norm of every query and key head and the position rotation, in one pass, and
// its gradients.
//
// A row x [D] of a token and head becomes n = x r w, r = (mean x^2 + eps)^(-1/2),
// and its channel pairs turn by the token's angles: y = R n. Backward, with
// g = R^T dy: dw = sum over rows of g x r, dx = r (g w - x r mean(g w x r)).
//
// A group of lanes holds a row, each lane one unit of V channel pairs: V channels of
// one run and the V that they turn with (the other half of the rotated channels, or,
// for pairs side by side and for channels that are not turned, the next V). So both
// members of a pair meet in one lane, the row's sum is one reduction over the
// group, and every channel is read and written once, in pieces of up to 16 bytes on
// any boundary. Cosines and sines of a workgroup's tokens go to LDS once, for all
// heads (the angle in 64-bit turns, so that a long context keeps its fraction).
// Bound by memory.
#include <type_traits>

#include "lanes.h"
#include "tokens.h"

namespace rel {

namespace {

constexpr int kT = 256;
constexpr int kMaxTokens = 8;     // tokens of a workgroup at a time
constexpr int kMaxGroups = 1024;  // workgroups of the backward pass

// N elements (of 2 to 16 bytes in all) on any element boundary, as floats.
template <typename TI, int N>
struct Piece {
  typedef TI V __attribute__((ext_vector_type(N), aligned(sizeof(TI))));
};
template <typename TI, int N>
__device__ __forceinline__ void load_piece(const TI* p, float (&x)[N]) {
  if constexpr (N == 1) {
    x[0] = (float)*p;
  } else if constexpr (sizeof(TI) == 4) {
    const typename Piece<float, N>::V u = *reinterpret_cast<const typename Piece<float, N>::V*>(p);
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = u[e];
  } else {
    typedef unsigned int U __attribute__((ext_vector_type(N / 2), aligned(2)));
    if constexpr (N == 2) {
      typedef unsigned int W __attribute__((aligned(2)));
      const unsigned int u = *reinterpret_cast<const W*>(p);
      x[0] = bf16_lo(u);
      x[1] = bf16_hi(u);
    } else {
      const U u = *reinterpret_cast<const U*>(p);
#pragma unroll
      for (int e = 0; e < N / 2; ++e) {
        x[2 * e] = bf16_lo(u[e]);
        x[2 * e + 1] = bf16_hi(u[e]);
      }
    }
  }
}
template <typename TI, int N>
__device__ __forceinline__ void store_piece(TI* p, const float (&x)[N]) {
  if constexpr (N == 1) {
    *p = (TI)x[0];
  } else if constexpr (sizeof(TI) == 4) {
    typename Piece<float, N>::V u;
#pragma unroll
    for (int e = 0; e < N; ++e) u[e] = x[e];
    *reinterpret_cast<typename Piece<float, N>::V*>(p) = u;
  } else {
    typedef __bf16 B __attribute__((ext_vector_type(N)));
    typedef float F __attribute__((ext_vector_type(N)));
    F f;
#pragma unroll
    for (int e = 0; e < N; ++e) f[e] = x[e];
    const B b = __builtin_convertvector(f, B);
    if constexpr (N == 2) {
      typedef unsigned int W __attribute__((aligned(2)));
      *reinterpret_cast<W*>(p) = __builtin_bit_cast(unsigned int, b);
    } else {
      typedef unsigned int U __attribute__((ext_vector_type(N / 2), aligned(2)));
      typedef unsigned int UA __attribute__((ext_vector_type(N / 2)));
      *reinterpret_cast<U*>(p) = __builtin_bit_cast(UA, b);
    }
  }
}

// Unit u of a row: the first channels of its two runs, and what they are.
struct Unit {
  int a, b;      // first channel of either run
  bool turned;   // the pairs turn; their angles are j0 ..
  int j0;
  bool some, both;  // the unit has channels; its second run has them too (an odd rest has not)
};
template <int V>
__device__ __forceinline__ Unit unit_of(const QkNormArgs& a, int u) {
  Unit x;
  const int ur = a.rope_dim / (2 * V);
  x.turned = u < ur;
  x.j0 = u * V;
  if (x.turned) {
    x.a = a.interleaved ? 2 * u * V : u * V;
    x.b = a.interleaved ? x.a + V : a.rope_dim / 2 + u * V;
  } else {
    x.a = a.rope_dim + 2 * V * (u - ur);
    x.b = x.a + V;
  }
  x.some = x.a < a.D;
  x.both = x.b < a.D;
  return x;
}

template <typename TI, int V>
__device__ __forceinline__ void load_unit(const TI* row, const Unit& u, float (&x)[2 * V]) {
  float p[V], q[V];
#pragma unroll
  for (int e = 0; e < V; ++e) p[e] = q[e] = 0.0f;
  if (u.some) load_piece<TI, V>(row + u.a, p);
  if (u.both) load_piece<TI, V>(row + u.b, q);
#pragma unroll
  for (int e = 0; e < V; ++e) {
    x[e] = p[e];
    x[V + e] = q[e];
  }
}
template <typename TI, int V>
__device__ __forceinline__ void store_unit(TI* row, const Unit& u, const float (&x)[2 * V]) {
  float p[V], q[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    p[e] = x[e];
    q[e] = x[V + e];
  }
  if (u.some) store_piece<TI, V>(row + u.a, p);
  if (u.both) store_piece<TI, V>(row + u.b, q);
}
template <int V>
__device__ __forceinline__ void load_weights(const QkNormArgs& a, const void* w, const Unit& u, float (&x)[2 * V]) {
  if (!w) {
#pragma unroll
    for (int e = 0; e < 2 * V; ++e) x[e] = 1.0f;
  } else if (a.weight_bf16) {
    load_unit<bf16, V>((const bf16*)w, u, x);
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) {
      x[e] = u.some ? ((const float*)w)[u.a + e] : 0.0f;
      x[V + e] = u.both ? ((const float*)w)[u.b + e] : 0.0f;
    }
  }
}

// The members of pair e of a unit: run a's and run b's e-th (HALF), or neighbours.
template <int V, bool INTER>
__device__ __forceinline__ constexpr int first_of(int e) { return INTER && V > 1 ? 2 * e : e; }
template <int V, bool INTER>
__device__ __forceinline__ constexpr int second_of(int e) { return INTER && V > 1 ? 2 * e + 1 : V + e; }

// x turned by the angles whose (cos, sin) stand at cs (BACK: turned back).
template <int V, bool INTER, bool BACK>
__device__ __forceinline__ void turn(float (&x)[2 * V], const float2* cs) {
#pragma unroll
  for (int e = 0; e < V; ++e) {
    const int i = first_of<V, INTER>(e), j = second_of<V, INTER>(e);
    const float2 t = cs[e];
    const float s = BACK ? -t.y : t.y, p = x[i], q = x[j];
    x[i] = p * t.x - q * s;
    x[j] = p * s + q * t.x;
  }
}

// (cos, sin) times the amplitude of the nt tokens from n0 on into cs [nt][rope_dim / 2]; live[n]: position not negative.
__device__ __forceinline__ void token_angles(const QkNormArgs& a, int64_t n0, int nt, float2* cs, int* live) {
  const int half = a.rope_dim >> 1;
  auto position = [&](int n) __attribute__((always_inline)) {
    const int64_t g = n0 + n, b = g / a.T, t = g - b * a.T;
    return a.positions ? a.positions[b * a.position_stride + t] : (int)t;
  };
  if ((int)threadIdx.x < nt) live[threadIdx.x] = position(threadIdx.x) >= 0;
  for (int i = threadIdx.x; i < nt * half; i += kT) {
    const int n = i / half, j = i - n * half;
    const double x = (double)position(n) * a.turns[j];
    float s, c;
    sincospif((float)(2.0 * (x - rint(x))), &s, &c);  // half turns in [-1, 1]
    cs[i] = make_float2(c * a.amplitude, s * a.amplitude);
  }
}

__device__ __forceinline__ int64_t row_at(const Strides& s, int T, int64_t token, int h) {
  const int64_t b = token / T;
  return b * s.b + h * s.h + (token - b * T) * s.t;
}

template <typename TI, int V, int LG, bool INTER>
__global__ __launch_bounds__(kT) void qk_norm_fwd_kernel(QkNormArgs a, int tpw) {
  extern __shared__ float2 cs[];  // [tpw][rope_dim / 2]
  __shared__ int live[kMaxTokens];
  const int64_t n0 = (int64_t)blockIdx.x * tpw;
  const int nt = (int)min((int64_t)tpw, a.tokens - n0);
  token_angles(a, n0, nt, cs, live);
  __syncthreads();
  const int grp = threadIdx.x / LG;
  const Unit u = unit_of<V>(a, threadIdx.x % LG);
  const float inv_d = 1.0f / (float)a.D;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    const NormTensor& s = a.s[which];
    if (s.H == 0) continue;
    float w[2 * V];
    load_weights<V>(a, s.w, u, w);
    const int rows = nt * s.H;
    for (int i0 = 0; i0 < rows; i0 += kT / LG) {  // every lane of a wave reaches the reduction
      const int i = min(i0 + grp, rows - 1), n = i / s.H, h = i - n * s.H;
      float x[2 * V];
      load_unit<TI, V>((const TI*)s.x + row_at(s.sx, a.T, n0 + n, h), u, x);
      if (a.norm) {
        float q = 0.0f;
#pragma unroll
        for (int e = 0; e < 2 * V; ++e) q = __builtin_fmaf(x[e], x[e], q);
        const float r = 1.0f / sqrtf(lane_group_sum<LG>(q) * inv_d + a.eps);
#pragma unroll
        for (int e = 0; e < 2 * V; ++e) x[e] = x[e] * r * w[e];
      }
      if (u.turned) turn<V, INTER, false>(x, cs + n * (a.rope_dim >> 1) + u.j0);
      if (!live[n]) {
#pragma unroll
        for (int e = 0; e < 2 * V; ++e) x[e] = 0.0f;
      }
      if (i0 + grp < rows) store_unit<TI, V>((TI*)s.y + row_at(s.sy, a.T, n0 + n, h), u, x);
    }
  }
}

// A workgroup goes over every gridDim.x-th run of tokens and keeps its sums for the weights in registers: a lane has
// the same channels in every row. At the end the workgroup's groups of lanes meet in LDS in a fixed order.
template <typename TI, int V, int LG, bool INTER>
__global__ __launch_bounds__(kT) void qk_norm_bwd_kernel(QkNormArgs a, int tpw) {
  extern __shared__ float2 cs[];
  __shared__ int live[kMaxTokens];
  __shared__ float sums[kT / LG][2 * V * LG + 1];
  const int grp = threadIdx.x / LG, lane = threadIdx.x % LG;
  const Unit u = unit_of<V>(a, lane);
  const float inv_d = 1.0f / (float)a.D;
  float dw[2][2 * V];
#pragma unroll
  for (int e = 0; e < 2 * V; ++e) dw[0][e] = dw[1][e] = 0.0f;
  for (int64_t n0 = (int64_t)blockIdx.x * tpw; n0 < a.tokens; n0 += (int64_t)gridDim.x * tpw) {
    const int nt = (int)min((int64_t)tpw, a.tokens - n0);
    __syncthreads();  // the angles before are read
    token_angles(a, n0, nt, cs, live);
    __syncthreads();
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      const NormTensor& s = a.s[which];
      if (s.H == 0) continue;
      float w[2 * V];
      load_weights<V>(a, s.w, u, w);
      const int rows = nt * s.H;
      for (int i0 = 0; i0 < rows; i0 += kT / LG) {
        const int i = min(i0 + grp, rows - 1), n = i / s.H, h = i - n * s.H;
        const bool mine = i0 + grp < rows;
        float x[2 * V], g[2 * V];
        load_unit<TI, V>((const TI*)s.x + row_at(s.sx, a.T, n0 + n, h), u, x);
        load_unit<TI, V>((const TI*)s.dy + row_at(s.sdy, a.T, n0 + n, h), u, g);
        if (u.turned) turn<V, INTER, true>(g, cs + n * (a.rope_dim >> 1) + u.j0);
        if (a.norm) {
          float q = 0.0f, d = 0.0f;
#pragma unroll
          for (int e = 0; e < 2 * V; ++e) {
            q = __builtin_fmaf(x[e], x[e], q);
            d = __builtin_fmaf(g[e] * w[e], x[e], d);
          }
          const float r = 1.0f / sqrtf(lane_group_sum<LG>(q) * inv_d + a.eps);
          const float k = lane_group_sum<LG>(d) * r * inv_d;  // mean(g w x r)
          const bool counts = mine && live[n];
#pragma unroll
          for (int e = 0; e < 2 * V; ++e) {
            const float xr = x[e] * r;
            if (counts) dw[which][e] = __builtin_fmaf(g[e], xr, dw[which][e]);
            g[e] = r * (g[e] * w[e] - xr * k);
          }
        }
        if (!live[n]) {
#pragma unroll
          for (int e = 0; e < 2 * V; ++e) g[e] = 0.0f;
        }
        if (mine) store_unit<TI, V>((TI*)s.y + row_at(s.sy, a.T, n0 + n, h), u, g);
      }
    }
  }
  for (int which = 0; which < 2; ++which) {
    if (!a.s[which].dw || a.s[which].H == 0) continue;
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 2 * V; ++e) sums[grp][e * LG + lane] = dw[which][e];
    __syncthreads();
    // thread (e, lane): the sum over the groups, to the channel that it is
    for (int i = threadIdx.x; i < 2 * V * LG; i += kT) {
      const int e = i / LG;
      const Unit v = unit_of<V>(a, i % LG);
      float s = 0.0f;
      for (int x = 0; x < kT / LG; ++x) s += sums[x][i];
      const int ch = e < V ? v.a + e : v.b + e - V;
      if (e < V ? v.some : v.both) a.ws[((int64_t)which * a.groups + blockIdx.x) * a.D + ch] = s;
    }
  }
}

// Channel blockIdx.x of either weight: the workgroups' sums, in a fixed order.
__global__ __launch_bounds__(64) void qk_norm_sum_kernel(QkNormArgs a) {
  const int ch = blockIdx.x, which = blockIdx.y;
  if (!a.s[which].dw) return;
  float s = 0.0f;
  if (a.s[which].H)
    for (int g = threadIdx.x; g < a.groups; g += 64) s += a.ws[((int64_t)which * a.groups + g) * a.D + ch];
  s = lane_group_sum<64>(s);
  if (threadIdx.x == 0) a.s[which].dw[ch] = s;
}

constexpr int lanes_for(int units) { return units <= 1 ? 1 : units <= 2 ? 2 : units <= 4 ? 4 : units <= 8 ? 8 : units <= 16 ? 16 : units <= 32 ? 32 : 64; }

// The widest pieces that the runs of a row are whole numbers of.
int piece_of(const QkNormArgs& a, int widest) {
  for (int v = widest; v > 1; v /= 2)
    if (a.rope_dim % (2 * v) == 0 && (a.D - a.rope_dim) % (2 * v) == 0) return v;
  return 1;
}

int tokens_per_group(const QkNormArgs& a) { return a.tokens >= 4096 ? kMaxTokens : 1; }

struct Forward {
  template <typename TI, int V, int LG, bool INTER>
  static void go(const QkNormArgs& a, hipStream_t stream) {
    const int tpw = tokens_per_group(a);
    hipLaunchKernelGGL((qk_norm_fwd_kernel<TI, V, LG, INTER>), dim3((unsigned)((a.tokens + tpw - 1) / tpw)), dim3(kT),
                       (size_t)tpw * (a.rope_dim / 2) * sizeof(float2), stream, a, tpw);
  }
};
struct Backward {
  template <typename TI, int V, int LG, bool INTER>
  static void go(const QkNormArgs& a, hipStream_t stream) {
    const int tpw = tokens_per_group(a);
    hipLaunchKernelGGL((qk_norm_bwd_kernel<TI, V, LG, INTER>), dim3((unsigned)a.groups), dim3(kT),
                       (size_t)tpw * (a.rope_dim / 2) * sizeof(float2), stream, a, tpw);
  }
};
template <class K, typename TI, int V, int LG>
void by_layout(const QkNormArgs& a, hipStream_t stream) {
  if (a.interleaved)
    K::template go<TI, V, LG, true>(a, stream);
  else
    K::template go<TI, V, LG, false>(a, stream);
}
template <class K, typename TI, int V>
void by_lanes(const QkNormArgs& a, hipStream_t stream) {
  const int units = (a.D + 2 * V - 1) / (2 * V);  // at most 64 / V
  switch (lanes_for(units)) {
    case 1: return by_layout<K, TI, V, 1>(a, stream);
    case 2: return by_layout<K, TI, V, 2>(a, stream);
    case 4: return by_layout<K, TI, V, 4>(a, stream);
    case 8: return by_layout<K, TI, V, 8>(a, stream);
    case 16: if constexpr (V <= 4) return by_layout<K, TI, V, 16>(a, stream); break;
    case 32: if constexpr (V <= 2) return by_layout<K, TI, V, 32>(a, stream); break;
    default: if constexpr (V == 1) return by_layout<K, TI, V, 64>(a, stream); break;
  }
}
template <class K>
hipError_t dispatch(const QkNormArgs& a, int dtype, hipStream_t stream) {
  const int v = piece_of(a, dtype == 1 ? 8 : 4);
  if (dtype == 1) {
    if (v == 8) by_lanes<K, bf16, 8>(a, stream);
    else if (v == 4) by_lanes<K, bf16, 4>(a, stream);
    else if (v == 2) by_lanes<K, bf16, 2>(a, stream);
    else by_lanes<K, bf16, 1>(a, stream);
  } else {
    if (v == 4) by_lanes<K, float, 4>(a, stream);
    else if (v == 2) by_lanes<K, float, 2>(a, stream);
    else by_lanes<K, float, 1>(a, stream);
  }
  return hipGetLastError();
}

}  // namespace

int qk_norm_groups(int64_t tokens) {
  QkNormArgs a{};
  a.tokens = tokens;
  const int tpw = tokens_per_group(a);
  const int64_t n = (tokens + tpw - 1) / tpw;
  return (int)(n < kMaxGroups ? n : kMaxGroups);
}

hipError_t launch_qk_norm_fwd(const QkNormArgs& a, int dtype, hipStream_t stream) {
  return dispatch<Forward>(a, dtype, stream);
}

hipError_t launch_qk_norm_bwd(const QkNormArgs& a, int dtype, hipStream_t stream) {
  if (a.groups) {
    const hipError_t e = dispatch<Backward>(a, dtype, stream);
    if (e != hipSuccess) return e;
  }
  if (a.s[0].dw || a.s[1].dw) hipLaunchKernelGGL(qk_norm_sum_kernel, dim3((unsigned)a.D, 2), dim3(64), 0, stream, a);
  return hipGetLastError();
}

}  // namespace rel
