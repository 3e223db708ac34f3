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
// heads of a tensor (the angle in 64-bit turns, so that a long context keeps its
// fraction), while the first rows are read.
// Bound by memory. 8 x 2048 tokens, 24 heads x 64 in bf16: forward (101 MB) 24 us, 4.2
// TB/s, backward (151 MB) 34, 4.5; 16384 x 20 heads x 128 36 and 53; fp32, 4 x 4096 x 16 x
// 64 24 (5.7 TB/s) and 38. 8 tokens a workgroup 26 and 42 of the first. One workgroup for
// both tensors, without rows read ahead, 25 and 59: the sums for both weights take 32
// registers, and rows came one after another. Widths whose runs are not whole pieces
// of 16 bytes pay for it: 60 (pieces of 4 bytes) 2.2 TB/s, 80 (five of eight lanes) 3.2.
#include <type_traits>

#include "lanes.h"
#include "tokens.h"

namespace rel {

namespace {

constexpr int kT = 256;
constexpr int kMaxTokens = 16;   // tokens of a workgroup at a time
constexpr int kMaxGroups = 512;  // workgroups of the backward pass a tensor: the two fill the chip once

// N elements (2 to 16 bytes) on any element boundary: as they are read, so that loads are in flight together, and as
// floats.
template <typename TI, int N>
struct Piece;
template <int N>
struct Piece<float, N> {
  typedef float V __attribute__((ext_vector_type(N), aligned(4)));
  static __device__ __forceinline__ void values(const V& u, float* x) {
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = u[e];
  }
  static __device__ __forceinline__ V from(const float* x) {
    V u;
#pragma unroll
    for (int e = 0; e < N; ++e) u[e] = x[e];
    return u;
  }
};
template <>
struct Piece<float, 1> {
  typedef float V;
  static __device__ __forceinline__ void values(const V& u, float* x) { x[0] = u; }
  static __device__ __forceinline__ V from(const float* x) { return x[0]; }
};
template <int N>
struct Piece<bf16, N> {
  typedef unsigned int V __attribute__((ext_vector_type(N / 2), aligned(2)));
  static __device__ __forceinline__ void values(const V& u, float* x) {
#pragma unroll
    for (int e = 0; e < N / 2; ++e) {
      x[2 * e] = bf16_lo(u[e]);
      x[2 * e + 1] = bf16_hi(u[e]);
    }
  }
  static __device__ __forceinline__ V from(const float* x) {
    typedef __bf16 B __attribute__((ext_vector_type(N)));
    typedef float F __attribute__((ext_vector_type(N)));
    typedef unsigned int U __attribute__((ext_vector_type(N / 2)));
    F f;
#pragma unroll
    for (int e = 0; e < N; ++e) f[e] = x[e];
    return __builtin_bit_cast(U, __builtin_convertvector(f, B));
  }
};
template <>
struct Piece<bf16, 2> {
  typedef unsigned int V __attribute__((aligned(2)));
  static __device__ __forceinline__ void values(const V& u, float* x) {
    x[0] = bf16_lo(u);
    x[1] = bf16_hi(u);
  }
  static __device__ __forceinline__ V from(const float* x) {
    typedef __bf16 B __attribute__((ext_vector_type(2)));
    typedef float F __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(unsigned int, __builtin_convertvector(F{x[0], x[1]}, B));
  }
};
template <>
struct Piece<bf16, 1> {
  typedef bf16 V;
  static __device__ __forceinline__ void values(const V& u, float* x) { x[0] = (float)u; }
  static __device__ __forceinline__ V from(const float* x) { return (bf16)x[0]; }
};

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

// A unit of a row, as it is read.
template <typename TI, int V>
struct RawUnit {
  typename Piece<TI, V>::V p, q;
  __device__ __forceinline__ void load(const TI* row, const Unit& u) {
    p = q = typename Piece<TI, V>::V{};
    if (u.some) p = *reinterpret_cast<const typename Piece<TI, V>::V*>(row + u.a);
    if (u.both) q = *reinterpret_cast<const typename Piece<TI, V>::V*>(row + u.b);
  }
  __device__ __forceinline__ void values(float (&x)[2 * V]) const {
    Piece<TI, V>::values(p, x);
    Piece<TI, V>::values(q, x + V);
  }
};
template <typename TI, int V>
__device__ __forceinline__ void store_unit(TI* row, const Unit& u, const float (&x)[2 * V]) {
  if (u.some) *reinterpret_cast<typename Piece<TI, V>::V*>(row + u.a) = Piece<TI, V>::from(x);
  if (u.both) *reinterpret_cast<typename Piece<TI, V>::V*>(row + u.b) = Piece<TI, V>::from(x + V);
}
template <int V>
__device__ __forceinline__ void load_weights(const QkNormArgs& a, const void* w, const Unit& u, float (&x)[2 * V]) {
  if (!w) {
#pragma unroll
    for (int e = 0; e < 2 * V; ++e) x[e] = 1.0f;
  } else if (a.weight_bf16) {
    RawUnit<bf16, V> r;
    r.load((const bf16*)w, u);
    r.values(x);
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

// The rows of one tensor and up to tpw tokens from n0 on, kT / LG at a time. The first rows are on their way while the
// angles are formed, the next while one is worked on.
template <int LG>
struct Rows {
  int64_t n0;
  int nt, H, rows, grp;
  __device__ __forceinline__ Rows(const QkNormArgs& a, const NormTensor& s, int64_t first, int tpw)
      : n0(first), nt((int)min((int64_t)tpw, a.tokens - first)), H(s.H), rows(nt * s.H), grp(threadIdx.x / LG) {}
  // token and head of row i0 + grp (the last row again behind it: every lane of a wave reaches the reductions)
  __device__ __forceinline__ int token(int i0) const { return min(i0 + grp, rows - 1) / H; }
  __device__ __forceinline__ int64_t at(const QkNormArgs& a, const Strides& s, int i0) const {
    const int i = min(i0 + grp, rows - 1), n = i / H;
    return row_at(s, a.T, n0 + n, i - n * H);
  }
  __device__ __forceinline__ bool mine(int i0) const { return i0 + grp < rows; }
};

template <typename TI, int V, int LG, bool INTER>
__global__ __launch_bounds__(kT) void qk_norm_fwd_kernel(QkNormArgs a, int tpw, int first_k) {
  extern __shared__ float2 cs[];  // [tpw][rope_dim / 2]
  __shared__ int live[kMaxTokens];
  const bool second = (int)blockIdx.x >= first_k;
  const NormTensor s = a.s[second];
  const Unit u = unit_of<V>(a, threadIdx.x % LG);
  const float inv_d = 1.0f / (float)a.D;
  const Rows<LG> r(a, s, (int64_t)(blockIdx.x - (second ? first_k : 0)) * tpw, tpw);
  RawUnit<TI, V> next;
  next.load((const TI*)s.x + r.at(a, s.sx, 0), u);
  float w[2 * V];
  load_weights<V>(a, s.w, u, w);
  token_angles(a, r.n0, r.nt, cs, live);
  __syncthreads();
  for (int i0 = 0; i0 < r.rows; i0 += kT / LG) {
    float x[2 * V];
    next.values(x);
    if (i0 + kT / LG < r.rows) next.load((const TI*)s.x + r.at(a, s.sx, i0 + kT / LG), u);
    const int n = r.token(i0);
    if (a.norm) {
      float q = 0.0f;
#pragma unroll
      for (int e = 0; e < 2 * V; ++e) q = __builtin_fmaf(x[e], x[e], q);
      const float c = 1.0f / sqrtf(lane_group_sum<LG>(q) * inv_d + a.eps);
#pragma unroll
      for (int e = 0; e < 2 * V; ++e) x[e] = x[e] * c * w[e];
    }
    if (u.turned) turn<V, INTER, false>(x, cs + n * (a.rope_dim >> 1) + u.j0);
    if (!live[n]) {
#pragma unroll
      for (int e = 0; e < 2 * V; ++e) x[e] = 0.0f;
    }
    if (r.mine(i0)) store_unit<TI, V>((TI*)s.y + r.at(a, s.sy, i0), u, x);
  }
}

// A workgroup goes over every so-many-th run of a tensor's tokens and keeps its sums for the weights in registers: a
// lane has the same channels in every row. At the end the workgroup's groups of lanes meet in LDS in a fixed order.
template <typename TI, int V, int LG, bool INTER>
__global__ __launch_bounds__(kT) void qk_norm_bwd_kernel(QkNormArgs a, int tpw) {
  extern __shared__ float2 cs[];
  __shared__ int live[kMaxTokens];
  __shared__ float sums[kT / LG][2 * V * LG + 1];
  const bool second = (int)blockIdx.x >= a.groups[0];
  const int group = blockIdx.x - (second ? a.groups[0] : 0), groups = a.groups[second];
  const NormTensor s = a.s[second];
  const int grp = threadIdx.x / LG, lane = threadIdx.x % LG;
  const Unit u = unit_of<V>(a, lane);
  const float inv_d = 1.0f / (float)a.D;
  float w[2 * V], dw[2 * V];
  load_weights<V>(a, s.w, u, w);
#pragma unroll
  for (int e = 0; e < 2 * V; ++e) dw[e] = 0.0f;
  for (int64_t n0 = (int64_t)group * tpw; n0 < a.tokens; n0 += (int64_t)groups * tpw) {
    const Rows<LG> r(a, s, n0, tpw);
    RawUnit<TI, V> xn, gn;
    xn.load((const TI*)s.x + r.at(a, s.sx, 0), u);
    gn.load((const TI*)s.dy + r.at(a, s.sdy, 0), u);
    __syncthreads();  // the angles before are read
    token_angles(a, n0, r.nt, cs, live);
    __syncthreads();
    for (int i0 = 0; i0 < r.rows; i0 += kT / LG) {
      float x[2 * V], g[2 * V];
      xn.values(x);
      gn.values(g);
      if (i0 + kT / LG < r.rows) {
        xn.load((const TI*)s.x + r.at(a, s.sx, i0 + kT / LG), u);
        gn.load((const TI*)s.dy + r.at(a, s.sdy, i0 + kT / LG), u);
      }
      const int n = r.token(i0);
      if (u.turned) turn<V, INTER, true>(g, cs + n * (a.rope_dim >> 1) + u.j0);
      const bool mine = r.mine(i0);
      if (a.norm) {
        float q = 0.0f, d = 0.0f;
#pragma unroll
        for (int e = 0; e < 2 * V; ++e) {
          q = __builtin_fmaf(x[e], x[e], q);
          d = __builtin_fmaf(g[e] * w[e], x[e], d);
        }
        const float c = 1.0f / sqrtf(lane_group_sum<LG>(q) * inv_d + a.eps);
        const float k = lane_group_sum<LG>(d) * c * inv_d;  // mean(g w x c)
        const bool counts = mine && live[n];
#pragma unroll
        for (int e = 0; e < 2 * V; ++e) {
          const float xc = x[e] * c;
          if (counts) dw[e] = __builtin_fmaf(g[e], xc, dw[e]);
          g[e] = c * (g[e] * w[e] - xc * k);
        }
      }
      if (!live[n]) {
#pragma unroll
        for (int e = 0; e < 2 * V; ++e) g[e] = 0.0f;
      }
      if (mine) store_unit<TI, V>((TI*)s.y + r.at(a, s.sy, i0), u, g);
    }
  }
  if (!s.dw) return;
#pragma unroll
  for (int e = 0; e < 2 * V; ++e) sums[grp][e * LG + lane] = dw[e];
  __syncthreads();
  // thread (e, lane): the sum over the groups, to the channel that it is
  float* part = a.ws + (second ? (int64_t)a.groups[0] * a.D : 0);  // [D][groups]
  for (int i = threadIdx.x; i < 2 * V * LG; i += kT) {
    const int e = i / LG;
    const Unit v = unit_of<V>(a, i % LG);
    float t = 0.0f;
    for (int x = 0; x < kT / LG; ++x) t += sums[x][i];
    const int ch = e < V ? v.a + e : v.b + e - V;
    if (e < V ? v.some : v.both) part[(int64_t)ch * groups + group] = t;
  }
}

// Channel blockIdx.x of either weight: the workgroups' sums, in a fixed order.
__global__ __launch_bounds__(kT) void qk_norm_sum_kernel(QkNormArgs a) {
  __shared__ float waves[kT / 64];
  const int ch = blockIdx.x, second = blockIdx.y, groups = a.groups[second];
  if (!a.s[second].dw) return;
  const float* part = a.ws + (second ? (int64_t)a.groups[0] * a.D : 0) + (int64_t)ch * groups;
  float s = 0.0f;
#pragma unroll 4
  for (int g = threadIdx.x; g < groups; g += kT) s += part[g];
  s = lane_group_sum<64>(s);
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) a.s[second].dw[ch] = (waves[0] + waves[1]) + (waves[2] + waves[3]);
}

constexpr int lanes_for(int units) { return units <= 1 ? 1 : units <= 2 ? 2 : units <= 4 ? 4 : units <= 8 ? 8 : units <= 16 ? 16 : units <= 32 ? 32 : 64; }

// The widest pieces that the runs of a row are whole numbers of.
int piece_of(const QkNormArgs& a, int widest) {
  for (int v = widest; v > 1; v /= 2)
    if (a.rope_dim % (2 * v) == 0 && (a.D - a.rope_dim) % (2 * v) == 0) return v;
  return 1;
}

int tokens_per_group(int64_t tokens) { return tokens >= 4096 ? kMaxTokens : 1; }

struct Forward {
  template <typename TI, int V, int LG, bool INTER>
  static void go(const QkNormArgs& a, hipStream_t stream) {
    const int tpw = tokens_per_group(a.tokens);
    const int64_t runs = (a.tokens + tpw - 1) / tpw, q = a.s[0].H ? runs : 0, k = a.s[1].H ? runs : 0;
    hipLaunchKernelGGL((qk_norm_fwd_kernel<TI, V, LG, INTER>), dim3((unsigned)(q + k)), dim3(kT),
                       (size_t)tpw * (a.rope_dim / 2) * sizeof(float2), stream, a, tpw, (int)q);
  }
};
struct Backward {
  template <typename TI, int V, int LG, bool INTER>
  static void go(const QkNormArgs& a, hipStream_t stream) {
    const int tpw = tokens_per_group(a.tokens);
    hipLaunchKernelGGL((qk_norm_bwd_kernel<TI, V, LG, INTER>), dim3((unsigned)(a.groups[0] + a.groups[1])), dim3(kT),
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
  const int tpw = tokens_per_group(tokens);
  const int64_t n = (tokens + tpw - 1) / tpw;
  return (int)(n < kMaxGroups ? n : kMaxGroups);
}

hipError_t launch_qk_norm_fwd(const QkNormArgs& a, int dtype, hipStream_t stream) {
  return dispatch<Forward>(a, dtype, stream);
}

hipError_t launch_qk_norm_bwd(const QkNormArgs& given, int dtype, hipStream_t stream) {
  QkNormArgs a = given;
  const int most = qk_norm_groups(a.tokens);
  for (int i = 0; i < 2; ++i) a.groups[i] = a.s[i].H ? most : 0;
  if (a.tokens && a.groups[0] + a.groups[1]) {
    const hipError_t e = dispatch<Backward>(a, dtype, stream);
    if (e != hipSuccess) return e;
  } else {
    a.groups[0] = a.groups[1] = 0;
  }
  if (a.s[0].dw || a.s[1].dw) hipLaunchKernelGGL(qk_norm_sum_kernel, dim3((unsigned)a.D, 2), dim3(kT), 0, stream, a);
  return hipGetLastError();
}

}  // namespace rel
