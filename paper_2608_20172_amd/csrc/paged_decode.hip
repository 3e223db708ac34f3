// Decode step of the causal Full Relation operator over a paged cache: the one
// new row of every (request, head), with keys and values in pages found through
// the request's block table (eq. 2 at position i = the request's length).
//
// The mathematics is that of decode.hip: the history is split into slices, each
// leaves its Exchange scan state (m, l, z) of eq. (11), and the states of a row
// are joined with Self and the count correction (eqs. 12-13). One workgroup
// reads a slice of one key head for up to GQ of the query heads that share it,
// so that shared keys are read once. The slice's block-table entries are turned
// into element offsets in LDS first; a key's row is then one LDS read away. A
// batch whose rows have one slice each is finished by the same launch.
//
// Bound by the reads of K and V.
#include "kernels.h"
#include "lanes.h"
#include "serve.h"

namespace rel {

namespace {

constexpr int kMergeT = 256;
constexpr int kUnroll = 2;  // keys per lane group whose loads are in flight together

template <typename TI, int VEC>
struct Row;
template <>
struct Row<bf16, 8> {
  static __device__ __forceinline__ void load(const bf16* p, float (&x)[8]) {
    const uintx4 u = *reinterpret_cast<const uintx4*>(p);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      x[2 * t] = bf16_lo(u[t]);
      x[2 * t + 1] = bf16_hi(u[t]);
    }
  }
};
template <>
struct Row<float, 4> {
  static __device__ __forceinline__ void load(const float* p, float (&x)[4]) {
    const float4 u = *reinterpret_cast<const float4*>(p);
    x[0] = u.x; x[1] = u.y; x[2] = u.z; x[3] = u.w;
  }
};

__device__ __forceinline__ float sigm(float x) { return fast_rcp(1.0f + fast_exp2(-x * kLog2e)); }

// The request's length, and 0 where it is outside 1 .. max_len (then nothing is read and NaN is written).
__device__ __forceinline__ int length_of(const PagedDecodeArgs& a, int b) {
  const int n = a.lengths[b];
  return n >= 1 && n <= a.max_len ? n : 0;
}

// Merges state (mo, lo, zo) into (m, l, z); an empty state has m = -inf, l = 0. A NaN in l stays.
template <int VEC>
__device__ __forceinline__ void merge_into(float& m, float& l, float (&z)[VEC], float mo, float lo,
                                           const float (&zo)[VEC]) {
  const float mn = fmaxf(m, mo);
  const float a = m == kNegInf ? 0.0f : fast_exp2((m - mn) * kLog2e);
  const float b = mo == kNegInf ? 0.0f : fast_exp2((mo - mn) * kLog2e);
  l = l * a + lo * b;
#pragma unroll
  for (int e = 0; e < VEC; ++e) z[e] = z[e] * a + zo[e] * b;
  m = mn;
}

// Element offset of the request's entry j (0-based) at head h; false if its page is not one of the pool's.
__device__ __forceinline__ bool entry_offset(const PagedDecodeArgs& a, int b, int h, int j, int64_t& off) {
  const int id = a.table[(int64_t)b * a.W + (j >> a.c.shift)];
  const bool ok = id >= 0 && id < a.c.num_pages;
  off = (int64_t)(ok ? id : 0) * a.c.sp + (int64_t)h * a.c.sh + (int64_t)(j & ((1 << a.c.shift) - 1)) * a.c.st;
  return ok;
}

// The Self entry's reads of one wave: lane holds channels lane and lane + 64.
struct SelfEntry {
  float dot, v0, v1;  // q . k over the lane's channels; the own value
  bool ok;
};
template <typename TI>
__device__ __forceinline__ SelfEntry read_self(const PagedDecodeArgs& a, int b, int hq, int len, int lane) {
  SelfEntry s{0.0f, 0.0f, 0.0f, false};
  if (len < 1) return s;
  int64_t off;
  s.ok = entry_offset(a, b, hq / a.G, len - 1, off);
  if (!s.ok) return s;
  const TI* q = (const TI*)a.q + ((int64_t)b * a.Hq + hq) * a.c.D;
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

// Eqs. 12-13 of one row by one wave: state (m, l) with z0, z1 at channels lane, lane + 64.
template <typename TI>
__device__ __forceinline__ void finish_row(const PagedDecodeArgs& a, int b, int hq, int len, int lane, SelfEntry s,
                                           float m, float l, float z0, float z1) {
  float d = s.dot;
  for (int o = 32; o >= 1; o >>= 1) d += __shfl_xor(d, o, 64);
  const float S = 1.0f / (1.0f + expf(-d * a.scale * a.inv_tau));
  const float ln_i = logf((float)len);
  const float lam = *a.lambda;
  float g = 0.0f, omg = 1.0f, zr0 = 0.0f, zr1 = 0.0f, lnZ = S;
  if (!(l == 0.0f)) {                               // some history (or a NaN in it)
    const float A = m + logf(l) - lam * ln_i;       // A_i = L^E_i - lambda ln i (eq. 5)
    g = 1.0f / (1.0f + expf(S - A));                // g = sigmoid(A - S)
    omg = 1.0f / (1.0f + expf(A - S));              // 1 - g = sigmoid(S - A)
    const float il = 1.0f / l;
    zr0 = z0 * il;
    zr1 = z1 * il;
    lnZ = fmaxf(S, A) + log1pf(expf(-fabsf(S - A)));
  }
  // a length outside 1 .. max_len or a page outside the pool: NaN, so that the error is seen
  const float nan = __builtin_nanf("");
  TI* o = (TI*)a.out + ((int64_t)b * a.Hq + hq) * a.c.D;
  if (lane < a.c.D) Elem<TI>::store(o + lane, s.ok ? omg * s.v0 + g * zr0 : nan);
  if (lane + 64 < a.c.D) Elem<TI>::store(o + lane + 64, s.ok ? omg * s.v1 + g * zr1 : nan);
  if (lane == 0 && a.row_stat) a.row_stat[(int64_t)b * a.Hq + hq] = s.ok ? lnZ + lam * ln_i : nan;
}

// Exchange states of one slice for the query heads [r GQ, r GQ + GQ) of one key
// head (workgroup = (request, key head, r, slice)). LPK lanes share a key: lane
// c of the group holds VEC channels (16 bytes) of the queries and reads those
// of the key and value rows; every lane group keeps its own running (m, l, z),
// and the groups of the workgroup meet in LDS in a fixed order.
template <typename TI, int VEC, int LPK, int GQ, int NT>
__global__ __launch_bounds__(NT) void paged_states_kernel(PagedDecodeArgs a) {
  constexpr int KPW = 64 / LPK;  // keys per wave and step
  constexpr int NW = NT / 64;
  static_assert(NW >= GQ, "a wave for each query head at the end");
  extern __shared__ int64_t offs[];  // the slice's pages: element offset of (page, head)
  __shared__ float red[NW][GQ][2 + 128];
  const int nr = (a.G + GQ - 1) / GQ;
  const int slice = blockIdx.x % a.nsplit;
  const int row = blockIdx.x / a.nsplit;  // (b, h, r)
  const int r = row % nr, h = row / nr % a.c.H, b = row / nr / a.c.H;
  const int hq0 = h * a.G + r * GQ, ng = min(GQ, a.G - r * GQ);
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int c = lane % LPK, kg = lane / LPK;
  const int c0 = c * VEC;
  const bool chan = c0 < a.c.D;
  const int len = length_of(a, b);
  const int s0 = slice * a.slice, s1 = min(s0 + a.slice, len - 1);  // Exchange keys only: j < i - 1 (zero-based)
  const int mask = (1 << a.c.shift) - 1, p0 = s0 >> a.c.shift;

  float m[GQ], l[GQ], z[GQ][VEC];
#pragma unroll
  for (int g = 0; g < GQ; ++g) {
    m[g] = kNegInf;
    l[g] = 0.0f;
#pragma unroll
    for (int e = 0; e < VEC; ++e) z[g][e] = 0.0f;
  }
  if (s1 > s0) {  // uniform in the workgroup
    int bad = 0;
    for (int p = p0 + threadIdx.x; p <= (s1 - 1) >> a.c.shift; p += NT) {
      const int id = a.table[(int64_t)b * a.W + p];
      const bool ok = id >= 0 && id < a.c.num_pages;
      offs[p - p0] = (int64_t)(ok ? id : 0) * a.c.sp + (int64_t)h * a.c.sh;
      bad |= !ok;
    }
    float q[GQ][VEC];
#pragma unroll
    for (int g = 0; g < GQ; ++g) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) q[g][e] = 0.0f;
      if (chan && g < ng) Row<TI, VEC>::load((const TI*)a.q + ((int64_t)b * a.Hq + hq0 + g) * a.c.D + c0, q[g]);
    }
    bad = __syncthreads_or(bad);
    const TI *K = (const TI*)a.k + c0, *V = (const TI*)a.v + c0;
    // kUnroll keys per lane group in flight; the loop runs on a wave-uniform
    // base, so that every lane reaches the lane moves
    for (int base = s0 + kUnroll * w * KPW; base < s1; base += kUnroll * NW * KPW) {
      float kx[kUnroll][VEC], vx[kUnroll][VEC];
      bool ok[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int j = base + u * KPW + kg;
        ok[u] = j < s1;
#pragma unroll
        for (int e = 0; e < VEC; ++e) kx[u][e] = vx[u][e] = 0.0f;
        if (ok[u] && chan) {
          const int64_t off = offs[(j >> a.c.shift) - p0] + (int64_t)((j & mask) * a.c.st);
          Row<TI, VEC>::load(K + off, kx[u]);
          Row<TI, VEC>::load(V + off, vx[u]);
        }
      }
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
#pragma unroll
        for (int g = 0; g < GQ; ++g) {
          float d = 0.0f;
#pragma unroll
          for (int e = 0; e < VEC; ++e) d = __builtin_fmaf(q[g][e], kx[u][e], d);
          d = lane_group_sum<LPK>(d);
          if (ok[u]) {
            const float uu = d * a.scale;
            const float E = uu * sigm(uu);  // Exchange map, eq. (2)
            const float mn = fmaxf(m[g], E);
            const float cr = m[g] == kNegInf ? 0.0f : fast_exp2((m[g] - mn) * kLog2e);
            const float p = fast_exp2((E - mn) * kLog2e);
            l[g] = l[g] * cr + p;
#pragma unroll
            for (int e = 0; e < VEC; ++e) z[g][e] = __builtin_fmaf(p, vx[u][e], z[g][e] * cr);
            m[g] = mn;
          }
        }
      }
    }
    if (bad) {
#pragma unroll
      for (int g = 0; g < GQ; ++g) l[g] = __builtin_nanf("");
    }
#pragma unroll
    for (int g = 0; g < GQ; ++g) {
      // merge the lane groups of a wave (lanes with equal c hold the same channels)
#pragma unroll
      for (int o = LPK; o < 64; o <<= 1) {
        float zo[VEC];
        const float mo = __shfl_xor(m[g], o, 64), lo = __shfl_xor(l[g], o, 64);
#pragma unroll
        for (int e = 0; e < VEC; ++e) zo[e] = __shfl_xor(z[g][e], o, 64);
        merge_into<VEC>(m[g], l[g], z[g], mo, lo, zo);
      }
    }
  }
  if (kg == 0) {
#pragma unroll
    for (int g = 0; g < GQ; ++g) {
      if (c == 0) {
        red[w][g][0] = m[g];
        red[w][g][1] = l[g];
      }
      if (chan) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) red[w][g][2 + c0 + e] = z[g][e];
      }
    }
  }
  __syncthreads();
  // wave g joins the waves' states of query head g: lane holds channels lane and lane + 64
  if (w >= ng) return;
  const int hq = hq0 + w;
  SelfEntry self;
  if (a.nsplit == 1) self = read_self<TI>(a, b, hq, len, lane);
  float mm = kNegInf, ll = 0.0f, zz[2] = {0.0f, 0.0f};
  for (int x = 0; x < NW; ++x) {
    const float zo[2] = {lane < a.c.D ? red[x][w][2 + lane] : 0.0f, lane + 64 < a.c.D ? red[x][w][2 + 64 + lane] : 0.0f};
    merge_into<2>(mm, ll, zz, red[x][w][0], red[x][w][1], zo);
  }
  if (a.nsplit == 1) {
    finish_row<TI>(a, b, hq, len, lane, self, mm, ll, zz[0], zz[1]);
    return;
  }
  float* st = a.states + ((int64_t)slice * a.B * a.Hq + (int64_t)b * a.Hq + hq) * (a.c.D + 2);
  if (lane == 0) {
    st[0] = mm;
    st[1] = ll;
  }
  if (lane < a.c.D) st[2 + lane] = zz[0];
  if (lane + 64 < a.c.D) st[2 + 64 + lane] = zz[1];
}

// One workgroup per (b, query head): joins the row's states. Only the slices
// that the request reaches were written with something; the others are not
// read. A lane holds a channel pair and G lanes a state; lane group g takes the
// states g, g + NG, ..., kBatch of them in flight, against its own running
// maximum, and the groups meet in LDS.
template <typename TI, int G>
__global__ __launch_bounds__(kMergeT) void paged_merge_kernel(PagedDecodeArgs a) {
  constexpr int NG = kMergeT / G, kBatch = 8;
  __shared__ float mls[NG][2];
  __shared__ float zsh[NG][2 * G];
  const int n = blockIdx.x;  // b * Hq + hq
  const int tid = threadIdx.x, w = tid >> 6, lane = tid & 63;
  const int b = n / a.Hq, hq = n % a.Hq;
  const int len = length_of(a, b);
  const int D = a.c.D;
  const int ns = len > 1 ? (len - 2) / a.slice + 1 : 0;  // slices with an Exchange key
  const int64_t stride_s = (int64_t)a.B * a.Hq * (D + 2);
  const float* st0 = a.states + (int64_t)n * (D + 2);
  SelfEntry self{};
  if (w == 0) self = read_self<TI>(a, b, hq, len, lane);  // first, so that it overlaps the states' reads
  const int grp = tid / G, c0 = 2 * (tid % G);
  const int cz = c0 < D ? c0 : 0;  // lanes past the width repeat the first pair; nobody reads theirs
  float m = kNegInf, l = 0.0f, z[2] = {0.0f, 0.0f};
  for (int s0 = grp; s0 < ns; s0 += NG * kBatch) {
    float2 ml[kBatch], zz[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {  // slots past the end read the last state and count for nothing
      const float* st = st0 + min(s0 + k * NG, ns - 1) * stride_s;
      ml[k] = *reinterpret_cast<const float2*>(st);  // 8-byte aligned: D + 2 and c0 even
      zz[k] = *reinterpret_cast<const float2*>(st + 2 + cz);
    }
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const float zo[2] = {zz[k].x, zz[k].y};
      if (s0 + k * NG < ns) merge_into<2>(m, l, z, ml[k].x, ml[k].y, zo);
    }
  }
  if (c0 == 0) {
    mls[grp][0] = m;
    mls[grp][1] = l;
  }
  *reinterpret_cast<float2*>(&zsh[grp][c0]) = float2{z[0], z[1]};
  __syncthreads();
  if (w != 0) return;  // the first wave finishes the row
  m = kNegInf;
  l = z[0] = z[1] = 0.0f;
#pragma unroll
  for (int x = 0; x < NG; ++x) {
    const float zo[2] = {zsh[x][lane], G > 32 ? zsh[x][(64 + lane) % (2 * G)] : 0.0f};
    merge_into<2>(m, l, z, mls[x][0], mls[x][1], zo);
  }
  finish_row<TI>(a, b, hq, len, lane, self, m, l, z[0], z[1]);
}

template <typename TI, int VEC, int LPK, int GQ>
void launch_states(const PagedDecodeArgs& a, hipStream_t stream) {
  constexpr int NT = 256;
  const int nr = (a.G + GQ - 1) / GQ;
  const size_t lds = (size_t)((a.slice >> a.c.shift) + 2) * sizeof(int64_t);
  hipLaunchKernelGGL((paged_states_kernel<TI, VEC, LPK, GQ, NT>), dim3((unsigned)((int64_t)a.nsplit * a.B * a.c.H * nr)),
                     dim3(NT), lds, stream, a);
}

template <typename TI, int VEC, int LPK>
void launch_states_g(const PagedDecodeArgs& a, hipStream_t stream) {
  if (a.G == 1)
    launch_states<TI, VEC, LPK, 1>(a, stream);
  else if (a.G == 2)
    launch_states<TI, VEC, LPK, 2>(a, stream);
  else
    launch_states<TI, VEC, LPK, 4>(a, stream);
}

template <typename TI, int VEC>
hipError_t launch_t(const PagedDecodeArgs& a, hipStream_t stream) {
  const int lanes = (a.c.D + VEC - 1) / VEC;
  if (lanes <= 4)
    launch_states_g<TI, VEC, 4>(a, stream);
  else if (lanes <= 8)
    launch_states_g<TI, VEC, 8>(a, stream);
  else if (lanes <= 16)
    launch_states_g<TI, VEC, 16>(a, stream);
  else
    launch_states_g<TI, VEC, 32>(a, stream);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.nsplit == 1) return e;
  const dim3 grid((unsigned)((int64_t)a.B * a.Hq));
  if (a.c.D <= 64)
    hipLaunchKernelGGL((paged_merge_kernel<TI, 32>), grid, dim3(kMergeT), 0, stream, a);
  else
    hipLaunchKernelGGL((paged_merge_kernel<TI, 64>), grid, dim3(kMergeT), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

void paged_decode_split(int64_t B, int64_t H, int64_t G, int64_t max_len, int* slice, int* nsplit) {
  const int64_t hist = max_len > 1 ? max_len - 1 : 1;
  *slice = 256;
  *nsplit = (int)((hist + *slice - 1) / *slice);
}

hipError_t launch_paged_decode(const PagedDecodeArgs& a, int dtype, hipStream_t stream) {
  return dtype == 1 ? launch_t<bf16, 8>(a, stream) : launch_t<float, 4>(a, stream);
}

}  // namespace rel
