// Decode step of the causal Full Relation operator over a paged cache: the one
// new row of every (request, head), with keys and values in pages found through
// the request's block table (eq. 2 at position i = the request's length).
//
// The mathematics is that of decode.hip: the history is split into slices, each
// leaves its Exchange scan state (m, l, z) of eq. (11), here with m in units of
// ln 2, and the states of a row are joined with Self and the count correction
// (eqs. 12-13). One workgroup reads a slice of one key head for the query heads
// that share it, so that shared keys are read once. The slice's block-table
// entries are turned into element offsets in LDS first; a key's row is then one
// LDS read away. A batch whose rows have one slice each is finished by the same
// launch.
//
// Two states kernels. In bf16 the products run on the matrix cores, also where
// a key head has one query: sixteen query columns cost what one does, and a wave
// then spends no vector instruction on products and no lane moves on sums. In
// fp32 lanes share a key and multiply themselves.
// Bound by the reads of K and V.
#include "kernels.h"
#include "lanes.h"
#include "serve.h"

namespace rel {

namespace {

constexpr int kMergeT = 256;
constexpr int kStatesT = 256;    // threads of the fp32 states kernel
constexpr int kDies = 8;         // L2 caches of the chip
constexpr int kPlaced = 64;      // groups from which on they are placed by die
// Workgroups (two per CU) below which the bf16 kernel gives them 8 waves instead of 4: 8 of 400 keys x 64 8.5 and 9.8
// us, 128 of 512 9.4 and 10.5. With more workgroups the 8 waves' LDS costs more: 1024 of width 128 189 and 181.
constexpr int kFewGroups = 512;
constexpr int kUnroll = 2;       // keys per lane group of the fp32 kernel whose loads are in flight together

struct Row {
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
  const float a = m == kNegInf ? 0.0f : fast_exp2(m - mn);
  const float b = mo == kNegInf ? 0.0f : fast_exp2(mo - mn);
  l = l * a + lo * b;
#pragma unroll
  for (int e = 0; e < VEC; ++e) z[e] = z[e] * a + zo[e] * b;
  m = mn;
}

// Slice, request and item (of `items` a request) of this workgroup; false past the
// end. The heads of a request stand together in its pages: the items of a slice
// and request run together. Where heads share cache lines (head stride no multiple
// of 128 bytes) they run on one die as well: workgroups go to the kDies dies in turn,
// each die has an L2 cache of its own, and a line read on two is read twice. Groups
// take the dies in turn, from kPlaced groups on. 3 requests of up to 24364 tokens, 12
// heads x 48, heads side by side (162 MB): 45 us, 58 without; width 80: 63 and 69; no
// difference where heads do not share lines.
__device__ __forceinline__ bool place_of(const PagedDecodeArgs& a, int items, int& slice, int& b, int& item) {
  const int groups = a.nsplit * a.B;
  int g;
  if (a.placed) {
    const int s = blockIdx.x / kDies;
    g = s / items * kDies + blockIdx.x % kDies;
    item = s % items;
  } else {
    g = blockIdx.x / items;
    item = blockIdx.x % items;
  }
  slice = g / a.B;
  b = g % a.B;
  return g < groups;
}
int64_t groups_launched(const PagedDecodeArgs& a) {
  const int64_t groups = (int64_t)a.nsplit * a.B;
  return a.placed ? (groups + kDies - 1) / kDies * kDies : groups;
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
  TI* o = (TI*)a.out + ((int64_t)b * a.Hq + hq) * a.c.D;
  if (lane < a.c.D) Elem<TI>::store(o + lane, s.ok ? omg * s.v0 + g * zr0 : nan);
  if (lane + 64 < a.c.D) Elem<TI>::store(o + lane + 64, s.ok ? omg * s.v1 + g * zr1 : nan);
  if (lane == 0 && a.row_stat) a.row_stat[(int64_t)b * a.Hq + hq] = s.ok ? lnZ + lam * ln_i : nan;
}

// Offsets (of head h) of the pages of slice [s0, s0 + slice) into LDS, by all NT
// threads, and whether the thread met a bad page that holds keys of the request's
// history. The table is read before the length is looked at: the two reads run side
// by side.
template <int NT>
__device__ __forceinline__ int page_offsets(const PagedDecodeArgs& a, int b, int h, int s0, int len, int64_t* offs) {
  const int p0 = s0 >> a.c.shift, p1 = min((s0 + a.slice - 1) >> a.c.shift, a.W - 1);
  const int32_t* row = a.table + (int64_t)b * a.W;
  int bad = 0;
  for (int p = p0 + threadIdx.x; p <= p1; p += NT) {
    const int id = row[p];
    const bool ok = id >= 0 && id < a.c.num_pages;
    offs[p - p0] = (int64_t)(ok ? id : 0) * a.c.sp + (int64_t)h * a.c.sh;
    bad |= !ok && (p << a.c.shift) < len - 1;
  }
  return bad;
}

// One wave joins the NW waves' states of a row, (m, l, z) at st + wave * stride in
// LDS, in the waves' order, and stores the slice's state, or finishes the row with
// its Self entry (one slice).
template <typename TI, int NW>
__device__ __forceinline__ void join_waves(const PagedDecodeArgs& a, int slice, int b, int hq, int len, int lane,
                                           const float* st, int stride, const SelfEntry& self) {
  const int D = a.c.D;
  float m = kNegInf, l = 0.0f, z[2] = {0.0f, 0.0f};
#pragma unroll
  for (int x = 0; x < NW; ++x) {
    const float* s = st + x * stride;
    const float zo[2] = {lane < D ? s[2 + lane] : 0.0f, lane + 64 < D ? s[2 + 64 + lane] : 0.0f};
    merge_into<2>(m, l, z, s[0], s[1], zo);
  }
  if (a.nsplit == 1) {
    finish_row<TI>(a, b, hq, len, lane, self, m, l, z[0], z[1]);
    return;
  }
  float* out = a.states + ((int64_t)slice * a.B * a.Hq + (int64_t)b * a.Hq + hq) * (D + 2);
  if (lane == 0) {
    out[0] = m;
    out[1] = l;
  }
  if (lane < D) out[2 + lane] = z[0];
  if (lane + 64 < D) out[2 + 64 + lane] = z[1];
}

// Exchange states of one slice for the query heads [r GQ, r GQ + GQ) of one key
// head (workgroup = (request, key head, r, slice)). LPK lanes share a key: lane
// c of the group holds VEC channels (16 bytes) of the queries and reads those
// of the key and value rows; every lane group keeps its own running (m, l, z),
// and the groups of the workgroup meet in LDS in a fixed order. Measured, 7
// requests of 41 to 2047 tokens, 8 heads x 80 (37 MB): 12.5 us, 3.0 TB/s; the same
// within 5% with 512 threads, slices of 64 keys, or four keys in flight; 19.4 with
// 1024 threads.
template <int LPK, int GQ>
__global__ __launch_bounds__(kStatesT) void paged_states_f32_kernel(PagedDecodeArgs a) {
  constexpr int NT = kStatesT;
  typedef float TI;
  constexpr int VEC = 4;
  constexpr int KPW = 64 / LPK;  // keys per wave and step
  constexpr int NW = NT / 64;
  static_assert(NW >= GQ, "a wave for each query head at the end");
  extern __shared__ int64_t offs[];  // the slice's pages: element offset of (page, head)
  __shared__ float red[NW][GQ][2 + 128];
  const int nr = (a.G + GQ - 1) / GQ;
  int slice, b, item;  // item: (h, r) of a request
  if (!place_of(a, a.c.H * nr, slice, b, item)) return;
  const int r = item % nr, h = item / nr;
  const int hq0 = h * a.G + r * GQ, ng = min(GQ, a.G - r * GQ);
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int c = lane % LPK, kg = lane / LPK;
  const int c0 = c * VEC;
  const bool chan = c0 < a.c.D;
  const int len = length_of(a, b);
  const int s0 = slice * a.slice, s1 = min(s0 + a.slice, len - 1);  // Exchange keys only: j < i - 1 (zero-based)
  const int mask = (1 << a.c.shift) - 1, p0 = s0 >> a.c.shift;
  int bad = page_offsets<NT>(a, b, h, s0, len, offs);
  SelfEntry self{};
  if (a.nsplit == 1 && w < ng) self = read_self<TI>(a, b, hq0 + w, len, lane);
  if (s1 <= s0 && a.nsplit > 1) return;  // a slice past the request's end: nobody reads its state

  float m[GQ], l[GQ], z[GQ][VEC];
#pragma unroll
  for (int g = 0; g < GQ; ++g) {
    m[g] = kNegInf;
    l[g] = 0.0f;
#pragma unroll
    for (int e = 0; e < VEC; ++e) z[g][e] = 0.0f;
  }
  if (s1 > s0) {  // uniform in the workgroup
    float q[GQ][VEC];
#pragma unroll
    for (int g = 0; g < GQ; ++g) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) q[g][e] = 0.0f;
      if (chan && g < ng) Row::load((const TI*)a.q + ((int64_t)b * a.Hq + hq0 + g) * a.c.D + c0, q[g]);
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
          Row::load(K + off, kx[u]);
          Row::load(V + off, vx[u]);
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
            const float E = uu * sigm(uu) * kLog2e;  // Exchange map, eq. (2)
            const float mn = fmaxf(m[g], E);
            const float cr = m[g] == kNegInf ? 0.0f : fast_exp2(m[g] - mn);
            const float p = fast_exp2(E - mn);
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
  // wave g joins the waves' states of query head g
  if (w < ng) join_waves<TI, NW>(a, slice, b, hq0 + w, len, lane, &red[0][w][0], GQ * (2 + 128), self);
}

// The same in bf16 on the matrix cores, for up to 16 query heads of a key head
// (workgroup = (request, key head, group of 16, slice)). A wave takes 32 keys at a
// time, two tiles of 16, DB blocks of 16 channels. Rows are read whole, neighbouring
// lanes neighbouring chunks of 16 bytes, and go through LDS (the wave's own, no
// barrier) into operands:
//   U^T = K q^T (16 x 16 x 32): lane (g, r) = (lane / 16, lane % 16) holds chunks g,
//     g + 4, ... of key r and of query r, and gets the evidence of keys 4 g .. 4 g + 3
//     for query r.
//   z^T += V^T P (16 x 16 x 32): P needs the lane's own eight values in place, the
//     contraction running over keys 4 g .. 4 g + 3 of both tiles; V comes back from LDS
//     by transpose reads.
// z of query r stays in lanes r, r + 16, ..., where its maximum is, so a new maximum
// rescales in place; that is rare after the first keys and costs a branch else.
// P is split as hi + lo, two bf16 numbers of 16 significant bits together: the
// matrix cores have the time, and z keeps fp32-like accuracy.
// Measured, 64 requests of 1024 to 4096 tokens, 12 heads x 64 (504 MB): 99 us, 5.1
// TB/s; 2 x 16 x 128 of up to 65536 (1.02 GB): 181 us, 5.6 TB/s. With each lane
// reading its operand of K from memory (64 bytes of a row per load) 123 and 188;
// with the slices of a row together rather than the heads of a slice 107 of the
// 123; with the vector unit's products (four query heads a pass) 99 and 184 at the
// same slices, but 135 against 73 for four query heads a key head (295 MB).
typedef float floatx4_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ floatx4_t mfma16(const bf16x8& x, const bf16x8& y, const floatx4_t& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, c, 0, 0, 0);
}
__device__ __forceinline__ bf16x8 pack8(const float (&x)[8]) {
  bf16x8 o;
#pragma unroll
  for (int e = 0; e < 8; ++e) o[e] = (bf16)x[e];
  return o;
}

// Orders a wave's LDS accesses for the compiler; in the hardware they keep their order as they are.
__device__ __forceinline__ void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

template <int DB, int NW>
__global__ __launch_bounds__(NW * 64) void paged_states_bf16_kernel(PagedDecodeArgs a) {
  constexpr int KS = (DB + 1) / 2;        // products of 32 channels
  constexpr int ROWB = DB * 32 + 32;      // bytes of a V row in LDS: 32 more, so that rows fall on other banks
  constexpr int WAVEB = 32 * ROWB > 16 * (2 + 16 * DB) * 4 ? 32 * ROWB : 16 * (2 + 16 * DB) * 4;
  static_assert(WAVEB % 16 == 0, "16-byte rows");
  __shared__ __align__(16) unsigned char vlds[NW][WAVEB];
  extern __shared__ int64_t offs[];       // the slice's pages: element offset of (page, head)
  const int nr = (a.G + 15) / 16;
  int slice, b, item;  // item: (h, group) of a request
  if (!place_of(a, a.c.H * nr, slice, b, item)) return;
  const int grp = item % nr, h = item / nr;
  const int hq0 = h * a.G + grp * 16, ng = min(16, a.G - grp * 16);
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int g = lane >> 4, r = lane & 15;
  const int len = length_of(a, b);
  const int s0 = slice * a.slice, s1 = min(s0 + a.slice, len - 1);  // Exchange keys only: j < i - 1 (zero-based)
  const int mask = (1 << a.c.shift) - 1, p0 = s0 >> a.c.shift;
  int bad = page_offsets<NW * 64>(a, b, h, s0, len, offs);
  SelfEntry self{};
  if (a.nsplit == 1 && w < ng) self = read_self<bf16>(a, b, hq0 + w, len, lane);
  if (s1 <= s0 && a.nsplit > 1) return;   // a slice past the request's end: nobody reads its state

  float m = kNegInf, l = 0.0f;
  floatx4_t z[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) z[d] = floatx4_t{0.0f, 0.0f, 0.0f, 0.0f};
  if (s1 > s0) {  // uniform in the workgroup
    const uintx4 none = {0, 0, 0, 0};
    bf16x8 q[KS];
    bool chan[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int c0 = (4 * s + g) * 8;
      chan[s] = c0 < a.c.D;
      uintx4 u = none;
      if (chan[s] && r < ng) u = *reinterpret_cast<const uintx4*>((const bf16*)a.q + ((int64_t)b * a.Hq + hq0 + r) * a.c.D + c0);
      q[s] = __builtin_bit_cast(bf16x8, u);
    }
    // 16-byte chunk x of the tile's 32 rows is row x / nch, chunk x % nch: lane and load i take chunk 64 i + lane
    const int nch = a.c.D / 8, nld = (nch + 1) / 2;
    int krow[DB], kcol[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i) {
      const int x = min(64 * i + lane, 32 * nch - 1);
      krow[i] = x / nch;
      kcol[i] = x - krow[i] * nch;
    }
    bad = __syncthreads_or(bad);
    const bf16 *K = (const bf16*)a.k, *V = (const bf16*)a.v;
    const unsigned char* kr = vlds[w] + r * ROWB + g * 16;                        // this lane's operand chunks of K
    const unsigned char* vr = vlds[w] + (4 * g + (r >> 2)) * ROWB + (r & 3) * 8;  // where its transpose reads start
    uintx4 kx[DB], vx[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i) kx[i] = vx[i] = none;
    auto load = [&](int base) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < DB; ++i) {
        if (i < nld) {
          const int j = min(base + krow[i], s1 - 1);  // past the end: the last key again, which counts for nothing
          const int64_t off = offs[(j >> a.c.shift) - p0] + (int64_t)((j & mask) * a.c.st + kcol[i] * 8);
          kx[i] = *reinterpret_cast<const uintx4*>(K + off);
          vx[i] = *reinterpret_cast<const uintx4*>(V + off);
        }
      }
    };
    if (s0 + 32 * w < s1) load(s0 + 32 * w);
    for (int base = s0 + 32 * w; base < s1; base += 32 * NW) {
      // K through LDS into operands, then V into the same place
      wave_order();
#pragma unroll
      for (int i = 0; i < DB; ++i)
        if (i < nld) *reinterpret_cast<uintx4*>(vlds[w] + krow[i] * ROWB + kcol[i] * 16) = kx[i];
      wave_order();
      floatx4_t u[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        u[t] = floatx4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          uintx4 x = none;
          if (chan[s]) x = *reinterpret_cast<const uintx4*>(kr + 16 * t * ROWB + 64 * s);
          u[t] = mfma16(__builtin_bit_cast(bf16x8, x), q[s], u[t]);
        }
      }
      wave_order();
#pragma unroll
      for (int i = 0; i < DB; ++i)
        if (i < nld) *reinterpret_cast<uintx4*>(vlds[w] + krow[i] * ROWB + kcol[i] * 16) = vx[i];
      wave_order();
      // the registers are free: the next keys' loads run beside the rest of this step
      if (base + 32 * NW < s1) load(base + 32 * NW);
      float e[8];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const float uu = u[t][x] * a.scale;
          const float E = uu * sigm(uu) * kLog2e;  // Exchange map, eq. (2)
          e[4 * t + x] = base + 16 * t + 4 * g + x < s1 ? E : kNegInf;
        }
      }
      float top = e[0];
#pragma unroll
      for (int x = 1; x < 8; ++x) top = fmaxf(top, e[x]);
      if (__any(top > m)) {  // a new maximum of some query
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float mn = fmaxf(m, top), cr = m == kNegInf ? 0.0f : fast_exp2(m - mn);
        l *= cr;
#pragma unroll
        for (int d = 0; d < DB; ++d) z[d] *= cr;
        m = mn;
      }
      float lo[8];
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        e[x] = fast_exp2(e[x] - m);
        l += e[x];
      }
      const bf16x8 ph = pack8(e);
      const uintx4 pu = __builtin_bit_cast(uintx4, ph);
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        lo[2 * x] = e[2 * x] - bf16_lo(pu[x]);
        lo[2 * x + 1] = e[2 * x + 1] - bf16_hi(pu[x]);
      }
      const bf16x8 pl = pack8(lo);
#pragma unroll
      for (int d = 0; d < DB; ++d) {
        const bf16x8 vt = tr_operand(vr + 32 * d, vr + 16 * ROWB + 32 * d);
        z[d] = mfma16(vt, ph, z[d]);
        z[d] = mfma16(vt, pl, z[d]);
      }
    }
    if (bad) l = __builtin_nanf("");
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
  }
  // the wave's state of query r into its LDS: m, l, z
  wave_order();
  constexpr int SW = 2 + 16 * DB;
  float* st = reinterpret_cast<float*>(vlds[w]);
  if (r < ng) {
    if (g == 0) {
      st[r * SW] = m;
      st[r * SW + 1] = l;
    }
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int x = 0; x < 4; ++x) st[r * SW + 2 + 16 * d + 4 * g + x] = z[d][x];
  }
  __syncthreads();
  for (int y = w; y < ng; y += NW) {
    if (a.nsplit == 1 && y >= NW) self = read_self<bf16>(a, b, hq0 + y, len, lane);
    join_waves<bf16, NW>(a, slice, b, hq0 + y, len, lane, reinterpret_cast<const float*>(vlds[0]) + y * SW, WAVEB / 4,
                         self);
  }
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

// Bytes of LDS for the offsets of a slice's pages.
size_t offsets_bytes(const PagedDecodeArgs& a) { return (size_t)((a.slice >> a.c.shift) + 2) * sizeof(int64_t); }

template <int LPK, int GQ>
void launch_f32(const PagedDecodeArgs& a, hipStream_t stream) {
  const int64_t grid = groups_launched(a) * a.c.H * ((a.G + GQ - 1) / GQ);
  hipLaunchKernelGGL((paged_states_f32_kernel<LPK, GQ>), dim3((unsigned)grid), dim3(kStatesT), offsets_bytes(a), stream, a);
}
template <int LPK>
void launch_f32_g(const PagedDecodeArgs& a, hipStream_t stream) {
  if (a.G == 1)
    launch_f32<LPK, 1>(a, stream);
  else if (a.G == 2)
    launch_f32<LPK, 2>(a, stream);
  else
    launch_f32<LPK, 4>(a, stream);
}

template <int DB>
void launch_bf16(const PagedDecodeArgs& a, hipStream_t stream) {
  const int64_t grid = groups_launched(a) * a.c.H * ((a.G + 15) / 16);
  if (grid < kFewGroups)
    hipLaunchKernelGGL((paged_states_bf16_kernel<DB, 8>), dim3((unsigned)grid), dim3(512), offsets_bytes(a), stream, a);
  else
    hipLaunchKernelGGL((paged_states_bf16_kernel<DB, 4>), dim3((unsigned)grid), dim3(256), offsets_bytes(a), stream, a);
}

template <typename TI>
hipError_t launch_merge(const PagedDecodeArgs& a, hipStream_t stream) {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.nsplit == 1) return e;
  const dim3 grid((unsigned)((int64_t)a.B * a.Hq));
  if (a.c.D <= 64)
    hipLaunchKernelGGL((paged_merge_kernel<TI, 32>), grid, dim3(kMergeT), 0, stream, a);
  else
    hipLaunchKernelGGL((paged_merge_kernel<TI, 64>), grid, dim3(kMergeT), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

// Slices of the history: about kTargetGroups workgroups, of at least kMinSlice
// keys (64 requests x 12 heads x 64 of up to 4096: slices of 512 94 us, 1024 96, 2048
// 99, 4096 115; 2 x 16 x 128 of up to 65536: 193, 189, 181, 214; 1 x 8 x 128 of 4096:
// 128 7.7, 256 10.0). A short history is not split and needs no second launch: one
// slice against states and merge, 8 heads, bf16: 1000 keys x 64 10.9 and 6.1 + 4.6
// us (16 requests 12.4 and 12.8 + 4.0); 500 x 128 11.4 and 7.4 + 4.3; 1000 x 128 15.4
// and 7.4 + 4.9; fp32, 250 x 64 8.7 and 6.1 + 4.3; 500 x 64, 16 requests, 16.2 and
// 9.4 + 4.0.
void paged_decode_split(int64_t B, int64_t H, int64_t G, int64_t max_len, int D, int dtype, int* slice, int* nsplit) {
  constexpr int64_t kTargetGroups = 1536, kMinSlice = 128, kMaxSlice = 4096;
  const int64_t hist = max_len > 1 ? max_len - 1 : 1, rows = B * H * ((G + 15) / 16);
  const int64_t one = dtype == 1 ? (D <= 64 ? 1024 : 512) : 256;
  int64_t s = kMinSlice;
  while (s < kMaxSlice && s * kTargetGroups < hist * rows) s *= 2;
  if (hist <= one) s = one;
  *slice = (int)s;
  *nsplit = (int)((hist + s - 1) / s);
}

hipError_t launch_paged_decode(const PagedDecodeArgs& given, int dtype, hipStream_t stream) {
  PagedDecodeArgs a = given;
  const int D = a.c.D;
  a.placed = (int64_t)a.nsplit * a.B >= kPlaced && (int64_t)a.c.sh * (dtype == 1 ? 2 : 4) % 128 != 0;
  if (dtype == 1) {
    if (D <= 32)
      launch_bf16<2>(a, stream);
    else if (D <= 64)
      launch_bf16<4>(a, stream);
    else if (D <= 96)
      launch_bf16<6>(a, stream);
    else
      launch_bf16<8>(a, stream);
    return launch_merge<bf16>(a, stream);
  }
  if (D <= 16)
    launch_f32_g<4>(a, stream);
  else if (D <= 32)
    launch_f32_g<8>(a, stream);
  else if (D <= 64)
    launch_f32_g<16>(a, stream);
  else
    launch_f32_g<32>(a, stream);
  return launch_merge<float>(a, stream);
}

}  // namespace rel
