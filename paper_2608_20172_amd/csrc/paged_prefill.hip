// Full Relation of chunks of new tokens over a paged cache: of every request b the
// rows at positions lengths[b] - n_b + 1 .. lengths[b] (eqs. 1-3 at those
// positions), n_b its tokens of this step, with keys and values in pages found
// through its block table.
//
// The scan is that of the fused forward pass (scan.h): 32x32 blocks of transposed
// evidence, the running reference held at 0 and checked at the end. What differs:
// * A tile has 128 rows of one request and key head, a row being a (token, query
//   head) pair with the G query heads of a token side by side, so that a key head
//   that they share is read once for all. A lane's row has a position of its own,
//   anywhere in its 32-key block.
// * The requests' tokens are packed; where they start is device data. Every
//   workgroup finds its tile by a scan over the requests' tile counts in LDS.
// * A tile of 64 keys is gathered: each lane looks up the page of the key row that
//   it loads, one tile ahead, and its 16-byte loads write LDS directly. Rows past
//   the tile's last position are that position's again (masked), so nothing past a
//   request's length is read.
// * What stands behind a row in the cache, NaN and infinities included, must not
//   reach it, but a masked weight of 0 times such a value would: a wave whose sums
//   are not finite scans again with those values taken apart.
#include "kernels.h"
#include "paged_row.h"
#include "scan.h"
#include "serve.h"

#include <type_traits>

namespace rel {

namespace {

constexpr int kNT = 256;   // threads of a workgroup
constexpr int kBK = 64;    // keys of a tile
constexpr int kRows = 128; // rows of a tile
constexpr unsigned kMany = 1u << 30;
constexpr int kNone = 0x7fffffff;

__device__ __forceinline__ unsigned add_many(unsigned x, unsigned y) { return min(x + y, kMany); }

// Tokens of request b and the first of them, whatever row_start holds.
__device__ __forceinline__ int tokens_of(const PagedPrefillArgs& a, int b, int& first) {
  first = min(max(a.row_start[b], 0), a.N);
  return min(max(a.row_start[b + 1], first), a.N) - first;
}
__device__ __forceinline__ int tiles_of(const PagedPrefillArgs& a, int b) {
  int first;
  return (tokens_of(a, b, first) * a.G + kRows - 1) / kRows;
}

// Request and tile of it that tile t of the batch is; false past the last. All threads call it; place has two ints.
__device__ __forceinline__ bool find_tile(const PagedPrefillArgs& a, unsigned t, int& b, int& own, int* place,
                                          unsigned* wsum) {
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int per = (a.B + kNT - 1) / kNT;
  const int b0 = min(tid * per, a.B), b1 = min(b0 + per, a.B);
  unsigned mine = 0;
  for (int x = b0; x < b1; ++x) mine = add_many(mine, (unsigned)tiles_of(a, x));
  unsigned incl = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const unsigned y = __shfl_up(incl, o, 64);
    if (lane >= o) incl = add_many(incl, y);
  }
  if (lane == 63) wsum[w] = incl;
  unsigned before = __shfl_up(incl, 1, 64);
  if (lane == 0) before = 0;
  if (tid == 0) place[0] = -1;
  __syncthreads();
#pragma unroll
  for (int x = 0; x < kNT / 64; ++x)
    if (x < w) before = add_many(before, wsum[x]);
  if (t >= before && t < add_many(before, mine)) {  // one thread at most
    for (int x = b0; x < b1; ++x) {
      const unsigned n = (unsigned)tiles_of(a, x);
      if (t - before < n) {
        place[0] = x;
        place[1] = (int)(t - before);
        break;
      }
      before += n;
    }
  }
  __syncthreads();
  b = __builtin_amdgcn_readfirstlane(place[0]);
  own = __builtin_amdgcn_readfirstlane(place[1]);
  return b >= 0;
}

// Which 1 KB segments of a tile a wave loads. In bf16 the segments of one wave are the same 16 rows at all channels, so
// that a lane meets one row; in fp32 each has rows of its own.
template <class P>
struct Gather {
  static constexpr int NSEG = kBK * P::ROWB / 1024, SEGW = NSEG / 4;
  static constexpr bool kOneRow = sizeof(typename P::T) == 2;
  static constexpr int ROWS = kOneRow ? 1 : SEGW;
  static __device__ __forceinline__ int seg(int w, int s) { return kOneRow ? w + 4 * s : w * SEGW + s; }
};

typedef const __attribute__((address_space(1))) void global_void;

// The first key whose page is not one of the pool's, of those that this lane met.
template <class P>
__device__ __forceinline__ void look_up(const PagedPrefillArgs& a, const int32_t* row, int kt, int w, int lane, int jlast,
                                        int (&id)[Gather<P>::ROWS]) {
#pragma unroll
  for (int s = 0; s < Gather<P>::ROWS; ++s) {
    int r, gbyte, lds_off;
    P::seg_map(Gather<P>::seg(w, s), lane, r, gbyte, lds_off);
    id[s] = row[min(kt * kBK + r, jlast) >> a.c.shift];
  }
}
template <class P>
__device__ __forceinline__ void load_tile(const PagedPrefillArgs& a, const char* k, const char* v, int kt, int w, int lane,
                                          int jlast, const int (&id)[Gather<P>::ROWS], unsigned char* Kd,
                                          unsigned char* Vd, int& bad) {
  constexpr int es = sizeof(typename P::T);
  const int mask = (1 << a.c.shift) - 1;
  int64_t off = 0;
#pragma unroll
  for (int s = 0; s < Gather<P>::SEGW; ++s) {
    int r, gbyte, lds_off;
    P::seg_map(Gather<P>::seg(w, s), lane, r, gbyte, lds_off);
    if (!Gather<P>::kOneRow || s == 0) {
      const int j = min(kt * kBK + r, jlast), x = id[Gather<P>::kOneRow ? 0 : s];
      const bool ok = x >= 0 && x < a.c.num_pages;
      if (!ok) bad = min(bad, j);
      off = ((int64_t)(ok ? x : 0) * a.c.sp + (int64_t)(j & mask) * a.c.st) * es;
    }
    if (gbyte < a.c.D * es) {  // channels that the cache has; the others' places hold zeros from the start
      __builtin_amdgcn_global_load_lds((global_void*)(k + off + gbyte), (lds_void*)(Kd + lds_off), 16, 0, 0);
      __builtin_amdgcn_global_load_lds((global_void*)(v + off + gbyte), (lds_void*)(Vd + lds_off), 16, 0, 0);
    }
  }
}

// The query operand of one row, zero past the cache's width (times c in mode 1).
template <class P, int KS, int QM>
__device__ __forceinline__ void load_row(const typename P::T* q, bool live, int width, const Lane& L, float c,
                                         typename P::Op (&qop)[KS]) {
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    qop[ks] = typename P::Op{};
    if constexpr (QM == 0) {
      if (live && 16 * ks + 8 * L.g < width) qop[ks] = P::row_op_g(q, ks, L);
    } else {
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        const int e = 16 * ks + 2 * t + L.g;
        if (live && e < width) qop[ks][t] = q[e] * c;
      }
    }
  }
}

// The 64 keys of a tile from global key k0 on, some of which may be at or past a row's own position `pos` (-1: no row).
// phi: the last position of the wave's rows.
template <class P, int D, int QM>
__device__ __forceinline__ void masked_keys64(const unsigned char* Ks, const unsigned char* Vs, int k0, int phi, int pos,
                                              const typename P::Op (&qop)[D / 16], floatx16 (&oacc)[D / 32], float m,
                                              float& l, float& uii, const Lane& L, float c) {
  constexpr int KS = D / 16;
  using Op = typename P::Op;
  const int k1 = k0 + 32;
  Op p0[2] = {Op{}, Op{}}, p1[2] = {Op{}, Op{}};
  floatx16 s1;
  if (k0 <= phi) {
    const floatx16 s0 = evidence<P, KS>(Ks, 0, qop, L);
    fast_block<P, D, QM, true>(s0, m, l, uii, p0, L, pos - k0, c);
  }
  if (k1 <= phi) s1 = evidence<P, KS>(Ks, 32, qop, L);
  __builtin_amdgcn_sched_barrier(0);
  add_values<P, D>(Vs, 0, 0, p0, oacc, L);
  __builtin_amdgcn_sched_barrier(0);
  if (k1 <= phi) fast_block<P, D, QM, true>(s1, m, l, uii, p1, L, pos - k1, c);
  add_values<P, D>(Vs, 0, 1, p1, oacc, L);
}

// One element of a tile.
template <class P>
__device__ __forceinline__ float tile_element(const unsigned char* lds, int row, int col) {
  if constexpr (sizeof(typename P::T) == 2)
    return (float)*reinterpret_cast<const bf16*>(lds + P::off(row, col));
  else
    return P::fp(lds)[row * P::ROWF + col];
}
// The values of a block that are not finite into the sums of the rows that they reach (weights are positive).
template <class P, int D>
__device__ __forceinline__ void add_not_finite(const unsigned char* Vs, int krow0, int self, floatx16 (&oacc)[D / 32],
                                               const Lane& L, int lane) {
  for (int kk = 0; kk < 32; ++kk) {
    bool some = false;
    for (int col = lane; col < D; col += 64) some |= !(fabsf(tile_element<P>(Vs, krow0 + kk, col)) < __builtin_inff());
    if (!wave_any(some)) continue;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float x = tile_element<P>(Vs, krow0 + kk, 32 * db + acc_row(r, L.g));
        if (kk < self && !(fabsf(x) < __builtin_inff())) oacc[db][r] += x;
      }
  }
}

// The 64 keys again with the reference raised as needed, and what is not finite kept from the rows before it. plo, phi:
// the first and last position of the wave's rows.
template <class P, int D, int QM>
__device__ __forceinline__ void slow_keys64(const unsigned char* Ks, const unsigned char* Vs, int kglob, int plo, int phi,
                                            int pos, const typename P::Op (&qop)[D / 16], floatx16 (&oacc)[D / 32],
                                            float& m, float& l, float& uii, const Lane& L, int lane, float c) {
  constexpr int KS = D / 16;
  for (int b = 0; b < 2; ++b) {
    const int k0 = kglob + 32 * b;
    if (k0 > phi) break;
    const floatx16 s = evidence<P, KS>(Ks, 32 * b, qop, L);
    if (k0 + 31 < plo) {
      scan_block<P, D, QM, false>(s, oacc, m, l, uii, Vs, 2 * b, L, 0, c);
    } else {
      scan_block<P, D, QM, true, true>(s, oacc, m, l, uii, Vs, 2 * b, L, pos - k0, c);
      add_not_finite<P, D>(Vs, 32 * b, pos - k0, oacc, L, lane);
    }
  }
}

// A row of a tile: its index in q and out, and its position.
struct TileRow {
  bool live;
  int64_t at;  // row of q, out and row_stat
  int pos;     // from 0; -1: no row
};

template <class P, int D>
constexpr int prefill_occupancy() {
  return sizeof(typename P::T) == 2 ? (D <= 64 ? 3 : 2) : (D <= 64 ? 2 : 1);  // waves per SIMD
}

template <class P, int D>
__global__ __launch_bounds__(kNT, (prefill_occupancy<P, D>())) void prefill_kernel(PagedPrefillArgs a) {
  using E = typename P::T;
  using Op = typename P::Op;
  constexpr int QM = sizeof(E) == 4 ? 1 : 0;
  constexpr int KS = D / 16, DB = D / 32;
  constexpr int TB = kBK * P::ROWB;
  // separate objects: the compiler can then see that reads of one do not wait for the loads in flight into another
  __shared__ __attribute__((aligned(1024))) unsigned char KA[TB];
  __shared__ __attribute__((aligned(1024))) unsigned char VA[TB];
  __shared__ __attribute__((aligned(1024))) unsigned char KB[TB];
  __shared__ __attribute__((aligned(1024))) unsigned char VB[TB];
  __shared__ int place[2], bad_key;
  __shared__ unsigned wsum[kNT / 64];

  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const Lane L(lane);
  int h, tile, b, own;
  if (!map_tile(a.map, blockIdx.x, h, tile, true)) return;
  if (tid == 0) bad_key = kNone;
  if (!find_tile(a, (unsigned)tile, b, own, place, wsum)) return;
  int first;
  const int n = tokens_of(a, b, first), len = a.lengths[b];
  const int width = a.c.D;
  const int row0 = own * kRows, rows = min(kRows, n * a.G - row0);
  auto row_of = [&](int r) __attribute__((always_inline)) {
    const int x = row0 + min(r, rows - 1), tok = x / a.G;
    TileRow t;
    t.live = r < rows;
    t.at = (int64_t)(first + tok) * a.Hq + h * a.G + (x - tok * a.G);
    t.pos = t.live ? len - n + tok : -1;
    return t;
  };
  if (len < n || len > a.max_len) {  // the error is seen
    for (int x = tid; x < rows * width; x += kNT) {
      const int r = x / width;
      Elem<E>::store((E*)a.out + row_of(r).at * width + (x - r * width), __builtin_nanf(""));
    }
    if (a.row_stat && tid < rows) a.row_stat[row_of(tid).at] = __builtin_nanf("");
    return;
  }
  const int p0 = len - n;
  const int wrow = 32 * w;
  const TileRow me = row_of(wrow + L.n);
  // positions: of the tile's first and last row, and of this wave's
  const int tlo = p0 + row0 / a.G, jlast = p0 + (row0 + rows - 1) / a.G;
  const int plo = p0 + (row0 + min(wrow, rows - 1)) / a.G;
  const int phi = wrow < rows ? p0 + (row0 + min(wrow + 31, rows - 1)) / a.G : -1;
  const float c = a.scale * kLog2e;
  const char* k = (const char*)a.k + (int64_t)h * a.c.sh * (int64_t)sizeof(E);
  const char* v = (const char*)a.v + (int64_t)h * a.c.sh * (int64_t)sizeof(E);
  const int32_t* trow = a.table + (int64_t)b * a.W;

  if (width < D) {  // channels past the cache's width: zeros that no load overwrites
    for (int x = tid; x < TB / 16; x += kNT) {
      const uintx4 none = {0, 0, 0, 0};
      *reinterpret_cast<uintx4*>(KA + 16 * x) = none;
      *reinterpret_cast<uintx4*>(VA + 16 * x) = none;
      *reinterpret_cast<uintx4*>(KB + 16 * x) = none;
      *reinterpret_cast<uintx4*>(VB + 16 * x) = none;
    }
    __syncthreads();
  }
  Op qop[KS];
  load_row<P, KS, QM>((const E*)a.q + me.at * width, me.live, width, L, c, qop);

  float m = 0.0f, l = 0.0f, uii = 0.0f;
  floatx16 oacc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) oacc[db] = floatx16{};
  int bad = kNone;
  const int nkt = jlast / kBK + 1;
  int id[Gather<P>::ROWS];
  auto load = [&](int kt, unsigned char* Kd, unsigned char* Vd) __attribute__((always_inline)) {
    load_tile<P>(a, k, v, kt, w, lane, jlast, id, Kd, Vd, bad);
    look_up<P>(a, trow, kt + 1, w, lane, jlast, id);  // past the last tile: the last key's page again
  };
  auto fast_step = [&](auto full, int kt, const unsigned char* Ks, const unsigned char* Vs, unsigned char* Kn,
                       unsigned char* Vn) __attribute__((always_inline)) {
    wait_loads();      // this wave's part of tile kt is in LDS, and the page ids of tile kt + 1 are here
    __syncthreads();   // ... and every wave's; tile kt - 1 is no longer read
    if (kt + 1 < nkt) load(kt + 1, Kn, Vn);
    if (decltype(full)::value)
      full_keys64<P, D, QM>(Ks, Vs, 0, qop, oacc, m, l, uii, L, c);
    else
      masked_keys64<P, D, QM>(Ks, Vs, kt * kBK, phi, me.pos, qop, oacc, m, l, uii, L, c);
  };
  auto run_fast = [&](int ka, int kb, auto full) __attribute__((always_inline)) {
    int kt = ka;
    if (kt < kb && (kt & 1)) {
      fast_step(full, kt, KB, VB, KA, VA);
      ++kt;
    }
    for (; kt < kb; kt += 2) {
      fast_step(full, kt, KA, VA, KB, VB);
      if (kt + 1 < kb) fast_step(full, kt + 1, KB, VB, KA, VA);
    }
  };
  look_up<P>(a, trow, 0, w, lane, jlast, id);
  load(0, KA, VA);
  const int kf = min(tlo / kBK, nkt);  // tiles before every row's position
  run_fast(0, kf, std::true_type{});
  run_fast(kf, nkt, std::false_type{});
  if (bad != kNone) atomicMin(&bad_key, bad);
  // As in the fused forward pass the scan ran with the reference at 0, which is exact while the row total stays under
  // 2^64. Sums that are not finite come from values that are not, perhaps behind the row.
  const float lt = l + xor32(l);
  float f = 0.0f;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) f = __builtin_fmaf(oacc[db][r], 0.0f, f);
  const bool again = me.live && (!(lt <= kSpecMax) || f != f);
  if (__syncthreads_or(again ? 1 : 0)) {
    const bool redo = wave_any(again);
    if (redo) {
      m = l = uii = 0.0f;
#pragma unroll
      for (int db = 0; db < DB; ++db) oacc[db] = floatx16{};
    }
    look_up<P>(a, trow, 0, w, lane, jlast, id);
    load(0, KA, VA);
    for (int kt = 0; kt < nkt; ++kt) {
      const bool odd = kt & 1;
      wait_loads();
      __syncthreads();
      if (kt + 1 < nkt) load(kt + 1, odd ? KA : KB, odd ? VA : VB);
      if (redo)
        slow_keys64<P, D, QM>(odd ? KB : KA, odd ? VB : VA, kt * kBK, plo, phi, me.pos, qop, oacc, m, l, uii, L, lane, c);
    }
  }
  const float total = l + xor32(l);
  const float un = (uii + xor32(uii)) * (QM == 0 ? c : 1.0f);  // one lane of the two has it, the other 0
  if (!me.live) return;
  const float lam = *a.lambda;
  const float ln_i = logf((float)(me.pos + 1));
  const RowEpilogue e = row_epilogue(m, total, un, a.inv_tau, lam, ln_i);
  const bool lost = bad_key <= me.pos || total != total;  // a page outside the pool, or a NaN among the keys
  int64_t off;
  entry_offset(a, b, h, me.pos, off);
  const E* vi = (const E*)a.v + off;
  E* o = (E*)a.out + me.at * width;
#pragma unroll
  for (int db = 0; db < DB; ++db) {
#pragma unroll
    for (int rq = 0; rq < 4; ++rq) {
      const int d0 = 32 * db + 8 * rq + 4 * L.g;
      if (d0 >= width) continue;
      const floatx4 x = P::load4(vi + d0);
      floatx4 y;
#pragma unroll
      for (int t = 0; t < 4; ++t)
        y[t] = lost ? __builtin_nanf("") : __builtin_fmaf(e.omg, x[t], e.inv_l * oacc[db][4 * rq + t]);
      P::store4(o + d0, y);
    }
  }
  if (L.g == 0 && a.row_stat) a.row_stat[me.at] = lost ? __builtin_nanf("") : e.lnZ + lam * ln_i;
}

template <class P, int D>
hipError_t launch_one(PagedPrefillArgs a, hipStream_t stream) {
  // at most so many tiles: each request has one that is not whole
  const int64_t tiles = (int64_t)a.N * a.G / kRows + a.B;
  a.map = make_tilemap(a.c.H, (int)tiles);
  hipLaunchKernelGGL((prefill_kernel<P, D>), dim3((unsigned)grid_size(a.map)), dim3(kNT), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_prefill(const PagedPrefillArgs& a, int dtype, hipStream_t stream) {
  const int D = a.c.D;
  if (dtype == 1) {
    if (D <= 32) return launch_one<PolBF16<32>, 32>(a, stream);
    if (D <= 64) return launch_one<PolBF16<64>, 64>(a, stream);
    if (D <= 96) return launch_one<PolBF16<96>, 96>(a, stream);
    return launch_one<PolBF16<128>, 128>(a, stream);
  }
  if (D <= 32) return launch_one<PolF32<32>, 32>(a, stream);
  if (D <= 64) return launch_one<PolF32<64>, 64>(a, stream);
  return launch_one<PolF32<128>, 128>(a, stream);
}

}  // namespace rel
