// Full Relation of chunks of new tokens over a paged cache: of every request b the
// rows at positions lengths[b] - n_b + 1 .. lengths[b] (eqs. 1-3 at those
// positions), n_b its tokens of this step, with keys and values in pages found
// through its block table.
//
// The scan is that of the fused forward pass (scan.h): 32x32 blocks of transposed
// evidence, the running reference held at 0 and checked at the end. What differs:
// * A tile has 128 rows of one request and key head, 32 a wave, a row being a
//   (token, query head) pair with the G query heads of a token side by side, so
//   that a key head that they share is read once for all. A lane's row has a
//   position of its own, anywhere in its 32-key block.
// * A tile of at most 32 rows (a decoding request among chunks, a short chunk) gives
//   each wave 32 of every 128 keys instead, which it loads for itself; the four
//   partial sums meet in LDS. With the reference at 0 they only add. (40 requests
//   that decode and 8 chunks of 128 to 256 tokens over 410 to 4096 keys, 16 heads of
//   width 128 on 4: 194 us with such a tile's rows all on one wave, 119 with barriers
//   around the loads, 91 without.) Its bf16 weights go into the products with V in two
//   parts, 16 significant bits, as the decode step's do, so that a request that decodes
//   loses nothing by coming here: 93 us against those 91, and one prompt of 2048 tokens (8
//   heads x 64, tiles of 32 rows) 27 against 25.
// * In tiles of 128 rows the weights are rounded to bf16 once, as in the fused forward
//   pass (each off by at most 2^-8 of itself, so y by 2^-8 of its weighted values): they
//   are bound by vector work, and two parts would cost 85 us against 74 for 8 prompts of
//   1024 to 2048 tokens, 12 heads x 64, and 868 against 672 for 2048 tokens after 32768, 16
//   heads of width 128 on 4. Their sum, in M and below the fraction, is of fp32 weights in both.
// * Where the tiles leave CUs idle the histories are split into slices whose terminal
//   states a second kernel merges, as the paged decode step does.
// * The requests' tokens are packed; where they start is device data. Every
//   workgroup finds its tile from the tile counts of all.
// * A tile of 64 keys is gathered: each lane looks up the page of the key row that
//   it loads, one tile ahead, and its 16-byte loads write LDS directly. Rows past
//   the tile's last position are that position's again (masked), so nothing past a
//   request's length is read.
// * What stands behind a row in the cache, NaN and infinities included, must not
//   reach it, but a masked weight of 0 times such a value would: a wave whose sums
//   are not finite scans again with those values taken apart.
//
// What bounds it is the vector work of a weight, about 9 instructions a lane and
// entry beside one matrix instruction, as in the fused forward pass, and the waits
// of a gather: a chunk of 2048 tokens after 32768, 16 heads of width 128 on 4, takes
// 660 to 690 us (0.82 PFLOP/s and more), 8 prompts of 1024 to 2048 tokens, 12 heads x 64, 73 us. On
// the same rows in one dense tensor the fused forward pass, which looks nothing up,
// takes 55 us against 61 (8 x 12 x 1536 x 64) and 164 against 185 (4 x 8 x 4096 x 128). In
// fp32 over 64 channels it is the LDS: the 32 rows of K that a half-wave reads stand 512
// bytes apart, on one bank (92% of the LDS's busy cycles at D = 80 are conflicts).
#include "kernels.h"
#include "lanes.h"
#include "paged_row.h"
#include "scan.h"
#include "serve.h"

#include <type_traits>

namespace rel {

namespace {

constexpr int kNT = 256;   // threads of a workgroup
constexpr int kBK = 64;    // keys of a tile
constexpr int kRows = 128; // rows of a tile, 32 a wave
constexpr int kFewRows = 32;  // rows of a tile that the four waves share
constexpr unsigned kMany = 1u << 30;
constexpr int kNone = 0x7fffffff;

__device__ __forceinline__ unsigned add_many(unsigned x, unsigned y) { return min(x + y, kMany); }

// f over the wave, by every lane: within rows of 16 lanes, then over the rows.
template <typename F>
__device__ __forceinline__ int over_wave(int x, F f) {
  x = f(x, __builtin_amdgcn_update_dpp(0, x, 0xB1, 0xF, 0xF, false));
  x = f(x, __builtin_amdgcn_update_dpp(0, x, 0x4E, 0xF, 0xF, false));
  x = f(x, __builtin_amdgcn_update_dpp(0, x, 0x141, 0xF, 0xF, false));
  x = f(x, __builtin_amdgcn_update_dpp(0, x, 0x140, 0xF, 0xF, false));
  return f(f(__builtin_amdgcn_readlane(x, 0), __builtin_amdgcn_readlane(x, 16)),
           f(__builtin_amdgcn_readlane(x, 32), __builtin_amdgcn_readlane(x, 48)));
}
// Of numbers whose sum stays under 2^31 for ascending row starts; others wrap, to some place.
__device__ __forceinline__ int wave_total(int x) {
  return over_wave(x, [](int y, int z) { return (int)((unsigned)y + (unsigned)z); }) & 0x7fffffff;
}
__device__ __forceinline__ int wave_most(int x) {
  return over_wave(x, [](int y, int z) { return max(y, z); });
}

// Tokens of request b and the first of them, whatever row_start holds.
__device__ __forceinline__ int tokens_of(const PagedPrefillArgs& a, int b, int& first) {
  first = min(max(a.row_start[b], 0), a.N);
  return min(max(a.row_start[b + 1], first), a.N) - first;
}
__device__ __forceinline__ int tiles_of(const PagedPrefillArgs& a, int b) {
  int first;
  return (tokens_of(a, b, first) * a.G + a.tile_rows - 1) / a.tile_rows;
}

// Slice, request and tile of it that item of the batch is; false past the last. Up to 64 requests stand in the lanes of
// every wave alike. Tiles of more than 32 rows come before those of few (with 128-row tiles; 40 requests that decode and 8
// chunks: 113 -> 104 us), and those with the most keys first, by levels: on level L a request has the tile that ends L
// tiles before the longest request's end, so that its tiles stand on levels off .. off + tiles - 1 and with S(L) the sum
// of clamp(L - off, 0, tiles) place t is on the level with S(L) <= t < S(L + 1). The tiles
// of a request still stand together where histories are long, and share its keys in the L2. (8 prompts of 1024 to 2048
// tokens, 12 heads x 64: 98 us request by request, 87 so; 8 chunks of 256 to 512 after 4096 to 8192, 32 heads x 128:
// 529 and 485, and 570 with levels from each request's own end.)
__device__ __forceinline__ bool find_tile_64(const PagedPrefillArgs& a, int item, int& slice, int& b, int& own) {
  const int lane = threadIdx.x & 63;
  int first;
  const int rows = lane < a.B ? tokens_of(a, lane, first) * a.G : 0, all = (rows + a.tile_rows - 1) / a.tile_rows;
  const bool few = all > 0 && a.tile_rows > kFewRows && rows - (all - 1) * a.tile_rows <= kFewRows;
  const int mine = all - few, most = min(wave_total(mine), a.tiles);  // of ascending row starts: all of them
  const unsigned long long behind = ((unsigned long long)1 << lane) - 1;  // the lanes before this one
  if (item < most * a.nsplit) {
    slice = item / most;
    const int t = item - slice * most, len = mine > 0 ? min(max(a.lengths[lane], 0), a.max_len) : 0;
    const int off = (wave_most(len) - len) / max(1, a.tile_rows / a.G), end = mine > 0 ? off + mine : 0;
    auto sum = [&](int level) __attribute__((always_inline)) { return wave_total(min(max(level - off, 0), mine)); };
    int level = 0;  // the largest with S(level) <= t
    for (int bit = 1 << (31 - __builtin_clz(wave_most(end) | 1)); bit; bit >>= 1)
      if (sum(level + bit) <= t) level += bit;
    const int rank = t - sum(level);
    const bool has = level >= off && level < end;
    const unsigned long long have = __ballot(has), it = __ballot(has && (int)__popcll(have & behind) == rank);
    if (!it) return false;
    b = __builtin_amdgcn_readfirstlane((int)__ffsll((long long)it) - 1);
    own = __builtin_amdgcn_readlane(mine - 1 - (level - off), b);
    return true;
  }
  const unsigned long long have = __ballot(few);
  const int rest = item - most * a.nsplit, number = (int)__popcll(have);
  if (!number) return false;
  slice = rest / number;
  const unsigned long long it = __ballot(few && (int)__popcll(have & behind) == rest - slice * number);
  if (slice >= a.nsplit || !it) return false;
  b = __builtin_amdgcn_readfirstlane((int)__ffsll((long long)it) - 1);
  own = __builtin_amdgcn_readlane(mine, b);
  return true;
}
// More requests: one after another, by a scan of all threads. place has two ints.
__device__ __forceinline__ bool find_tile_many(const PagedPrefillArgs& a, unsigned t, int& b, int& own, int* place,
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
        place[1] = (int)(n - 1 - (t - before));
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

// The pages of the key rows that this lane loads of tile kt.
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
// One segment of a row's channels that the cache has; the others' places hold zeros from the start. The instruction's
// own offset, the segment's 64 bytes of the row, counts at both ends.
template <class P, int S>
__device__ __forceinline__ void load_segment(const PagedPrefillArgs& a, const char* k, const char* v, int w, int lane,
                                             unsigned char* Kd, unsigned char* Vd, int gbyte0) {
  int r, gbyte, lds_off;
  P::seg_map(Gather<P>::seg(w, S), lane, r, gbyte, lds_off);
  constexpr int off = Gather<P>::kOneRow ? 64 * S : 0;
  if (gbyte0 + off < a.c.D * (int)sizeof(typename P::T)) {
    __builtin_amdgcn_global_load_lds((global_void*)k, (lds_void*)(Kd + (lds_off - off)), 16, off, 0);
    __builtin_amdgcn_global_load_lds((global_void*)v, (lds_void*)(Vd + (lds_off - off)), 16, off, 0);
  }
}
// All of a lane's segments of a tile. bad: the first key whose page is not one of the pool's, of those that it met.
template <class P, int S = 0>
__device__ __forceinline__ void load_segments(const PagedPrefillArgs& a, const char* k, const char* v, int kt, int w,
                                              int lane, int jlast, const int (&id)[Gather<P>::ROWS], unsigned char* Kd,
                                              unsigned char* Vd, int& bad) {
  if constexpr (S < Gather<P>::SEGW) {
    int r, gbyte, lds_off;
    P::seg_map(Gather<P>::seg(w, S), lane, r, gbyte, lds_off);
    const int j = min(kt * kBK + r, jlast), x = id[Gather<P>::kOneRow ? 0 : S];
    const bool ok = (unsigned)x < (unsigned)a.c.num_pages;
    if (!ok) bad = min(bad, j);
    const int64_t off = ((int64_t)(ok ? x : 0) * a.c.sp + (int64_t)((j & ((1 << a.c.shift) - 1)) * a.c.st)) *
                            (int64_t)sizeof(typename P::T) + gbyte;
    if constexpr (Gather<P>::kOneRow) {  // the same row, 64 bytes on
      const char *kr = k + off, *vr = v + off;
      load_segment<P, 0>(a, kr, vr, w, lane, Kd, Vd, gbyte);
      if constexpr (Gather<P>::SEGW > 1) load_segment<P, 1>(a, kr, vr, w, lane, Kd, Vd, gbyte);
      if constexpr (Gather<P>::SEGW > 2) load_segment<P, 2>(a, kr, vr, w, lane, Kd, Vd, gbyte);
      if constexpr (Gather<P>::SEGW > 3) load_segment<P, 3>(a, kr, vr, w, lane, Kd, Vd, gbyte);
    } else {
      load_segment<P, S>(a, k + off, v + off, w, lane, Kd, Vd, gbyte);
      load_segments<P, S + 1>(a, k, v, kt, w, lane, jlast, id, Kd, Vd, bad);
    }
  }
}
template <class P>
__device__ __forceinline__ void load_tile(const PagedPrefillArgs& a, const char* k, const char* v, int kt, int w, int lane,
                                          int jlast, const int (&id)[Gather<P>::ROWS], unsigned char* Kd,
                                          unsigned char* Vd, int& bad) {
  static_assert(!Gather<P>::kOneRow || Gather<P>::SEGW <= 4, "segments of a row");
  load_segments<P>(a, k, v, kt, w, lane, jlast, id, Kd, Vd, bad);
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
  constexpr bool kParts = sizeof(typename P::T) == 2;  // as the first scan of few rows; it is rare enough for all to have them
  for (int b = 0; b < 2; ++b) {
    const int k0 = kglob + 32 * b;
    if (k0 > phi) break;
    const floatx16 s = evidence<P, KS>(Ks, 32 * b, qop, L);
    if (k0 + 31 < plo) {
      scan_block<P, D, QM, false, false, kParts>(s, oacc, m, l, uii, Vs, 2 * b, L, 0, c);
    } else {
      scan_block<P, D, QM, true, true, kParts>(s, oacc, m, l, uii, Vs, 2 * b, L, pos - k0, c);
      add_not_finite<P, D>(Vs, 32 * b, pos - k0, oacc, L, lane);
    }
  }
}

// A tile of a step: rows row0 .. row0 + rows - 1 of request b at key head h, over the key tiles kt0 .. nkt - 1.
struct Tile {
  int b, h, first, n, len;  // the request's first token and their number, its length
  int row0, rows;
  int slice, kt0, nkt;
  bool few;                 // the four waves share the rows
};
// A row of it: its index in q and out, and its position.
struct TileRow {
  bool live;
  int64_t at;  // row of q, out and row_stat
  int pos;     // from 0; -1: no row
};
__device__ __forceinline__ TileRow row_of(const PagedPrefillArgs& a, const Tile& t, int r) {
  const int x = t.row0 + min(r, t.rows - 1), tok = x / a.G;
  TileRow y;
  y.live = r < t.rows;
  y.at = (int64_t)(t.first + tok) * a.Hq + t.h * a.G + (x - tok * a.G);
  y.pos = y.live ? t.len - t.n + tok : -1;
  return y;
}
__device__ __forceinline__ int position_of(const PagedPrefillArgs& a, const Tile& t, int r) {
  return t.len - t.n + (t.row0 + min(r, t.rows - 1)) / a.G;
}
template <typename E>
__device__ __forceinline__ const char* head_of(const PagedPrefillArgs& a, const void* pool, int h) {
  return (const char*)pool + (int64_t)h * a.c.sh * (int64_t)sizeof(E);
}

// The row of this lane (and of the one 32 away) from its terminal state: into out, or into the slice's states.
template <class P, int D>
__device__ __forceinline__ void finish_tile_row(const PagedPrefillArgs& a, const Tile& t, const TileRow& me, float m, float l,
                                                float uii, const floatx16 (&oacc)[D / 32], int bad_key, const Lane& L) {
  using E = typename P::T;
  constexpr int DB = D / 32;
  const int width = a.c.D;
  const float total = l + xor32(l);
  const float un = (uii + xor32(uii)) * (sizeof(E) == 4 ? 1.0f : a.scale * kLog2e);  // one of the two has it, the other 0
  if (!me.live) return;
  const bool lost = bad_key <= me.pos || total != total;  // a page outside the pool, or a NaN among the keys
  if (a.nsplit > 1) {
    float* st = a.states + ((int64_t)t.slice * a.N * a.Hq + me.at) * (width + 2);
#pragma unroll
    for (int db = 0; db < DB; ++db) {
#pragma unroll
      for (int rq = 0; rq < 4; ++rq) {
        const int d0 = 32 * db + 8 * rq + 4 * L.g;
        if (d0 >= width) continue;
#pragma unroll
        for (int e = 0; e < 4; e += 2)  // 8-byte aligned: the width is a multiple of 4
          *reinterpret_cast<float2*>(st + 2 + d0 + e) = float2{oacc[db][4 * rq + e], oacc[db][4 * rq + e + 1]};
      }
    }
    if (L.g == 0) *reinterpret_cast<float2*>(st) = float2{m, lost ? __builtin_nanf("") : total};
    return;
  }
  const float lam = *a.lambda;
  const float ln_i = logf((float)(me.pos + 1));
  const RowEpilogue e = row_epilogue(m, total, un, a.inv_tau, lam, ln_i);
  int64_t off;
  entry_offset(a, t.b, t.h, me.pos, off);
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
      for (int i = 0; i < 4; ++i)
        y[i] = lost ? __builtin_nanf("") : __builtin_fmaf(e.omg, x[i], e.inv_l * oacc[db][4 * rq + i]);
      P::store4(o + d0, y);
    }
  }
  if (L.g == 0 && a.row_stat) a.row_stat[me.at] = lost ? __builtin_nanf("") : e.lnZ + lam * ln_i;
}

// The scan of a tile again, by the waves whose first one failed its check (redo); all of them load. A function of its
// own, so that its registers are not the fast scan's.
template <class P, int D>
__device__ __attribute__((noinline)) void scan_again(PagedPrefillArgs a, Tile t, bool redo, int bad_key, unsigned char* K0,
                                                     unsigned char* V0, unsigned char* K1, unsigned char* V1) {
  using E = typename P::T;
  constexpr int QM = sizeof(E) == 4 ? 1 : 0;
  constexpr int KS = D / 16, DB = D / 32;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const Lane L(lane);
  const int wrow = t.few ? 0 : 32 * w, jlast = position_of(a, t, t.rows - 1);
  const TileRow me = row_of(a, t, wrow + L.n);
  const int plo = position_of(a, t, wrow), phi = wrow < t.rows ? position_of(a, t, wrow + 31) : -1;
  const float c = a.scale * kLog2e;
  const char *k = head_of<E>(a, a.k, t.h), *v = head_of<E>(a, a.v, t.h);
  const int32_t* trow = a.table + (int64_t)t.b * a.W;
  typename P::Op qop[KS];
  load_row<P, KS, QM>((const E*)a.q + me.at * a.c.D, me.live, a.c.D, L, c, qop);
  float m = 0.0f, l = 0.0f, uii = 0.0f;
  floatx16 oacc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) oacc[db] = floatx16{};
  int bad = kNone, id[Gather<P>::ROWS];
  for (int kt = t.kt0; kt < t.nkt; ++kt) {
    const bool odd = kt & 1;
    look_up<P>(a, trow, kt, w, lane, jlast, id);
    load_tile<P>(a, k, v, kt, w, lane, jlast, id, odd ? K1 : K0, odd ? V1 : V0, bad);
    wait_loads();
    __syncthreads();  // the other buffer is read up to here
    if (redo) slow_keys64<P, D, QM>(odd ? K1 : K0, odd ? V1 : V0, kt * kBK, plo, phi, me.pos, qop, oacc, m, l, uii, L, lane, c);
  }
  if (redo) finish_tile_row<P, D>(a, t, me, m, l, uii, oacc, bad_key, L);
}

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
  constexpr bool kParts = sizeof(E) == 2;  // weights of few rows are in two parts
  // separate objects: the compiler can then see that reads of one do not wait for the loads in flight into another
  __shared__ __attribute__((aligned(1024))) unsigned char KA[TB];
  __shared__ __attribute__((aligned(1024))) unsigned char VA[TB];
  __shared__ __attribute__((aligned(1024))) unsigned char KB[TB];
  __shared__ __attribute__((aligned(1024))) unsigned char VB[TB];
  __shared__ int place[2], bad_key;
  __shared__ float shared_l[kNT / 64][64], shared_u[kNT / 64][64];
  __shared__ unsigned wsum[kNT / 64];

  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const Lane L(lane);
  Tile t;
  int item, own;
  if (!map_tile(a.map, blockIdx.x, t.h, item, false)) return;
  if (tid == 0) bad_key = kNone;
  if (a.B <= 64) {
    if (!find_tile_64(a, item, t.slice, t.b, own)) return;
  } else {
    t.slice = item / a.tiles;
    if (!find_tile_many(a, (unsigned)(item - t.slice * a.tiles), t.b, own, place, wsum)) return;
  }
  t.n = tokens_of(a, t.b, t.first);
  t.len = a.lengths[t.b];
  t.row0 = own * a.tile_rows;
  t.rows = min(a.tile_rows, t.n * a.G - t.row0);
  t.few = t.rows <= kFewRows;
  const int width = a.c.D;
  if (t.len < t.n || t.len > a.max_len) {  // the error is seen (with several slices the merge sees it)
    if (a.nsplit > 1) return;
    for (int x = tid; x < t.rows * width; x += kNT) {
      const int r = x / width;
      Elem<E>::store((E*)a.out + row_of(a, t, r).at * width + (x - r * width), __builtin_nanf(""));
    }
    if (a.row_stat && tid < t.rows) a.row_stat[row_of(a, t, tid).at] = __builtin_nanf("");
    return;
  }
  const int jlast = position_of(a, t, t.rows - 1);  // the last row's position
  t.kt0 = t.slice * (a.slice / kBK);
  t.nkt = min(t.kt0 + a.slice / kBK, jlast / kBK + 1);
  const int kt0 = t.kt0, nkt = t.nkt;
  if (kt0 >= nkt) return;  // a slice behind every row: nobody reads its states
  const bool few = t.few;  // the four waves share the rows and take a block of 32 keys each
  const int wrow = few ? 0 : 32 * w;
  TileRow me = row_of(a, t, wrow + L.n);
  const int tlo = position_of(a, t, 0);  // the first row's position
  const float c = a.scale * kLog2e;
  const char *k = head_of<E>(a, a.k, t.h), *v = head_of<E>(a, a.v, t.h);
  const int32_t* trow = a.table + (int64_t)t.b * a.W;

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
  int id[Gather<P>::ROWS];
  auto load = [&](int kt, unsigned char* Kd, unsigned char* Vd) __attribute__((always_inline)) {
    load_tile<P>(a, k, v, kt, w, lane, jlast, id, Kd, Vd, bad);
    look_up<P>(a, trow, kt + 1, w, lane, jlast, id);  // past the last tile: the last key's page again
  };
  if (few) {
    // 128 keys at a time: waves 0, 1 the blocks of the first tile, waves 2, 3 those of the second. A wave loads what it
    // reads, and waits for nobody.
    const int krow = 32 * (w & 1), part = 2 * (w & 1);
    unsigned char* Ks = w >> 1 ? KB : KA;
    unsigned char* Vs = w >> 1 ? VB : VA;
    int kt = kt0 + (w >> 1), id2[Gather<P>::ROWS];
    look_up<P>(a, trow, kt, part, lane, jlast, id);
    look_up<P>(a, trow, kt, part + 1, lane, jlast, id2);
    for (; kt * kBK + krow <= jlast && kt < nkt; kt += 2) {
      load_tile<P>(a, k, v, kt, part, lane, jlast, id, Ks, Vs, bad);
      load_tile<P>(a, k, v, kt, part + 1, lane, jlast, id2, Ks, Vs, bad);
      look_up<P>(a, trow, kt + 2, part, lane, jlast, id);
      look_up<P>(a, trow, kt + 2, part + 1, lane, jlast, id2);
      wait_loads();
      asm volatile("" ::: "memory");  // no read of them before
      Op pop[2];
      const floatx16 s = evidence<P, KS>(Ks, krow, qop, L);
      if constexpr (kParts) {
        Op rest[2];
        fast_block<P, D, QM, true, true>(s, m, l, uii, pop, L, me.pos - kt * kBK - krow, c, rest);
        add_values<P, D>(Vs, krow, 0, pop, rest, oacc, L);
      } else {
        fast_block<P, D, QM, true>(s, m, l, uii, pop, L, me.pos - kt * kBK - krow, c);
        add_values<P, D>(Vs, krow, 0, pop, oacc, L);
      }
      asm volatile("" ::: "memory");
      __builtin_amdgcn_s_waitcnt(0xc07f);  // the reads from LDS have ended
    }
    __syncthreads();  // bad_key is set
  } else {
    look_up<P>(a, trow, kt0, w, lane, jlast, id);
    const int phi = wrow < t.rows ? position_of(a, t, wrow + 31) : -1;  // the wave's last position
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
    load(kt0, KA, VA);                                  // kt0 is even
    const int kf = max(kt0, min(tlo / kBK, nkt));       // tiles before every row's position
    run_fast(kt0, kf, std::true_type{});
    run_fast(kf, nkt, std::false_type{});
  }
  if (bad != kNone) atomicMin(&bad_key, bad);
  // As in the fused forward pass the scan ran with the reference at 0, which is exact while the row total stays under
  // 2^64; 2^62 is asked for here, in every tile, so that the four parts of one of few rows stay under it together. Sums
  // that are not finite come from values that are not, perhaps behind the row.
  const float lt = l + xor32(l);
  float f = 0.0f;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) f = __builtin_fmaf(oacc[db][r], 0.0f, f);
  const bool again = me.live && (!(lt <= kSpecMax * 0.25f) || f != f);
  const bool any = __syncthreads_or(again ? 1 : 0);
  if (few && !any) {
    // the waves' sums meet in the tiles' memory, which the barrier has freed, and the first wave has them all
    if (w > 0) {
      float* z = reinterpret_cast<float*>(w == 1 ? VA : w == 2 ? KB : VB);
#pragma unroll
      for (int x = 0; x < 4 * DB; ++x)
        *reinterpret_cast<floatx4*>(z + (x * 64 + lane) * 4) =
            floatx4{oacc[x / 4][4 * (x % 4)], oacc[x / 4][4 * (x % 4) + 1], oacc[x / 4][4 * (x % 4) + 2],
                    oacc[x / 4][4 * (x % 4) + 3]};
      shared_l[w][lane] = l;
      shared_u[w][lane] = uii;
    }
    __syncthreads();
    if (w > 0) return;
#pragma unroll
    for (int x = 0; x < 4 * DB; ++x) {
      const int at = (x * 64 + lane) * 16;
      const floatx4 z = (*reinterpret_cast<const floatx4*>(VA + at) + *reinterpret_cast<const floatx4*>(KB + at)) +
                        *reinterpret_cast<const floatx4*>(VB + at);
#pragma unroll
      for (int i = 0; i < 4; ++i) oacc[x / 4][4 * (x % 4) + i] += z[i];
    }
    l += (shared_l[1][lane] + shared_l[2][lane]) + shared_l[3][lane];
    uii += (shared_u[1][lane] + shared_u[2][lane]) + shared_u[3][lane];  // one wave has met the row's own key, the rest 0
  }
  const bool redo = any && (few ? w == 0 : wave_any(again));
  if (!redo && !(any && few)) finish_tile_row<P, D>(a, t, me, m, l, uii, oacc, bad_key, L);
  if (any) scan_again<P, D>(a, t, redo, bad_key, KA, VA, KB, VB);
}

// The slices of each row joined, with its Self entry (eqs. 12-13), by 16 lanes of 8 channels each: what is the same for
// all channels of a row, most of the work, is done for four rows by one instruction. (A wave a row: 26 us against 13 for
// 25216 rows x 128 of four slices.)
template <class P>
__global__ __launch_bounds__(kNT) void prefill_merge_kernel(PagedPrefillArgs a) {
  using TI = typename P::T;
  constexpr int kLanes = 16, kBatch = 4;
  const int64_t rows = (int64_t)a.N * a.Hq, mine = (int64_t)blockIdx.x * (kNT / kLanes) + threadIdx.x / kLanes;
  const int64_t at = min(mine, rows - 1);  // whole waves reach the lane moves
  const int sub = threadIdx.x & (kLanes - 1), D = a.c.D, c0 = 8 * sub;
  // the first states are on their way while the row's request is looked up; those that nobody wrote count for nothing
  float2 ml[kBatch], zo[kBatch][4];
  auto load = [&](int s0, int last) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const float* st = a.states + ((int64_t)min(s0 + u, last) * rows + at) * (D + 2);  // 8-byte aligned
      ml[u] = *reinterpret_cast<const float2*>(st);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        zo[u][i] = float2{0.0f, 0.0f};
        if (c0 + 2 * i < D) zo[u][i] = *reinterpret_cast<const float2*>(st + 2 + c0 + 2 * i);
      }
    }
  };
  load(0, a.nsplit - 1);
  const int tok = (int)(at / a.Hq), hq = (int)(at - (int64_t)tok * a.Hq);
  // the number of requests that end at or before the token: 16 places of their ends at a time
  int b = 0;
#pragma unroll
  for (int step = 256; step; step /= 16) {
    const int i = b + (sub + 1) * step;
    const unsigned long long end = __ballot(i <= a.B && a.row_start[min(i, a.B)] <= tok);
    b += step * (int)__popc((unsigned)(end >> (threadIdx.x & 48)) & 0xffffu);
  }
  int first = 0, n = 0, pos = -1;
  const int bb = min(b, a.B - 1);
  n = tokens_of(a, bb, first);
  const bool is = b < a.B && tok >= first && tok < first + n && mine < rows;  // else a token of no request
  const int len = a.lengths[bb];
  if (is && len >= n && len <= a.max_len) pos = len - n + tok - first;
  // Self
  int64_t off = 0;
  const bool ok = pos >= 0 && entry_offset(a, bb, hq / a.G, pos, off);
  floatx4 v[2] = {};
  float dot = 0.0f;
#pragma unroll
  for (int i = 0; i < 2; ++i) {  // widths are multiples of 4
    if (ok && c0 + 4 * i < D) {
      const floatx4 x = P::load4((const TI*)a.q + at * D + c0 + 4 * i), y = P::load4((const TI*)a.k + off + c0 + 4 * i);
      v[i] = P::load4((const TI*)a.v + off + c0 + 4 * i);
#pragma unroll
      for (int e = 0; e < 4; ++e) dot = __builtin_fmaf(x[e], y[e], dot);
    }
  }
  dot = lane_group_sum<kLanes>(dot);
  const int ns = pos > 0 ? (pos - 1) / a.slice + 1 : 0;  // slices with an Exchange key
  float m = 0.0f, l = 0.0f, z[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) z[e] = 0.0f;
  for (int s0 = 0; s0 < ns; s0 += kBatch) {
    if (s0) load(s0, ns - 1);
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      if (s0 + u >= ns) break;
      const float zu[8] = {zo[u][0].x, zo[u][0].y, zo[u][1].x, zo[u][1].y, zo[u][2].x, zo[u][2].y, zo[u][3].x, zo[u][3].y};
      merge_into<8>(m, l, z, ml[u].x, ml[u].y, zu);
    }
  }
  if (!is) return;
  const float lam = *a.lambda, ln_i = logf((float)(pos + 1));
  const RowEpilogue ep = row_epilogue(m, l, dot * a.scale * kLog2e, a.inv_tau, lam, ln_i);
  const bool lost = !ok || l != l;  // a bad length, a page outside the pool, or a NaN among the keys
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    floatx4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      y[e] = lost ? __builtin_nanf("") : __builtin_fmaf(ep.omg, v[i][e], ep.inv_l * z[4 * i + e]);
    if (c0 + 4 * i < D) P::store4((TI*)a.out + at * D + c0 + 4 * i, y);
  }
  if (sub == 0 && a.row_stat) a.row_stat[at] = lost ? __builtin_nanf("") : ep.lnZ + lam * ln_i;
}

template <class P, int D>
hipError_t launch_one(PagedPrefillArgs a, hipStream_t stream) {
  a.tiles = (int)((int64_t)a.N * a.G / a.tile_rows + a.B);  // each request has one that is not whole
  a.map = make_tilemap(a.c.H, a.tiles * a.nsplit);
  hipLaunchKernelGGL((prefill_kernel<P, D>), dim3((unsigned)grid_size(a.map)), dim3(kNT), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.nsplit == 1) return e;
  const int64_t rows = (int64_t)a.N * a.Hq;
  using M = std::conditional_t<sizeof(typename P::T) == 2, PolBF16<32>, PolF32<32>>;  // its loads and stores, of any width
  hipLaunchKernelGGL((prefill_merge_kernel<M>), dim3((unsigned)((rows + kNT / 16 - 1) / (kNT / 16))), dim3(kNT), 0,
                     stream, a);
  return hipGetLastError();
}

}  // namespace

// Rows of a tile and slices of the histories, by sizes alone (the lengths are device data), so that the chip is full.
// * Tiles of 32 rows where tiles of 128 would not give every CU one and the histories are short, and, where requests
//   have 64 rows and more, up to two tiles a CU of 64 channels, five for four CUs of more. One prompt of 2048 tokens, 8
//   heads x 64, 27 us against 33 in slices of 128-row tiles, four of 1536 39 against 46 (416 tiles), two of 3000 60 against
//   63 (384); 8 heads x 128, one of 4096 93 against 95 (264), but four of 1536 71 against 61 (416); five chunks of 151 to 301
//   tokens after up to 777, 8 heads x 80 in fp32, 87 against 109. With longer histories the keys that every tile reads
//   again cost more than slices of 128-row tiles: a chunk of 64 tokens after 16384, 8 heads x 64, takes 31 us in 32 slices,
//   274 in one.
// * As many slices as bring the workgroups to what the chip holds at once (three a CU for bf16 of up to 64 channels,
//   else two), each of 512 keys or more: a chunk of 2048 after 32768, 16 heads on 4 x 128, 687 to 716 us in two slices,
//   903 to 927 in one, 683 to 706 in four; 7 chunks of 128 to 256 after up to 4096 78 in four, 124 in one. Tiles of 32
//   rows that give every CU one are not split: a merge costs more than is won (13 us for 25216 rows of four slices).
PrefillPlan paged_prefill_plan(int64_t N, int64_t B, int64_t H, int64_t G, int64_t max_len, int D, int dtype) {
  constexpr int64_t kMinSlice = 512;
  const int64_t kTarget = dtype == 1 && D <= 64 ? 768 : 512;  // what the chip holds at once
  PrefillPlan p;
  auto groups = [&](int64_t rows) { return (N * G / rows + B) * H; };
  const int64_t scarce = N * G < 64 * B ? 256 : D <= 64 ? 512 : 320;
  p.tile_rows = groups(kRows) <= scarce && max_len <= 4096 ? kFewRows : kRows;
  const int64_t have = groups(p.tile_rows);
  int64_t split = p.tile_rows == kFewRows && have >= 256 ? 1 : (kTarget + have - 1) / have;
  const int64_t most = (max_len + kMinSlice - 1) / kMinSlice;
  if (split > most) split = most;
  int64_t slice = (max_len + split - 1) / split;
  slice = (slice + 2 * kBK - 1) / (2 * kBK) * (2 * kBK);  // pairs of tiles
  p.slice = (int)slice;
  p.nsplit = (int)((max_len + slice - 1) / slice);
  return p;
}

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
  if (D <= 96) return launch_one<PolF32<128>, 96>(a, stream);  // rows as for 128, three quarters of the products
  return launch_one<PolF32<128>, 128>(a, stream);
}

}  // namespace rel
