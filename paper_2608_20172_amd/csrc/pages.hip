// Block tables and slot maps of a serving step, and the rows of its tokens
// written into a paged cache.
#include "kernels.h"
#include "serve.h"

namespace rel {

namespace {

// ---------------------------------------------------------------------------
// Page map. With c_b tokens cached and a_b added, request b needs
//   need_b = ceil((c_b + a_b) / p) - ceil(c_b / p)
// pages, and takes them from the free list at the sum of the needs before it;
// its tokens stand at the sum of the a's before it. Both sums are one scan over
// the batch, which every workgroup makes for itself in LDS (8 bytes a request
// read, no second launch and no pass through memory between them); then a
// thread finds its token's request by bisection of the ends.
// Latency-bound: a launch, two dependent reads (lengths, then page ids) and the
// scan. Sums are held at kFull, over any bound that they are compared with, so
// that they stay in 32 bits whatever the counts.
// ---------------------------------------------------------------------------
constexpr int kMapT = 256;
constexpr unsigned kFull = (1u << 30) + 1;

__device__ __forceinline__ unsigned add_full(unsigned x, unsigned y) { return min(x + y, kFull); }

// first b in [0, B) with x[b] > v (x ascending); B if none
__device__ __forceinline__ int first_above(const unsigned* x, int B, unsigned v) {
  int lo = 0, hi = B;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (x[mid] > v)
      hi = mid;
    else
      lo = mid + 1;
  }
  return lo;
}

__global__ __launch_bounds__(kMapT) void page_map_kernel(PageMapArgs a) {
  constexpr int NW = kMapT / 64;
  extern __shared__ unsigned lds[];
  unsigned* end = lds;           // [B] sums of tokens; before the scan the count itself
  unsigned* pages = lds + a.B;   // [B] sums of needs
  int* held = (int*)(lds + 2 * a.B);  // [B] tokens cached, -1 where the request is not served
  __shared__ unsigned wsum[2][NW];
  __shared__ int total[3][NW];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int64_t p1 = (1 << a.shift) - 1;
  const bool first_wg = blockIdx.x == 0;
  const int per = (a.B + kMapT - 1) / kMapT;
  const int b0 = min(tid * per, a.B), b1 = min(b0 + per, a.B);
  unsigned t = 0, n = 0;
  for (int b = b0; b < b1; ++b) {
    const int64_t c = a.cached[b], add = a.added[b];
    const int64_t have = (c + p1) >> a.shift, want = (c + add + p1) >> a.shift;
    const bool valid = c >= 0 && add >= 0 && want <= a.W;
    end[b] = add > 0 ? min((unsigned)add, kFull) : 0;
    pages[b] = valid ? (unsigned)(want - have) : 0;
    held[b] = valid ? (int)c : -1;
    t = add_full(t, end[b]);
    n = add_full(n, pages[b]);
  }
  const unsigned t0 = t, n0 = n;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const unsigned tt = __shfl_up(t, o, 64), nn = __shfl_up(n, o, 64);
    if (lane >= o) {
      t = add_full(t, tt);
      n = add_full(n, nn);
    }
  }
  if (lane == 63) {
    wsum[0][w] = t;
    wsum[1][w] = n;
  }
  // the sums before this thread's requests: those of the lane before, and of the waves before
  t = __shfl_up(t, 1, 64);
  n = __shfl_up(n, 1, 64);
  if (lane == 0) t = n = 0;
  __syncthreads();
#pragma unroll
  for (int x = 0; x < NW; ++x) {
    if (x < w) {
      t = add_full(t, wsum[0][x]);
      n = add_full(n, wsum[1][x]);
    }
  }
  int taken = 0, mapped = 0, refused = 0;
  for (int b = b0; b < b1; ++b) {
    const unsigned tokens = end[b], need = pages[b];
    t = add_full(t, tokens);
    n = add_full(n, need);
    const bool served = held[b] >= 0 && (tokens == 0 || t <= (unsigned)a.N) && (need == 0 || n <= (unsigned)a.F);
    if (first_wg) {
      a.lengths[b] = served ? held[b] + (int)tokens : 0;
      a.row_start[b + 1] = (int)min(t, (unsigned)a.N);
      taken += served ? (int)need : 0;
      mapped += served ? (int)tokens : 0;
      refused += !served;
    }
    end[b] = t;
    pages[b] = n;
    if (!served) held[b] = -1;
  }
  if (first_wg) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
      taken += __shfl_xor(taken, o, 64);
      mapped += __shfl_xor(mapped, o, 64);
      refused += __shfl_xor(refused, o, 64);
    }
    if (lane == 0) {
      total[0][w] = taken;
      total[1][w] = mapped;
      total[2][w] = refused;
    }
  }
  __syncthreads();
  if (first_wg && tid < 3) {
    int s = 0;
    for (int x = 0; x < NW; ++x) s += total[tid][x];
    a.counts[tid] = s;
    if (tid == 0) a.row_start[0] = 0;
  }

  // pages taken, in the order of the free list
  const int64_t stride = (int64_t)gridDim.x * kMapT, first = (int64_t)blockIdx.x * kMapT + tid;
  const int avail = a.B ? (int)min(pages[a.B - 1], (unsigned)a.F) : 0;
  for (int64_t i = first; i < avail; i += stride) {
    const int id = a.free_pages[i];
    const int b = first_above(pages, a.B, (unsigned)i);
    if (held[b] >= 0) {
      const int64_t have = (held[b] + p1) >> a.shift;
      a.table[(int64_t)b * a.W + have + (i - (b ? pages[b - 1] : 0))] = id;
    }
  }

  // tokens
#pragma unroll 4
  for (int64_t i = first; i < a.N; i += stride) {
    int64_t slot = -1;
    int pos = -1;
    const int b = first_above(end, a.B, (unsigned)i);
    if (b < a.B && held[b] >= 0) {
      pos = held[b] + (int)(i - (b ? end[b - 1] : 0));
      const int j = pos >> a.shift, have = (int)((held[b] + p1) >> a.shift);
      // a page of this step is read from the free list: its table entry may not be written yet
      const int64_t id = j < have ? a.table[(int64_t)b * a.W + j] : a.free_pages[(b ? pages[b - 1] : 0) + (unsigned)(j - have)];
      slot = id * (1 << a.shift) + (pos & (int)p1);
    }
    a.slots[i] = slot;
    a.positions[i] = pos;
  }
}

// ---------------------------------------------------------------------------
// Rows into the cache. One workgroup takes `tpw` tokens: cos and sin of their
// channel pairs go to LDS once (the angle in 64-bit turns, so that a long
// context keeps its fraction), then the rows of all heads are moved by threads
// that hold a chunk of the first half and the one it turns with. Every channel
// is read and written once: bound by memory.
// Chunks are of 16 bytes whatever the width and the alignment: the last chunk of
// a half is moved back to end with it, and repeats some channels of the one before
// (the same values into the same places). 16384 tokens of 12 heads in bf16: width
// 64 33 us (151 MB, 4.6 TB/s); width 60 in a cache of 64 51 us (146 MB), 64 with
// 4-byte chunks, which divide a half of 30.
// ---------------------------------------------------------------------------
constexpr int kAppT = 256;
constexpr int kAppMaxTokens = 8;

// VEC elements (16 bytes, or one) on any element boundary, as floats.
template <typename TI, int VEC>
__device__ __forceinline__ void load_vec(const TI* p, float (&x)[VEC]) {
  if constexpr (VEC == 1) {
    x[0] = (float)*p;
  } else if constexpr (sizeof(TI) == 2) {
    typedef unsigned int U __attribute__((ext_vector_type(4), aligned(2)));
    const U u = *reinterpret_cast<const U*>(p);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[2 * e] = bf16_lo(u[e]);
      x[2 * e + 1] = bf16_hi(u[e]);
    }
  } else {
    typedef float V __attribute__((ext_vector_type(4), aligned(4)));
    const V u = *reinterpret_cast<const V*>(p);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = u[e];
  }
}
template <typename TI, int VEC>
__device__ __forceinline__ void store_vec(TI* p, const float (&x)[VEC]) {
  if constexpr (VEC == 1) {
    *p = (TI)x[0];
  } else if constexpr (sizeof(TI) == 2) {
    typedef unsigned int U __attribute__((ext_vector_type(4), aligned(2)));
    bf16x8 o;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = (bf16)x[e];
    *reinterpret_cast<U*>(p) = __builtin_bit_cast(uintx4, o);
  } else {
    typedef float V __attribute__((ext_vector_type(4), aligned(4)));
    *reinterpret_cast<V*>(p) = V{x[0], x[1], x[2], x[3]};
  }
}

template <typename TI, int VEC>
__global__ __launch_bounds__(kAppT) void append_kernel(AppendArgs a, int tpw) {
  extern __shared__ float2 cs[];  // [tpw][D / 2]
  __shared__ int64_t row0[kAppMaxTokens];  // cache offset of the token's first head, or -1: not written
  const int tid = threadIdx.x;
  const int n0 = blockIdx.x * tpw, nt = min(tpw, a.N - n0);
  const int half = a.D >> 1, Dc = a.c.D;
  if (tid < nt) {
    const int64_t slot = a.slots[n0 + tid];
    const bool in = a.positions[n0 + tid] >= 0 && slot >= 0 && (slot >> a.c.shift) < a.c.num_pages;
    row0[tid] = in ? (slot >> a.c.shift) * a.c.sp + (slot & ((1 << a.c.shift) - 1)) * (int64_t)a.c.st : -1;
  }
  if (a.rope) {
    for (int i = tid; i < nt * half; i += kAppT) {
      const int n = i / half, j = i - n * half;
      const double x = (double)a.positions[n0 + n] * a.turns[j];
      const float f = (float)(2.0 * (x - rint(x)));  // half turns in [-1, 1]
      float s, c;
      sincospif(f, &s, &c);
      cs[i] = make_float2(c, s);
    }
  }
  __syncthreads();
  const int nq = a.q ? a.Hq : 0, heads = nq + a.c.H;
  // q and k: tasks (token, head, chunk), a chunk of each half with RoPE
  const int run = a.rope ? half : a.D, ch = (run + VEC - 1) / VEC;
  for (int i = tid; i < nt * heads * ch; i += kAppT) {
    const int c = i % ch, nh = i / ch, h = nh % heads, n = nh / heads;
    const bool isq = h < nq;
    const int64_t r0 = row0[n];
    if (!isq && r0 < 0) continue;
    const int hk = h - nq;
    const TI* src = isq ? (const TI*)a.q + (n0 + n) * a.q_token + h * a.q_head
                        : (const TI*)a.k + (n0 + n) * a.kv_token + hk * a.kv_head;
    TI* dst = isq ? (TI*)a.q_out + ((int64_t)(n0 + n) * a.Hq + h) * Dc : (TI*)a.k_cache + r0 + (int64_t)hk * a.c.sh;
    const int e0 = min(c * VEC, run - VEC);
    float x[VEC], y[VEC];
    load_vec<TI, VEC>(src + e0, x);
    if (a.rope) {
      load_vec<TI, VEC>(src + half + e0, y);
      float u[VEC], v[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float2 t = cs[n * half + e0 + e];
        u[e] = x[e] * t.x - y[e] * t.y;
        v[e] = x[e] * t.y + y[e] * t.x;
      }
      if (r0 < 0) {  // a token of no request
#pragma unroll
        for (int e = 0; e < VEC; ++e) u[e] = v[e] = 0.0f;
      }
      store_vec<TI, VEC>(dst + e0, u);
      store_vec<TI, VEC>(dst + half + e0, v);
    } else {
      if (r0 < 0) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) x[e] = 0.0f;
      }
      store_vec<TI, VEC>(dst + e0, x);
    }
  }
  // v: a head pair's chunk with Givens mixing, else one head's
  const int vch = (a.D + VEC - 1) / VEC, vh = a.givens ? a.c.H / 2 : a.c.H;
  for (int i = tid; i < nt * vh * vch; i += kAppT) {
    const int c = i % vch, nh = i / vch, h = nh % vh, n = nh / vh;
    const int64_t r0 = row0[n];
    if (r0 < 0) continue;
    const int e0 = min(c * VEC, a.D - VEC);
    const TI* src = (const TI*)a.v + (n0 + n) * a.kv_token + e0;
    TI* dst = (TI*)a.v_cache + r0 + e0;
    float x[VEC], y[VEC];
    if (a.givens) {
      const int p = 2 * h + (a.givens == 2 ? 1 : 0), p2 = p + 1 == a.c.H ? 0 : p + 1;
      float sn, cn;
      sincosf(a.theta[h], &sn, &cn);
      load_vec<TI, VEC>(src + p * a.kv_head, x);
      load_vec<TI, VEC>(src + p2 * a.kv_head, y);
      float u[VEC], v[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        u[e] = cn * x[e] - sn * y[e];
        v[e] = sn * x[e] + cn * y[e];
      }
      store_vec<TI, VEC>(dst + (int64_t)p * a.c.sh, u);
      store_vec<TI, VEC>(dst + (int64_t)p2 * a.c.sh, v);
    } else {
      load_vec<TI, VEC>(src + h * a.kv_head, x);
      store_vec<TI, VEC>(dst + (int64_t)h * a.c.sh, x);
    }
  }
  // zeros in channels D .. Dc - 1, as words where the element is half a word and D even
  const int words = sizeof(TI) == 2 && a.D % 2 == 0;
  const int pad = words ? (Dc - a.D) / 2 : Dc - a.D, ph = nq + 2 * a.c.H;
  for (int i = tid; i < nt * ph * pad; i += kAppT) {
    const int e = a.D + (i % pad << words), nh = i / pad, h = nh % ph, n = nh / ph;
    const int64_t r0 = row0[n];
    if (h >= nq && r0 < 0) continue;
    TI* dst = h < nq            ? (TI*)a.q_out + ((int64_t)(n0 + n) * a.Hq + h) * Dc
              : h < nq + a.c.H  ? (TI*)a.k_cache + r0 + (int64_t)(h - nq) * a.c.sh
                                : (TI*)a.v_cache + r0 + (int64_t)(h - nq - a.c.H) * a.c.sh;
    if (words)
      *reinterpret_cast<unsigned int*>(dst + e) = 0;
    else
      dst[e] = (TI)0.0f;
  }
}

template <typename TI, int VEC>
hipError_t append_t(const AppendArgs& a, hipStream_t stream) {
  const int tpw = a.N >= 4096 ? kAppMaxTokens : 1;
  hipLaunchKernelGGL((append_kernel<TI, VEC>), dim3((unsigned)((a.N + tpw - 1) / tpw)), dim3(kAppT),
                     (size_t)tpw * (a.D / 2) * sizeof(float2), stream, a, tpw);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_page_map(const PageMapArgs& a, hipStream_t stream) {
  // a token per thread: 64 requests and 69 tokens 4.1 us, 96 and 66000 4.9 (8.4 with four tokens a thread)
  const int64_t want = ((int64_t)a.N + kMapT - 1) / kMapT;
  const unsigned grid = (unsigned)(want < 1 ? 1 : want > 2048 ? 2048 : want);
  hipLaunchKernelGGL(page_map_kernel, dim3(grid), dim3(kMapT), (size_t)a.B * 12, stream, a);
  return hipGetLastError();
}

hipError_t launch_append(const AppendArgs& a, int dtype, hipStream_t stream) {
  const int run = a.rope ? a.D / 2 : a.D, vec = dtype == 1 ? 8 : 4;
  if (run >= vec) return dtype == 1 ? append_t<bf16, 8>(a, stream) : append_t<float, 4>(a, stream);
  return dtype == 1 ? append_t<bf16, 1>(a, stream) : append_t<float, 1>(a, stream);  // narrower than a chunk
}

}  // namespace rel
