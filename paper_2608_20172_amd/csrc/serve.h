// Internal launch interface of the serving kernels: page maps, rows into a
// paged cache, the decode step and chunks of new tokens over pages, and sampling.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.h"

namespace rel {

// A paged cache as the kernels see it: row (page, head, offset) of D elements
// at page * sp + head * sh + offset * st. A page spans less than 2^31 elements.
struct PagedCache {
  int num_pages, shift;  // page_size = 1 << shift
  int64_t sp;
  int sh, st;
  int H, D;
};

// The largest batch of a page map: its scan lives in LDS, 12 bytes a request.
constexpr int kMapMaxB = 4096;

struct PageMapArgs {
  const int32_t* cached;
  const int32_t* added;
  const int32_t* free_pages;
  int32_t* table;      // [B, W]
  int32_t* lengths;    // [B]
  int32_t* row_start;  // [B + 1]
  int64_t* slots;      // [N]
  int32_t* positions;  // [N]
  int32_t* counts;     // pages taken, tokens mapped, requests not served
  int B, W, shift, N, F;
};
hipError_t launch_page_map(const PageMapArgs& a, hipStream_t stream);

struct AppendArgs {
  const void* q;       // [N, Hq, D] with (q_token, q_head), or null
  const void* k;       // [N, H, D] with (kv_token, kv_head)
  const void* v;
  const int64_t* slots;
  const int32_t* positions;
  const float* theta;  // [H / 2] (givens != 0)
  void* q_out;         // [N, Hq, c.D] dense
  void* k_cache;
  void* v_cache;
  PagedCache c;        // c.D: the cache's width >= D
  int64_t q_token, q_head, kv_token, kv_head;
  int N, Hq, D;
  int givens;          // 0 none, 1 pairing A, 2 pairing B
  int rope;            // 1: rotate q and k
  double turns[64];    // turns of channel pair j per position: base^(-2j/D) / (2 pi)
};
hipError_t launch_append(const AppendArgs& a, int dtype, hipStream_t stream);

struct PagedDecodeArgs {
  const void* q;           // [B, Hq, D] dense
  const void* k;
  const void* v;
  const int32_t* table;    // [B, W]
  const int32_t* lengths;  // [B]
  const float* lambda;
  PagedCache c;
  int B, Hq, G, W;         // Hq = G * c.H
  int max_len;             // lengths above it are refused (NaN)
  int nsplit, slice;       // slices of `slice` keys
  int placed;              // 1: workgroups that share cache lines on one die (set by the launch)
  float scale, inv_tau;
  float* states;           // [nsplit][B Hq][D + 2] (nsplit > 1)
  void* out;               // [B, Hq, D] dense
  float* row_stat;         // [B, Hq] or null
};
// Slices of a step: slice length and their number, by the host's bounds alone.
void paged_decode_split(int64_t B, int64_t H, int64_t G, int64_t max_len, int D, int dtype, int* slice, int* nsplit);
hipError_t launch_paged_decode(const PagedDecodeArgs& a, int dtype, hipStream_t stream);

struct PagedPrefillArgs {
  const void* q;             // [N, Hq, D] dense
  const void* k;
  const void* v;
  const int32_t* table;      // [B, W]
  const int32_t* lengths;    // [B]
  const int32_t* row_start;  // [B + 1]
  const float* lambda;
  PagedCache c;
  int B, N, Hq, G, W;        // Hq = G * c.H
  int max_len;               // lengths above it are refused (NaN)
  float scale, inv_tau;
  void* out;                 // [N, Hq, D] dense
  float* row_stat;           // [N, Hq] or null
  float* states;             // [nsplit][N Hq][D + 2] (nsplit > 1)
  int tile_rows;             // rows of a tile
  int nsplit, slice;         // slices of `slice` keys
  int tiles;                 // at most so many tiles (set by the launch)
  TileMap map;               // key heads x tiles x slices (set by the launch)
};
// The largest batch: every workgroup finds its tile by a scan over the requests.
constexpr int kPrefillMaxB = 4096;
struct PrefillPlan {
  int tile_rows, nsplit, slice;
};
// How a step is cut, by the host's bounds alone.
PrefillPlan paged_prefill_plan(int64_t N, int64_t B, int64_t H, int64_t G, int64_t max_len, int D, int dtype);
hipError_t launch_paged_prefill(const PagedPrefillArgs& a, int dtype, hipStream_t stream);

struct SampleArgs {
  const void* logits;        // [B, V] with row stride `sl`
  const float* noise;        // [B, V] with row stride `sn`
  int64_t sl, sn;
  const float* temperature;  // [B] each, or null: 1 / off / off / off
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  int64_t* tokens;           // [B]
  float* logprob;            // [B] or null
  int B, V;
  void* ws;
};
constexpr int64_t kSampleMaxV = 1 << 22;  // the largest row
size_t sample_workspace_bytes(int64_t B, int64_t V, int dtype);
hipError_t launch_sample(const SampleArgs& a, int dtype, hipStream_t stream);

}  // namespace rel
