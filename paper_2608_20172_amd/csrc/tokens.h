// Internal launch interface of the operators around the mixer that go token by
// token: norms and rotation of query and key heads, log-probabilities of tokens.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.h"

namespace rel {

struct Strides {
  int64_t b, h, t;
};

// One of the two tensors of a call.
struct NormTensor {
  const void* x;     // [B, H, T, D]
  const void* w;     // [D] or null
  const void* dy;    // backward: the gradient that comes in
  void* y;           // forward: the output; backward: the gradient of x
  Strides sx, sdy, sy;
  float* dw;         // backward: [D] or null
  int H;             // 0: absent
};
struct QkNormArgs {
  NormTensor s[2];
  const int32_t* positions;  // or null: 0 .. T - 1
  int64_t position_stride;
  int64_t tokens;            // B T
  int T, D;
  int rope_dim, interleaved, norm, weight_bf16;
  float eps, amplitude;
  float* ws;                 // backward: partial sums of the weights' gradients, [D][groups] of either tensor
  int groups[2];             // workgroups of either tensor (set by the launch)
  double turns[64];          // turns of channel pair j per position
};
// The most workgroups that the backward pass has of one tensor, each with a partial sum of every channel.
int qk_norm_groups(int64_t tokens);
hipError_t launch_qk_norm_fwd(const QkNormArgs& a, int dtype, hipStream_t stream);
hipError_t launch_qk_norm_bwd(const QkNormArgs& a, int dtype, hipStream_t stream);

struct LogprobArgs {
  const void* logits;     // [N, V] with row stride sl
  const int64_t* tokens;  // [N]
  int64_t sl;
  float* logprob;         // each may be null
  float* entropy;
  int32_t* rank;
  int64_t* top_tokens;    // [N, K] (K > 0)
  float* top_logprobs;
  float* stats;           // [N, 4]
  int N, V, K;
  void* ws;
};
struct LogprobGradArgs {
  const void* logits;
  const int64_t* tokens;
  const float* stats;
  const float* dlogprob;  // or null
  const float* dentropy;  // or null
  void* dlogits;          // [N, V] with row stride sg
  int64_t sl, sg;
  int N, V;
};
constexpr int64_t kLogprobMaxV = 1 << 22;
constexpr int kLogprobMaxK = 32;
// Bytes that a call needs, and enough for every call of up to N rows.
size_t logprobs_scratch_bytes(int64_t N, int64_t V, int64_t K, int dtype);
size_t logprobs_workspace_bytes(int64_t N, int64_t V, int64_t K, int dtype);
hipError_t launch_logprobs_fwd(const LogprobArgs& a, int dtype, hipStream_t stream);
hipError_t launch_logprobs_bwd(const LogprobGradArgs& a, int dtype, hipStream_t stream);

}  // namespace rel
