// C-ABI layer of the operators that go token by token: norms and rotation of query
// and key heads, log-probabilities of given tokens. Arguments are checked on the
// host; device data (positions, tokens) where the kernels read it.
#include "../../include/relation.h"

#include <algorithm>
#include <cmath>

#include "api_checks.h"
#include "tokens.h"

namespace {

constexpr int64_t kFarStride = 1LL << 40;

// Elements from the first to past the last of a [B, H, T, D] tensor.
int64_t extent(const rel_qk_norm* p, int64_t H, const rel_strides& s) {
  return (p->B - 1) * s.b + (H - 1) * s.h + (p->T - 1) * s.t + p->D;
}
rel::ApiLattice lattice(const rel_qk_norm* p, int64_t H, const rel_strides& s) {
  return {{s.b, s.h, s.t}, {p->B, H, p->T}, p->D};
}

rel_status check_strides(const rel_qk_norm* p, int64_t H, const rel_strides& s, const char* name, bool output) {
  if (s.b < 0 || s.h < 0 || s.t < 0) return api_fail(REL_ERR_INVALID_ARG, "negative stride of %s", name);
  const int64_t count[3] = {p->B, H, p->T}, stride[3] = {s.b, s.h, s.t};
  for (int i = 0; i < 3; ++i)
    if (stride[i] > kFarStride || (count[i] > 1 && stride[i] > kFarStride / (count[i] - 1)))
      return api_fail(REL_ERR_UNSUPPORTED, "%s spans over 2^40 elements", name);
  if (output && !rel::api_nested(lattice(p, H, s)))
    return api_fail(REL_ERR_INVALID_ARG, "strides make distinct rows of %s overlap", name);
  return REL_OK;
}

rel_status check_norm(const rel_qk_norm* p, bool* empty) {
  if (!p) return api_fail(REL_ERR_INVALID_ARG, "norm description is null");
  if (p->B < 0 || p->T < 0 || p->Hq < 0 || p->H < 0) return api_fail(REL_ERR_INVALID_ARG, "negative size");
  for (int32_t d : {p->dtype, p->weight_dtype})
    if (d != REL_F32 && d != REL_BF16) return api_fail(REL_ERR_UNSUPPORTED, "unknown dtype %d", (int)d);
  if (p->D < 1 || p->D > 128) return api_fail(REL_ERR_UNSUPPORTED, "head width %lld is not in 1..128", (long long)p->D);
  if (p->norm != 0 && p->norm != 1) return api_fail(REL_ERR_INVALID_ARG, "norm must be 0 or 1");
  if (p->norm && !(std::isfinite(p->eps) && p->eps > 0.0f))
    return api_fail(REL_ERR_INVALID_ARG, "eps must be finite and > 0 (got %g)", (double)p->eps);
  if (p->rope_dim < 0 || p->rope_dim > p->D || p->rope_dim % 2)
    return api_fail(REL_ERR_INVALID_ARG, "rope_dim must be even, from 0 to the head width (got %lld)", (long long)p->rope_dim);
  if (p->rope_dim) {
    if (p->layout != REL_ROPE_HALF && p->layout != REL_ROPE_INTERLEAVED)
      return api_fail(REL_ERR_INVALID_ARG, "unknown layout %d of the rotated pairs", (int)p->layout);
    if (!(std::isfinite(p->rope_base) && p->rope_base > 1.0))
      return api_fail(REL_ERR_INVALID_ARG, "rope_base must be finite and over 1");
    if (!(std::isfinite(p->factor) && p->factor >= 1.0))
      return api_fail(REL_ERR_INVALID_ARG, "factor must be finite and at least 1");
    if (p->original_length < 0) return api_fail(REL_ERR_INVALID_ARG, "negative original_length");
    if (!(std::isfinite(p->low) && std::isfinite(p->high) && p->low < p->high))
      return api_fail(REL_ERR_INVALID_ARG, "low and high must be finite, low the smaller");
    if (!std::isfinite(p->amplitude)) return api_fail(REL_ERR_INVALID_ARG, "amplitude must be finite");
  }
  *empty = p->B == 0 || p->T == 0 || (p->Hq == 0 && p->H == 0);
  if (*empty) return REL_OK;
  if (p->B > (1 << 30) || p->T > (1 << 30) || p->B * p->T > (1 << 26) || p->Hq > (1 << 16) || p->H > (1 << 16))
    return api_fail(REL_ERR_UNSUPPORTED, "over 2^26 tokens or 2^16 heads");
  if (p->position_stride < 0 || (p->position_stride && p->B > 1 && p->position_stride < p->T))
    return api_fail(REL_ERR_INVALID_ARG, "position_stride must be 0 or at least T");
  if (p->B > 1 && p->position_stride > kFarStride / (p->B - 1)) return api_fail(REL_ERR_UNSUPPORTED, "positions span over 2^40");
  return REL_OK;
}

// The rows of the two outputs share no element, as far as ranges and equal strides tell.
rel_status outputs_apart(const rel_qk_norm* p, const void* x, const rel_strides& sx, const char* nx, const void* y,
                         const rel_strides& sy, const char* ny) {
  if (!x || !y) return REL_OK;
  const size_t es = elem_size(p->dtype);
  const Range r[] = {{x, (size_t)extent(p, p->Hq, sx) * es, nx, true}, {y, (size_t)extent(p, p->H, sy) * es, ny, true}};
  if (disjoint(r, 2) == REL_OK) return REL_OK;
  // heads of one buffer: apart where both have its strides and the later ones start behind the earlier ones
  const bool same = (p->B == 1 || sx.b == sy.b) && sx.h == sy.h && (p->T == 1 || sx.t == sy.t) && sx.h > 0;
  const int64_t delta = (int64_t)((intptr_t)y - (intptr_t)x), step = sx.h * (int64_t)es;
  if (same && delta % step == 0) {
    const int64_t heads = delta / step;
    if (heads >= p->Hq && rel::api_nested(lattice(p, heads + p->H, sx))) return REL_OK;
    if (-heads >= p->H && rel::api_nested(lattice(p, -heads + p->Hq, sx))) return REL_OK;
  }
  return api_fail(REL_ERR_INVALID_ARG, "output %s overlaps %s", nx, ny);
}

void fill(rel::QkNormArgs& a, const rel_qk_norm* p, const int32_t* positions) {
  a.positions = positions;
  a.position_stride = p->B > 1 ? p->position_stride : 0;
  a.tokens = p->B * p->T;
  a.T = (int)p->T; a.D = (int)p->D;
  a.rope_dim = (int)p->rope_dim;
  a.interleaved = p->layout == REL_ROPE_INTERLEAVED;
  a.norm = p->norm; a.weight_bf16 = p->weight_dtype == REL_BF16;
  a.eps = p->eps; a.amplitude = p->amplitude;
  constexpr double tau = 6.283185307179586476925286766559;
  for (int j = 0; j < a.rope_dim / 2; ++j) {
    const double v = std::exp(-2.0 * j / a.rope_dim * std::log(p->rope_base));
    const double often = (double)p->original_length * v / tau;
    const double c = p->original_length ? std::min(std::max((often - p->low) / (p->high - p->low), 0.0), 1.0) : 0.0;
    a.turns[j] = p->factor == 1.0 ? v / tau : v * (c + (1.0 - c) / p->factor) / tau;
  }
}

rel::Strides strides_of(const rel_strides& s) { return {s.b, s.h, s.t}; }

}  // namespace

extern "C" {

rel_status relation_qk_norm_fwd(const rel_qk_norm* p, const void* q, const void* k, const void* q_weight,
                                const void* k_weight, const int32_t* positions, void* q_out, void* k_out, void* stream) {
  bool empty = false;
  REL_TRY(check_norm(p, &empty));
  if (empty) return REL_OK;
  const size_t es = elem_size(p->dtype), ws = elem_size(p->weight_dtype);
  const bool has[2] = {p->Hq > 0, p->H > 0};
  if (has[0]) {
    REL_TRY(check_strides(p, p->Hq, p->q, "q", false));
    REL_TRY(check_strides(p, p->Hq, p->q_out, "q_out", true));
  }
  if (has[1]) {
    REL_TRY(check_strides(p, p->H, p->k, "k", false));
    REL_TRY(check_strides(p, p->H, p->k_out, "k_out", true));
  }
  REL_TRY(aligned(q, es, "q", has[0]));
  REL_TRY(aligned(k, es, "k", has[1]));
  REL_TRY(aligned(q_out, es, "q_out", has[0]));
  REL_TRY(aligned(k_out, es, "k_out", has[1]));
  REL_TRY(aligned(q_weight, ws, "q_weight", false));
  REL_TRY(aligned(k_weight, ws, "k_weight", false));
  REL_TRY(aligned(positions, 4, "positions", false));
  const size_t pos = ((size_t)(p->B - 1) * (size_t)(p->B > 1 ? p->position_stride : 0) + (size_t)p->T) * 4;
  const Range in[] = {{q, has[0] ? (size_t)extent(p, p->Hq, p->q) * es : 0, "q", false},
                      {k, has[1] ? (size_t)extent(p, p->H, p->k) * es : 0, "k", false},
                      {q_weight, (size_t)p->D * ws, "q_weight", false},
                      {k_weight, (size_t)p->D * ws, "k_weight", false},
                      {positions, pos, "positions", false}};
  const Range out[] = {{has[0] ? q_out : nullptr, has[0] ? (size_t)extent(p, p->Hq, p->q_out) * es : 0, "q_out", true},
                       {has[1] ? k_out : nullptr, has[1] ? (size_t)extent(p, p->H, p->k_out) * es : 0, "k_out", true}};
  for (const Range& o : out) {
    Range r[6];
    std::copy(in, in + 5, r);
    r[5] = o;
    REL_TRY(disjoint(r, 6));
  }
  REL_TRY(outputs_apart(p, out[0].ptr, p->q_out, "q_out", out[1].ptr, p->k_out, "k_out"));
  if (rel::api_fail_launch()) return api_fail(REL_ERR_HIP, "HIP launch failure injected by RELATION_TEST_FAIL_LAUNCH");
  rel::QkNormArgs a{};
  fill(a, p, positions);
  a.s[0] = {q, q_weight, nullptr, q_out, strides_of(p->q), {}, strides_of(p->q_out), nullptr, (int)p->Hq};
  a.s[1] = {k, k_weight, nullptr, k_out, strides_of(p->k), {}, strides_of(p->k_out), nullptr, (int)p->H};
  return hip_status(rel::launch_qk_norm_fwd(a, p->dtype, (hipStream_t)stream), "qk norm launch");
}

size_t relation_qk_norm_bwd_workspace_bytes(const rel_qk_norm* p) {
  bool empty = false;
  if (check_norm(p, &empty) != REL_OK || empty || !p->norm) return 0;
  return (size_t)2 * (size_t)rel::qk_norm_groups(p->B * p->T) * (size_t)p->D * 4;
}

rel_status relation_qk_norm_bwd(const rel_qk_norm* p, const void* q, const void* k, const void* q_weight,
                                const void* k_weight, const int32_t* positions, const void* dq_out, const void* dk_out,
                                void* dq, void* dk, float* dq_weight, float* dk_weight, void* workspace,
                                size_t workspace_bytes, void* stream) {
  bool empty = false;
  REL_TRY(check_norm(p, &empty));
  if ((dq_weight || dk_weight) && !p->norm) return api_fail(REL_ERR_INVALID_ARG, "gradients of weights without a norm");
  const size_t es = elem_size(p->dtype), ws = elem_size(p->weight_dtype);
  const bool has[2] = {!empty && p->Hq > 0, !empty && p->H > 0};
  if (has[0]) {
    REL_TRY(check_strides(p, p->Hq, p->q, "q", false));
    REL_TRY(check_strides(p, p->Hq, p->q_out, "dq_out", false));
    REL_TRY(check_strides(p, p->Hq, p->dq, "dq", true));
  }
  if (has[1]) {
    REL_TRY(check_strides(p, p->H, p->k, "k", false));
    REL_TRY(check_strides(p, p->H, p->k_out, "dk_out", false));
    REL_TRY(check_strides(p, p->H, p->dk, "dk", true));
  }
  const size_t need = dq_weight || dk_weight ? relation_qk_norm_bwd_workspace_bytes(p) : 0;
  if (need && (!workspace || workspace_bytes < need))
    return api_fail(REL_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", need, workspace ? workspace_bytes : (size_t)0);
  REL_TRY(aligned(q, es, "q", has[0]));
  REL_TRY(aligned(k, es, "k", has[1]));
  REL_TRY(aligned(dq_out, es, "dq_out", has[0]));
  REL_TRY(aligned(dk_out, es, "dk_out", has[1]));
  REL_TRY(aligned(dq, es, "dq", has[0]));
  REL_TRY(aligned(dk, es, "dk", has[1]));
  REL_TRY(aligned(q_weight, ws, "q_weight", false));
  REL_TRY(aligned(k_weight, ws, "k_weight", false));
  REL_TRY(aligned(dq_weight, 4, "dq_weight", false));
  REL_TRY(aligned(dk_weight, 4, "dk_weight", false));
  REL_TRY(aligned(positions, 4, "positions", false));
  REL_TRY(aligned(workspace, 16, "workspace", need > 0));
  const size_t D = (size_t)p->D;
  auto span = [&](int i, const rel_strides& s) { return has[i] ? (size_t)extent(p, i ? p->H : p->Hq, s) * es : (size_t)0; };
  const size_t pos = empty ? 0 : ((size_t)(p->B - 1) * (size_t)(p->B > 1 ? p->position_stride : 0) + (size_t)p->T) * 4;
  const Range in[] = {{q, span(0, p->q), "q", false},
                      {k, span(1, p->k), "k", false},
                      {dq_out, span(0, p->q_out), "dq_out", false},
                      {dk_out, span(1, p->k_out), "dk_out", false},
                      {q_weight, D * ws, "q_weight", false},
                      {k_weight, D * ws, "k_weight", false},
                      {positions, pos, "positions", false}};
  const Range out[] = {{has[0] ? dq : nullptr, span(0, p->dq), "dq", true},
                       {has[1] ? dk : nullptr, span(1, p->dk), "dk", true}};
  const Range small[] = {{dq_weight, D * 4, "dq_weight", true}, {dk_weight, D * 4, "dk_weight", true},
                         {need ? workspace : nullptr, need, "workspace", true}};
  for (const Range& o : out) {
    Range r[11];
    std::copy(in, in + 7, r);
    std::copy(small, small + 3, r + 7);
    r[10] = o;
    REL_TRY(disjoint(r, 11));
  }
  if (!empty) REL_TRY(outputs_apart(p, out[0].ptr, p->dq, "dq", out[1].ptr, p->dk, "dk"));
  if (empty && !dq_weight && !dk_weight) return REL_OK;
  if (rel::api_fail_launch()) return api_fail(REL_ERR_HIP, "HIP launch failure injected by RELATION_TEST_FAIL_LAUNCH");
  rel::QkNormArgs a{};
  fill(a, p, positions);
  a.s[0] = {q, q_weight, dq_out, dq, strides_of(p->q), strides_of(p->q_out), strides_of(p->dq), dq_weight, has[0] ? (int)p->Hq : 0};
  a.s[1] = {k, k_weight, dk_out, dk, strides_of(p->k), strides_of(p->k_out), strides_of(p->dk), dk_weight, has[1] ? (int)p->H : 0};
  a.ws = (float*)workspace;
  if (empty) a.tokens = 0;
  return hip_status(rel::launch_qk_norm_bwd(a, p->dtype, (hipStream_t)stream), "qk norm backward launch");
}

static rel_status check_logprobs(const rel_token_logprobs* p, bool grad, bool* empty) {
  if (!p) return api_fail(REL_ERR_INVALID_ARG, "log-probability description is null");
  if (p->N < 0 || p->V < 0 || p->K < 0) return api_fail(REL_ERR_INVALID_ARG, "negative size");
  if (p->dtype != REL_F32 && p->dtype != REL_BF16) return api_fail(REL_ERR_UNSUPPORTED, "unknown dtype %d", (int)p->dtype);
  *empty = p->N == 0;
  if (*empty) return REL_OK;
  if (p->V < 1) return api_fail(REL_ERR_INVALID_ARG, "a row without tokens");
  if (p->V > rel::kLogprobMaxV || p->N > (1 << 20)) return api_fail(REL_ERR_UNSUPPORTED, "V is at most 2^22 and N at most 2^20");
  if (p->N * p->V > (1LL << 36)) return api_fail(REL_ERR_UNSUPPORTED, "N * V is over 2^36");
  if (!grad && p->K > rel::kLogprobMaxK) return api_fail(REL_ERR_UNSUPPORTED, "%lld alternatives: at most %d", (long long)p->K, rel::kLogprobMaxK);
  if (!grad && p->K > p->V) return api_fail(REL_ERR_INVALID_ARG, "more alternatives than tokens");
  if (p->N > 1 && p->stride_logits && p->stride_logits < p->V)
    return api_fail(REL_ERR_INVALID_ARG, "stride_logits must be 0 or at least V");
  if (grad && p->N > 1 && p->stride_grad < p->V) return api_fail(REL_ERR_INVALID_ARG, "stride_grad must be at least V");
  if (p->N > 1 && (p->stride_logits > kFarStride || (grad && p->stride_grad > kFarStride)))
    return api_fail(REL_ERR_UNSUPPORTED, "row stride over 2^40");
  return REL_OK;
}

size_t relation_token_logprobs_workspace_bytes(const rel_token_logprobs* p) {
  bool empty = false;
  if (check_logprobs(p, false, &empty) != REL_OK || empty) return 0;
  return rel::logprobs_workspace_bytes(p->N, p->V, p->K, p->dtype);
}

rel_status relation_token_logprobs_fwd(const rel_token_logprobs* p, const void* logits, const int64_t* tokens,
                                       float* logprob, float* entropy, int32_t* rank, int64_t* top_tokens,
                                       float* top_logprobs, float* stats, void* workspace, size_t workspace_bytes,
                                       void* stream) {
  bool empty = false;
  REL_TRY(check_logprobs(p, false, &empty));
  if (empty) return REL_OK;
  const size_t need = rel::logprobs_scratch_bytes(p->N, p->V, p->K, p->dtype);
  if (need && (!workspace || workspace_bytes < need))
    return api_fail(REL_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", need, workspace ? workspace_bytes : (size_t)0);
  const size_t es = elem_size(p->dtype), N = (size_t)p->N, K = (size_t)p->K;
  REL_TRY(aligned(logits, es, "logits"));
  REL_TRY(aligned(tokens, 8, "tokens"));
  REL_TRY(aligned(logprob, 4, "logprob", false));
  REL_TRY(aligned(entropy, 4, "entropy", false));
  REL_TRY(aligned(rank, 4, "rank", false));
  REL_TRY(aligned(top_tokens, 8, "top_tokens", K > 0));
  REL_TRY(aligned(top_logprobs, 4, "top_logprobs", K > 0));
  REL_TRY(aligned(stats, 16, "stats", false));
  REL_TRY(aligned(workspace, 16, "workspace", need > 0));
  const Range r[] = {{logits, ((N - 1) * (size_t)(N > 1 ? p->stride_logits : 0) + (size_t)p->V) * es, "logits", false},
                     {tokens, N * 8, "tokens", false},
                     {logprob, N * 4, "logprob", true},
                     {entropy, N * 4, "entropy", true},
                     {rank, N * 4, "rank", true},
                     {top_tokens, N * K * 8, "top_tokens", true},
                     {top_logprobs, N * K * 4, "top_logprobs", true},
                     {stats, N * 16, "stats", true},
                     {workspace, need, "workspace", true}};
  REL_TRY(disjoint(r, 9));
  if (rel::api_fail_launch()) return api_fail(REL_ERR_HIP, "HIP launch failure injected by RELATION_TEST_FAIL_LAUNCH");
  rel::LogprobArgs a{};
  a.logits = logits; a.tokens = tokens;
  a.sl = N > 1 ? p->stride_logits : 0;
  a.logprob = logprob; a.entropy = entropy; a.rank = rank;
  a.top_tokens = top_tokens; a.top_logprobs = top_logprobs; a.stats = stats;
  a.N = (int)p->N; a.V = (int)p->V; a.K = (int)p->K;
  a.ws = workspace;
  return hip_status(rel::launch_logprobs_fwd(a, p->dtype, (hipStream_t)stream), "log-probability launch");
}

rel_status relation_token_logprobs_bwd(const rel_token_logprobs* p, const void* logits, const int64_t* tokens,
                                       const float* stats, const float* dlogprob, const float* dentropy, void* dlogits,
                                       void* stream) {
  bool empty = false;
  REL_TRY(check_logprobs(p, true, &empty));
  if (empty) return REL_OK;
  const size_t es = elem_size(p->dtype), N = (size_t)p->N, V = (size_t)p->V;
  REL_TRY(aligned(logits, es, "logits"));
  REL_TRY(aligned(tokens, 8, "tokens"));
  REL_TRY(aligned(stats, 16, "stats"));
  REL_TRY(aligned(dlogprob, 4, "dlogprob", false));
  REL_TRY(aligned(dentropy, 4, "dentropy", false));
  REL_TRY(aligned(dlogits, es, "dlogits"));
  const Range r[] = {{logits, ((N - 1) * (size_t)(N > 1 ? p->stride_logits : 0) + V) * es, "logits", false},
                     {tokens, N * 8, "tokens", false},
                     {stats, N * 16, "stats", false},
                     {dlogprob, N * 4, "dlogprob", false},
                     {dentropy, N * 4, "dentropy", false},
                     {dlogits, ((N - 1) * (size_t)(N > 1 ? p->stride_grad : 0) + V) * es, "dlogits", true}};
  REL_TRY(disjoint(r, 6));
  if (rel::api_fail_launch()) return api_fail(REL_ERR_HIP, "HIP launch failure injected by RELATION_TEST_FAIL_LAUNCH");
  rel::LogprobGradArgs a{};
  a.logits = logits; a.tokens = tokens; a.stats = stats; a.dlogprob = dlogprob; a.dentropy = dentropy; a.dlogits = dlogits;
  a.sl = N > 1 ? p->stride_logits : 0;
  a.sg = N > 1 ? p->stride_grad : 0;
  a.N = (int)p->N; a.V = (int)p->V;
  return hip_status(rel::launch_logprobs_bwd(a, p->dtype, (hipStream_t)stream), "log-probability gradient launch");
}

}  // extern "C"
