// C-ABI layer of the serving entry points: page maps, rows into a paged cache,
// the decode step and chunks of new tokens over pages, and sampling. Arguments are checked on the host;
// device data (lengths, page ids, slots) is checked where the kernels read it.
#include "../../include/relation.h"

#include <cmath>

#include "api_checks.h"
#include "serve.h"

namespace {

bool power_of_two(int64_t x) { return x > 0 && (x & (x - 1)) == 0; }

int log2_of(int64_t x) {
  int s = 0;
  while ((1LL << s) < x) ++s;
  return s;
}

rel_status check_pages(const rel_pages* c, bool* empty) {
  if (!c) return api_fail(REL_ERR_INVALID_ARG, "cache description is null");
  if (c->num_pages < 0 || c->H < 0 || c->D < 0) return api_fail(REL_ERR_INVALID_ARG, "negative size of the cache");
  if (c->dtype != REL_F32 && c->dtype != REL_BF16) return api_fail(REL_ERR_UNSUPPORTED, "unknown dtype %d", (int)c->dtype);
  if (!power_of_two(c->page_size) || c->page_size > 65536)
    return api_fail(REL_ERR_UNSUPPORTED, "page_size %lld is not a power of two up to 65536", (long long)c->page_size);
  const int64_t vec = 16 / (int64_t)elem_size(c->dtype);
  if (c->D < 1 || c->D > 128 || c->D % vec)
    return api_fail(REL_ERR_UNSUPPORTED, "cache width %lld is not a multiple of 16 bytes in 1..128 elements", (long long)c->D);
  *empty = c->num_pages == 0 || c->H == 0;
  if (*empty) return REL_OK;
  if (c->num_pages > (1 << 28) || c->H > (1 << 16)) return api_fail(REL_ERR_UNSUPPORTED, "too many pages or heads");
  if (c->stride_page < 0 || c->stride_head < 0 || c->stride_token < 0)
    return api_fail(REL_ERR_INVALID_ARG, "negative stride");
  if (c->stride_page % vec || c->stride_head % vec || c->stride_token % vec)
    return api_fail(REL_ERR_INVALID_ARG, "strides must be multiples of 16 bytes");
  if (c->stride_page > kInt32Max || c->stride_head > kInt32Max || c->stride_token > kInt32Max ||
      (c->H - 1) * c->stride_head + (c->page_size - 1) * c->stride_token + c->D > kInt32Max)
    return api_fail(REL_ERR_UNSUPPORTED, "a page, or a stride, of 2^31 elements or more");
  const rel::ApiLattice L = {{c->stride_page, c->stride_head, c->stride_token}, {c->num_pages, c->H, c->page_size}, c->D};
  if (!rel::api_nested(L)) return api_fail(REL_ERR_INVALID_ARG, "strides make distinct rows of the cache overlap");
  return REL_OK;
}

// Elements from the first to past the last of the pool.
int64_t pool_extent(const rel_pages* c) {
  return (c->num_pages - 1) * c->stride_page + (c->H - 1) * c->stride_head + (c->page_size - 1) * c->stride_token + c->D;
}

rel::PagedCache cache_of(const rel_pages* c) {
  rel::PagedCache p{};
  p.num_pages = (int)c->num_pages;
  p.shift = log2_of(c->page_size);
  p.sp = c->stride_page;
  p.sh = (int)c->stride_head;
  p.st = (int)c->stride_token;
  p.H = (int)c->H;
  p.D = (int)c->D;
  return p;
}

rel_status check_query(const rel_pages* c, const rel_paged_query* d, bool* empty) {
  REL_TRY(check_pages(c, empty));
  if (!d) return api_fail(REL_ERR_INVALID_ARG, "query description is null");
  if (d->B < 0 || d->Hq < 0 || d->table_width < 0) return api_fail(REL_ERR_INVALID_ARG, "negative size of the query");
  if (!(std::isfinite(d->tau_s) && d->tau_s > 0.0f))
    return api_fail(REL_ERR_INVALID_ARG, "tau_s must be finite and > 0 (got %g)", (double)d->tau_s);
  if (!std::isfinite(d->scale)) return api_fail(REL_ERR_INVALID_ARG, "scale must be finite");
  if (d->B == 0 || d->Hq == 0) {
    *empty = true;
    return REL_OK;
  }
  if (*empty) return api_fail(REL_ERR_INVALID_ARG, "the pool has no pages or no heads");
  if (d->table_width < 1) return api_fail(REL_ERR_INVALID_ARG, "the block table has no columns");
  if (d->Hq % c->H)
    return api_fail(REL_ERR_INVALID_ARG, "query heads (%lld) must be a multiple of the cache's (%lld)", (long long)d->Hq,
                    (long long)c->H);
  if (d->table_width > (1 << 30) || d->table_width * c->page_size > (1 << 30))
    return api_fail(REL_ERR_UNSUPPORTED, "a block table row spans over 2^30 tokens");
  if (d->B > (1 << 30) || d->Hq > (1 << 30) || d->B * d->Hq > (1 << 30)) return api_fail(REL_ERR_UNSUPPORTED, "B * Hq exceeds 2^30");
  return REL_OK;
}

int64_t longest(const rel_pages* c, const rel_paged_query* d) {
  const int64_t cap = d->table_width * c->page_size;
  return d->max_length > 0 && d->max_length < cap ? d->max_length : cap;
}

}  // namespace

extern "C" {

rel_status relation_page_map(const rel_page_map* m, const int32_t* cached, const int32_t* added,
                             const int32_t* free_pages, int32_t* table, int32_t* lengths, int32_t* row_start,
                             int64_t* slots, int32_t* positions, int32_t* counts, void* stream) {
  if (!m) return api_fail(REL_ERR_INVALID_ARG, "page map description is null");
  if (m->B < 0 || m->table_width < 0 || m->max_tokens < 0 || m->num_free < 0)
    return api_fail(REL_ERR_INVALID_ARG, "negative size");
  if (!power_of_two(m->page_size) || m->page_size > 65536)
    return api_fail(REL_ERR_UNSUPPORTED, "page_size %lld is not a power of two up to 65536", (long long)m->page_size);
  if (m->B > rel::kMapMaxB)
    return api_fail(REL_ERR_UNSUPPORTED, "%lld requests: at most %d in one map", (long long)m->B, rel::kMapMaxB);
  const bool some = m->B > 0;
  if (some && m->table_width < 1) return api_fail(REL_ERR_INVALID_ARG, "the block table has no columns");
  if (m->table_width > (1 << 30) || m->table_width * m->page_size > (1 << 30))
    return api_fail(REL_ERR_UNSUPPORTED, "a block table row spans over 2^30 tokens");
  if (m->max_tokens > (1 << 30) || m->num_free > (1 << 30))
    return api_fail(REL_ERR_UNSUPPORTED, "max_tokens and num_free are at most 2^30");
  REL_TRY(aligned(cached, 4, "cached", some));
  REL_TRY(aligned(added, 4, "added", some));
  REL_TRY(aligned(free_pages, 4, "free_pages", m->num_free > 0));
  REL_TRY(aligned(table, 4, "table", some));
  REL_TRY(aligned(lengths, 4, "lengths", some));
  REL_TRY(aligned(row_start, 4, "row_start"));
  REL_TRY(aligned(slots, 8, "slots", m->max_tokens > 0));
  REL_TRY(aligned(positions, 4, "positions", m->max_tokens > 0));
  REL_TRY(aligned(counts, 4, "counts"));
  const size_t B = (size_t)m->B, N = (size_t)m->max_tokens;
  const Range r[] = {{cached, B * 4, "cached", false},
                     {added, B * 4, "added", false},
                     {free_pages, (size_t)m->num_free * 4, "free_pages", false},
                     {table, B * (size_t)m->table_width * 4, "table", true},
                     {lengths, B * 4, "lengths", true},
                     {row_start, (B + 1) * 4, "row_start", true},
                     {slots, N * 8, "slots", true},
                     {positions, N * 4, "positions", true},
                     {counts, 12, "counts", true}};
  REL_TRY(disjoint(r, 9));
  if (rel::api_fail_launch()) return api_fail(REL_ERR_HIP, "HIP launch failure injected by RELATION_TEST_FAIL_LAUNCH");
  rel::PageMapArgs a{};
  a.cached = cached; a.added = added; a.free_pages = free_pages;
  a.table = table; a.lengths = lengths; a.row_start = row_start;
  a.slots = slots; a.positions = positions; a.counts = counts;
  a.B = (int)m->B; a.W = (int)m->table_width; a.shift = log2_of(m->page_size);
  a.N = (int)m->max_tokens; a.F = (int)m->num_free;
  return hip_status(rel::launch_page_map(a, (hipStream_t)stream), "page map launch");
}

rel_status relation_paged_append(const rel_pages* c, const rel_append* n, const void* q, const void* k, const void* v,
                                 const int64_t* slots, const int32_t* positions, const float* theta, void* q_out,
                                 void* k_cache, void* v_cache, void* stream) {
  bool empty = false;
  REL_TRY(check_pages(c, &empty));
  if (!n) return api_fail(REL_ERR_INVALID_ARG, "append description is null");
  if (n->N < 0 || n->Hq < 0 || n->D < 0) return api_fail(REL_ERR_INVALID_ARG, "negative size");
  if (n->D < 1 || n->D > c->D)
    return api_fail(REL_ERR_INVALID_ARG, "width %lld is not in 1 .. the cache's %lld", (long long)n->D, (long long)c->D);
  if (!(std::isfinite(n->rope_base) && n->rope_base >= 0.0) || (n->rope_base > 0.0 && n->rope_base <= 1.0))
    return api_fail(REL_ERR_INVALID_ARG, "rope_base must be 0 (none) or finite and over 1");
  if (n->rope_base > 0.0 && n->D % 2)
    return api_fail(REL_ERR_INVALID_ARG, "RoPE needs an even head width (D = %lld)", (long long)n->D);
  if (n->givens < REL_GIVENS_NONE || n->givens > REL_GIVENS_B)
    return api_fail(REL_ERR_INVALID_ARG, "unknown Givens pairing %d", (int)n->givens);
  if (n->givens != REL_GIVENS_NONE && c->H % 2)
    return api_fail(REL_ERR_INVALID_ARG, "Givens mixing pairs heads: H = %lld is odd", (long long)c->H);
  if (n->N == 0) return REL_OK;
  if (empty) return api_fail(REL_ERR_INVALID_ARG, "the pool has no pages or no heads");
  const bool has_q = q && n->Hq > 0;
  if (n->N > (1 << 26) || n->Hq > (1 << 16)) return api_fail(REL_ERR_UNSUPPORTED, "over 2^26 tokens or 2^16 heads");
  if ((has_q && (n->q_token < 0 || n->q_head < 0)) || n->kv_token < 0 || n->kv_head < 0)
    return api_fail(REL_ERR_INVALID_ARG, "negative stride");
  const int64_t far = 1LL << 32;
  if ((has_q && (n->q_token > far || n->q_head > far)) || n->kv_token > far || n->kv_head > far)
    return api_fail(REL_ERR_UNSUPPORTED, "stride over 2^32");
  const size_t es = elem_size(c->dtype);
  REL_TRY(aligned(k, es, "k"));
  REL_TRY(aligned(v, es, "v"));
  REL_TRY(aligned(q, es, "q", false));
  REL_TRY(aligned(slots, 8, "slots"));
  REL_TRY(aligned(positions, 4, "positions"));
  REL_TRY(aligned(theta, 4, "theta", n->givens != REL_GIVENS_NONE));
  REL_TRY(aligned(q_out, 16, "q_out", has_q));
  REL_TRY(aligned(k_cache, 16, "k_cache"));
  REL_TRY(aligned(v_cache, 16, "v_cache"));
  const size_t pool = (size_t)pool_extent(c) * es;
  const size_t kv = (size_t)((n->N - 1) * n->kv_token + (c->H - 1) * n->kv_head + n->D) * es;
  const size_t qb = has_q ? (size_t)((n->N - 1) * n->q_token + (n->Hq - 1) * n->q_head + n->D) * es : 0;
  const size_t qo = has_q ? (size_t)(n->N * n->Hq * c->D) * es : 0;
  const Range in[] = {{q, qb, "q", false},
                      {k, kv, "k", false},
                      {v, kv, "v", false},
                      {slots, (size_t)n->N * 8, "slots", false},
                      {positions, (size_t)n->N * 4, "positions", false},
                      {theta, n->givens ? (size_t)(c->H / 2) * 4 : 0, "theta", false}};
  const Range out[] = {{q_out, qo, "q_out", true}, {k_cache, pool, "k_cache", true}, {v_cache, pool, "v_cache", true}};
  for (int o = 0; o < 3; ++o) {
    Range r[7];
    for (int i = 0; i < 6; ++i) r[i] = in[i];
    r[6] = out[o];
    REL_TRY(disjoint(r, 7));
  }
  for (int o = 1; o < 3; ++o) {
    const Range r[] = {out[0], out[o]};
    REL_TRY(disjoint(r, 2));
  }
  // the two caches may be interleaved in one allocation, as long as no element is shared
  const rel::ApiLattice L = {{c->stride_page, c->stride_head, c->stride_token}, {c->num_pages, c->H, c->page_size}, c->D};
  if (rel::api_alias(L, k_cache, v_cache, es)) return api_fail(REL_ERR_INVALID_ARG, "output k_cache overlaps v_cache");
  if (rel::api_fail_launch()) return api_fail(REL_ERR_HIP, "HIP launch failure injected by RELATION_TEST_FAIL_LAUNCH");
  rel::AppendArgs a{};
  a.q = has_q ? q : nullptr; a.k = k; a.v = v;
  a.slots = slots; a.positions = positions; a.theta = theta;
  a.q_out = q_out; a.k_cache = k_cache; a.v_cache = v_cache;
  a.c = cache_of(c);
  a.q_token = n->q_token; a.q_head = n->q_head; a.kv_token = n->kv_token; a.kv_head = n->kv_head;
  a.N = (int)n->N; a.Hq = has_q ? (int)n->Hq : 0; a.D = (int)n->D;
  a.givens = n->givens;
  a.rope = n->rope_base > 0.0;
  if (a.rope)
    for (int j = 0; j < a.D / 2; ++j)
      a.turns[j] = std::exp(-2.0 * j / a.D * std::log(n->rope_base)) / 6.283185307179586476925286766559;
  return hip_status(rel::launch_append(a, c->dtype, (hipStream_t)stream), "paged append launch");
}

size_t relation_paged_decode_workspace_bytes(const rel_pages* c, const rel_paged_query* d) {
  bool empty = false;
  if (check_query(c, d, &empty) != REL_OK || empty) return 0;
  int slice = 0, nsplit = 0;
  rel::paged_decode_split(d->B, c->H, d->Hq / c->H, longest(c, d), (int)c->D, c->dtype, &slice, &nsplit);
  if (nsplit == 1) return 0;
  return (size_t)nsplit * (size_t)(d->B * d->Hq) * (size_t)(c->D + 2) * 4;
}

rel_status relation_paged_decode(const rel_pages* c, const rel_paged_query* d, const void* q, const void* k_cache,
                                 const void* v_cache, const int32_t* table, const int32_t* lengths,
                                 const float* lambda, void* out, float* row_stat, void* workspace,
                                 size_t workspace_bytes, void* stream) {
  bool empty = false;
  REL_TRY(check_query(c, d, &empty));
  if (empty) return REL_OK;
  rel::PagedDecodeArgs a{};
  a.max_len = (int)longest(c, d);
  a.G = (int)(d->Hq / c->H);
  rel::paged_decode_split(d->B, c->H, a.G, a.max_len, (int)c->D, c->dtype, &a.slice, &a.nsplit);
  if ((int64_t)a.nsplit * d->B * d->Hq > (1 << 22))
    return api_fail(REL_ERR_UNSUPPORTED, "%lld rows of up to %d tokens are over 2^22 slices: pass max_length, or fewer requests",
                    (long long)(d->B * d->Hq), a.max_len);
  const size_t need = a.nsplit == 1 ? 0 : (size_t)a.nsplit * (size_t)(d->B * d->Hq) * (size_t)(c->D + 2) * 4;
  if (need && (!workspace || workspace_bytes < need))
    return api_fail(REL_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", need, workspace ? workspace_bytes : (size_t)0);
  REL_TRY(aligned(q, 16, "q"));
  REL_TRY(aligned(k_cache, 16, "k_cache"));
  REL_TRY(aligned(v_cache, 16, "v_cache"));
  REL_TRY(aligned(table, 4, "table"));
  REL_TRY(aligned(lengths, 4, "lengths"));
  REL_TRY(aligned(lambda, 4, "lambda"));
  REL_TRY(aligned(out, 16, "out"));
  REL_TRY(aligned(row_stat, 4, "row_stat", false));
  REL_TRY(aligned(workspace, 16, "workspace", need > 0));
  const size_t es = elem_size(c->dtype), pool = (size_t)pool_extent(c) * es;
  const size_t rows = (size_t)(d->B * d->Hq);
  const Range r[] = {{q, rows * (size_t)c->D * es, "q", false},
                     {k_cache, pool, "k_cache", false},
                     {v_cache, pool, "v_cache", false},
                     {table, (size_t)(d->B * d->table_width) * 4, "table", false},
                     {lengths, (size_t)d->B * 4, "lengths", false},
                     {lambda, 4, "lambda", false},
                     {out, rows * (size_t)c->D * es, "out", true},
                     {row_stat, rows * 4, "row_stat", true},
                     {workspace, need, "workspace", true}};
  REL_TRY(disjoint(r, 9));
  if (rel::api_fail_launch()) return api_fail(REL_ERR_HIP, "HIP launch failure injected by RELATION_TEST_FAIL_LAUNCH");
  a.q = q; a.k = k_cache; a.v = v_cache; a.table = table; a.lengths = lengths; a.lambda = lambda;
  a.c = cache_of(c);
  a.B = (int)d->B; a.Hq = (int)d->Hq; a.W = (int)d->table_width;
  a.scale = d->scale > 0.0f ? d->scale : 1.0f / std::sqrt((float)c->D);
  a.inv_tau = 1.0f / d->tau_s;
  a.states = (float*)workspace; a.out = out; a.row_stat = row_stat;
  return hip_status(rel::launch_paged_decode(a, c->dtype, (hipStream_t)stream), "paged decode launch");
}

// The step as a query of B requests, for the checks that the two share.
static rel_status check_chunk(const rel_pages* c, const rel_paged_chunk* d, rel_paged_query* q, bool* empty) {
  *q = rel_paged_query{};
  if (d) *q = rel_paged_query{d->B, d->Hq, d->table_width, d->max_length, d->tau_s, d->scale};
  REL_TRY(check_query(c, d ? q : nullptr, empty));
  if (d->N < 0) return api_fail(REL_ERR_INVALID_ARG, "negative size of the query");
  if (d->N == 0) *empty = true;
  if (*empty) return REL_OK;
  if (d->B > rel::kPrefillMaxB)
    return api_fail(REL_ERR_UNSUPPORTED, "%lld requests: at most %d in one chunk step", (long long)d->B, rel::kPrefillMaxB);
  if (d->B * c->H > (1 << 22)) return api_fail(REL_ERR_UNSUPPORTED, "B * H exceeds 2^22");
  if (d->N > (1 << 26) || d->N * d->Hq > (1 << 30)) return api_fail(REL_ERR_UNSUPPORTED, "over 2^26 tokens or 2^30 rows");
  return REL_OK;
}

size_t relation_paged_prefill_workspace_bytes(const rel_pages* c, const rel_paged_chunk* d) {
  bool empty = false;
  rel_paged_query q;
  if (check_chunk(c, d, &q, &empty) != REL_OK || empty) return 0;
  const rel::PrefillPlan p = rel::paged_prefill_plan(d->N, d->B, c->H, d->Hq / c->H, longest(c, &q), (int)c->D, c->dtype);
  return p.nsplit == 1 ? 0 : (size_t)p.nsplit * (size_t)(d->N * d->Hq) * (size_t)(c->D + 2) * 4;
}

rel_status relation_paged_prefill(const rel_pages* c, const rel_paged_chunk* d, const void* q, const void* k_cache,
                                  const void* v_cache, const int32_t* table, const int32_t* lengths,
                                  const int32_t* row_start, const float* lambda, void* out, float* row_stat,
                                  void* workspace, size_t workspace_bytes, void* stream) {
  bool empty = false;
  rel_paged_query as_query;
  REL_TRY(check_chunk(c, d, &as_query, &empty));
  if (empty) return REL_OK;
  const size_t need = relation_paged_prefill_workspace_bytes(c, d);
  if (need && (!workspace || workspace_bytes < need))
    return api_fail(REL_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", need, workspace ? workspace_bytes : (size_t)0);
  REL_TRY(aligned(q, 16, "q"));
  REL_TRY(aligned(k_cache, 16, "k_cache"));
  REL_TRY(aligned(v_cache, 16, "v_cache"));
  REL_TRY(aligned(table, 4, "table"));
  REL_TRY(aligned(lengths, 4, "lengths"));
  REL_TRY(aligned(row_start, 4, "row_start"));
  REL_TRY(aligned(lambda, 4, "lambda"));
  REL_TRY(aligned(out, 16, "out"));
  REL_TRY(aligned(row_stat, 4, "row_stat", false));
  REL_TRY(aligned(workspace, 16, "workspace", need > 0));
  const size_t es = elem_size(c->dtype), pool = (size_t)pool_extent(c) * es;
  const size_t rows = (size_t)(d->N * d->Hq);
  const Range r[] = {{q, rows * (size_t)c->D * es, "q", false},
                     {k_cache, pool, "k_cache", false},
                     {v_cache, pool, "v_cache", false},
                     {table, (size_t)(d->B * d->table_width) * 4, "table", false},
                     {lengths, (size_t)d->B * 4, "lengths", false},
                     {row_start, (size_t)(d->B + 1) * 4, "row_start", false},
                     {lambda, 4, "lambda", false},
                     {out, rows * (size_t)c->D * es, "out", true},
                     {row_stat, rows * 4, "row_stat", true},
                     {workspace, need, "workspace", true}};
  REL_TRY(disjoint(r, 10));
  if (rel::api_fail_launch()) return api_fail(REL_ERR_HIP, "HIP launch failure injected by RELATION_TEST_FAIL_LAUNCH");
  rel::PagedPrefillArgs a{};
  a.q = q; a.k = k_cache; a.v = v_cache; a.table = table; a.lengths = lengths; a.row_start = row_start; a.lambda = lambda;
  a.c = cache_of(c);
  a.B = (int)d->B; a.N = (int)d->N; a.Hq = (int)d->Hq; a.G = (int)(d->Hq / c->H); a.W = (int)d->table_width;
  a.max_len = (int)longest(c, &as_query);
  a.scale = d->scale > 0.0f ? d->scale : 1.0f / std::sqrt((float)c->D);
  a.inv_tau = 1.0f / d->tau_s;
  const rel::PrefillPlan plan = rel::paged_prefill_plan(d->N, d->B, c->H, a.G, a.max_len, (int)c->D, c->dtype);
  a.tile_rows = plan.tile_rows; a.nsplit = plan.nsplit; a.slice = plan.slice;
  a.states = (float*)workspace;
  a.out = out; a.row_stat = row_stat;
  return hip_status(rel::launch_paged_prefill(a, c->dtype, (hipStream_t)stream), "paged prefill launch");
}

static rel_status check_sample(const rel_sample* s, bool* empty) {
  if (!s) return api_fail(REL_ERR_INVALID_ARG, "sample description is null");
  if (s->B < 0 || s->V < 0) return api_fail(REL_ERR_INVALID_ARG, "negative size");
  if (s->dtype != REL_F32 && s->dtype != REL_BF16) return api_fail(REL_ERR_UNSUPPORTED, "unknown dtype %d", (int)s->dtype);
  *empty = s->B == 0;
  if (*empty) return REL_OK;
  if (s->V < 1) return api_fail(REL_ERR_INVALID_ARG, "a row without tokens");
  if (s->V > rel::kSampleMaxV || s->B > (1 << 20)) return api_fail(REL_ERR_UNSUPPORTED, "V is at most 2^22 and B at most 2^20");
  if (s->B * s->V > (1LL << 36)) return api_fail(REL_ERR_UNSUPPORTED, "B * V is over 2^36");
  // rows are only read: 0, one row for all, does no harm
  if (s->B > 1 && ((s->stride_logits && s->stride_logits < s->V) || (s->stride_noise && s->stride_noise < s->V)))
    return api_fail(REL_ERR_INVALID_ARG, "row strides must be 0 or at least V");
  if (s->B > 1 && (s->stride_logits > (1LL << 40) || s->stride_noise > (1LL << 40)))
    return api_fail(REL_ERR_UNSUPPORTED, "row stride over 2^40");
  return REL_OK;
}

size_t relation_sample_workspace_bytes(const rel_sample* s) {
  bool empty = false;
  if (check_sample(s, &empty) != REL_OK || empty) return 0;
  return rel::sample_workspace_bytes(s->B, s->V, s->dtype);
}

rel_status relation_sample(const rel_sample* s, const void* logits, const float* noise, const float* temperature,
                           const int32_t* top_k, const float* top_p, const float* min_p, int64_t* tokens,
                           float* logprob, void* workspace, size_t workspace_bytes, void* stream) {
  bool empty = false;
  REL_TRY(check_sample(s, &empty));
  if (empty) return REL_OK;
  const size_t need = rel::sample_workspace_bytes(s->B, s->V, s->dtype);
  if (need && (!workspace || workspace_bytes < need))
    return api_fail(REL_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", need, workspace ? workspace_bytes : (size_t)0);
  const size_t es = elem_size(s->dtype), B = (size_t)s->B;
  REL_TRY(aligned(logits, es, "logits"));
  REL_TRY(aligned(noise, 4, "noise"));
  REL_TRY(aligned(temperature, 4, "temperature", false));
  REL_TRY(aligned(top_k, 4, "top_k", false));
  REL_TRY(aligned(top_p, 4, "top_p", false));
  REL_TRY(aligned(min_p, 4, "min_p", false));
  REL_TRY(aligned(tokens, 8, "tokens"));
  REL_TRY(aligned(logprob, 4, "logprob", false));
  REL_TRY(aligned(workspace, 16, "workspace", need > 0));
  const Range r[] = {{logits, ((B - 1) * (size_t)(B > 1 ? s->stride_logits : 0) + (size_t)s->V) * es, "logits", false},
                     {noise, ((B - 1) * (size_t)(B > 1 ? s->stride_noise : 0) + (size_t)s->V) * 4, "noise", false},
                     {temperature, B * 4, "temperature", false},
                     {top_k, B * 4, "top_k", false},
                     {top_p, B * 4, "top_p", false},
                     {min_p, B * 4, "min_p", false},
                     {tokens, B * 8, "tokens", true},
                     {logprob, B * 4, "logprob", true},
                     {workspace, need, "workspace", true}};
  REL_TRY(disjoint(r, 9));
  if (rel::api_fail_launch()) return api_fail(REL_ERR_HIP, "HIP launch failure injected by RELATION_TEST_FAIL_LAUNCH");
  rel::SampleArgs a{};
  a.logits = logits; a.noise = noise;
  a.sl = s->B > 1 ? s->stride_logits : 0;
  a.sn = s->B > 1 ? s->stride_noise : 0;
  a.temperature = temperature; a.top_k = top_k; a.top_p = top_p; a.min_p = min_p;
  a.tokens = tokens; a.logprob = logprob;
  a.B = (int)s->B; a.V = (int)s->V; a.ws = workspace;
  return hip_status(rel::launch_sample(a, s->dtype, (hipStream_t)stream), "sample launch");
}

}  // extern "C"
