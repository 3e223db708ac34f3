// Checks that the C-ABI sources share: alignment, overlaps, HIP errors.
#pragma once

#include <hip/hip_runtime.h>

#include "api.h"

namespace {

using rel::api_fail;

#define REL_TRY(x)               \
  do {                           \
    rel_status _s = (x);         \
    if (_s != REL_OK) return _s; \
  } while (0)

size_t elem_size(int32_t dtype) { return dtype == REL_BF16 ? 2 : 4; }

rel_status hip_status(hipError_t e, const char* where) {
  return e == hipSuccess ? REL_OK : api_fail(REL_ERR_HIP, "%s: %s", where, hipGetErrorString(e));
}

rel_status aligned(const void* p, size_t align, const char* name, bool required = true) {
  if (!p) return required ? api_fail(REL_ERR_INVALID_ARG, "%s is null", name) : REL_OK;
  if ((uintptr_t)p % align) return api_fail(REL_ERR_INVALID_ARG, "%s is not %zu-byte aligned", name, align);
  return REL_OK;
}

// A byte range of an argument. Outputs may overlap nothing.
struct Range {
  const void* ptr;
  size_t bytes;
  const char* name;
  bool output;
};

rel_status disjoint(const Range* r, int n) {
  for (int i = 0; i < n; ++i) {
    if (!r[i].ptr || !r[i].output || !r[i].bytes) continue;
    for (int j = 0; j < n; ++j) {
      if (i == j || !r[j].ptr || !r[j].bytes || (r[j].output && j < i)) continue;
      const uintptr_t x = (uintptr_t)r[i].ptr, y = (uintptr_t)r[j].ptr;
      if (x < y + r[j].bytes && y < x + r[i].bytes)
        return api_fail(REL_ERR_INVALID_ARG, "output %s overlaps %s", r[i].name, r[j].name);
    }
  }
  return REL_OK;
}

constexpr int64_t kInt32Max = 0x7fffffff;

}  // namespace
