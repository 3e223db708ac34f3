// Host helpers of relation_api.cpp that the other C-ABI sources use.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "../../include/relation.h"

namespace rel {

// Sets the calling thread's error message and returns s. Never throws.
rel_status api_fail(rel_status s, const char* fmt, ...) noexcept __attribute__((format(printf, 2, 3)));

// Whether the launch failure of RELATION_TEST_FAIL_LAUNCH is asked for.
bool api_fail_launch() noexcept;

// Rows of `width` elements at the offsets sum_i c_i stride_i, 0 <= c_i < count_i.
struct ApiLattice {
  int64_t stride[3];
  int64_t count[3];
  int64_t width;
};
// Whether distinct indices never share an element (each stride passes the span of the smaller ones).
bool api_nested(const ApiLattice& a) noexcept;
// Whether the lattice at x and the same lattice at y share an element (`elem` bytes each).
bool api_alias(const ApiLattice& a, const void* x, const void* y, size_t elem) noexcept;

}  // namespace rel
