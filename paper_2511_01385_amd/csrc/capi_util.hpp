// capi_util.hpp -- what the C entry points share: checks of pointers and sizes, and the device.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rdfft.h"

namespace rdfft {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// [a, a+na) and [b, b+nb) share a byte
inline bool overlaps(const void* a, int64_t na, const void* b, int64_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return na > 0 && nb > 0 && x < y + (uintptr_t)nb && y < x + (uintptr_t)na;
}

inline int elem_bytes(int dtype) { return dtype == RDFFT_F32 ? 4 : 2; }

// products of sizes that must not overflow int64
inline bool mul_ok(int64_t a, int64_t b, int64_t* out) {
  if (a < 0 || b < 0) return false;
  if (a != 0 && b > INT64_MAX / a) return false;
  *out = a * b;
  return true;
}

// The current device's twiddle table and (num_cu may be null) number of CUs.  A device's first use
// checks that it is a gfx950 and uploads the table.
int ensure_device(const float2** tw, int* num_cu);

}  // namespace rdfft
