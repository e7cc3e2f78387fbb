// eql_check.h -- argument checks shared by the C-ABI sources.  Host code only.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "../../include/eqlinear.h"

namespace eqk {

inline size_t elem_bytes(int dtype) { return dtype == EQL_F32 ? 4 : 2; }
inline bool valid_dtype(int dtype) { return dtype == EQL_F32 || dtype == EQL_F16 || dtype == EQL_BF16; }

inline size_t align256(size_t v) { return (v + 255) / 256 * 256; }

struct Range {
  const void* p;
  size_t bytes;
};

inline bool overlaps(Range a, Range b) {
  if (!a.p || !b.p || a.bytes == 0 || b.bytes == 0) return false;
  const uintptr_t a0 = (uintptr_t)a.p, a1 = a0 + a.bytes;
  const uintptr_t b0 = (uintptr_t)b.p, b1 = b0 + b.bytes;
  return a0 < b1 && b0 < a1;
}

inline bool any_overlap(const Range* r, int n) {
  for (int i = 0; i < n; ++i)
    for (int j = i + 1; j < n; ++j)
      if (overlaps(r[i], r[j])) return true;
  return false;
}

inline bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }

// EQL_OK on a gfx950 device, filling its cached properties (eql_api.cpp).
int check_device();

}  // namespace eqk
