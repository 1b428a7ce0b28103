// sv_host.h — host helpers that the entry points of every source share: element
// sizes, workspace alignment and the address checks of strided tensors.
#pragma once

#include <cstddef>
#include <cstdint>

#include "specverify.h"

namespace sv {

inline size_t esize_of(spec_dtype dt) { return dt == SPEC_BF16 ? 2 : 4; }
inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// The last byte a tensor of n0 x n1 rows of V elements (strides s0, s1 in
// elements, both >= 0) occupies from base lies within the address space: the
// kernels' 64-bit row offsets then never overflow.
inline bool extent_ok(const void* base, int64_t n0, int64_t s0, int64_t n1, int64_t s1, int V, size_t esize) {
  int64_t a, b, last, bytes;
  if (__builtin_mul_overflow(n0 - 1, s0, &a) || __builtin_mul_overflow(n1 - 1, s1, &b) ||
      __builtin_add_overflow(a, b, &last) || __builtin_add_overflow(last, static_cast<int64_t>(V), &last) ||
      __builtin_mul_overflow(last, static_cast<int64_t>(esize), &bytes))
    return false;
  uintptr_t end;
  return !__builtin_add_overflow(reinterpret_cast<uintptr_t>(base), static_cast<uintptr_t>(bytes), &end);
}

}  // namespace sv
