// Arithmetic of the projection's reads of whole arrays, apart from the kernels so
// that it can be checked on the host.
#pragma once

#include <stdint.h>

namespace wd {

constexpr int64_t kLoad = 8;  // elements of a load

// Whether an array of `rows` rows of n elements, `ld` apart, ends before a load from
// its start does: the last load of the array would begin before it.
inline bool shorter_than_a_load(int64_t rows, int64_t ld, int64_t n) {
  return n < kLoad && (rows - 1) * (ld < kLoad ? ld : kLoad) + n < kLoad;
}

}  // namespace wd
