// Checks of the C ABI's arguments that its entry points share: byte ranges and what overlaps, strides, alignment.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace npd {

struct Range {
  uintptr_t b, e;
};

inline Range range_of(const void* p, size_t bytes) {
  const uintptr_t b = reinterpret_cast<uintptr_t>(p);
  return Range{b, b + bytes};
}

inline bool overlaps(const Range& x, const Range& y) { return x.b < y.e && y.b < x.e && x.b != x.e && y.b != y.e; }

inline size_t rows_bytes(int64_t T, int64_t stride, int64_t width, size_t elem) {
  return (size_t)(((T - 1) * stride + width) * (int64_t)elem);
}

// a row stride the byte extent of [T, stride] bf16 / fp32 arrays can be computed with in 64 bits
inline bool stride_fits(int64_t T, int64_t stride) { return stride <= (INT64_MAX / 8) / T; }

// a pointer that is not a multiple of its element size (NULL counts as aligned)
inline bool misaligned(const void* p, uintptr_t elem) { return (reinterpret_cast<uintptr_t>(p) & (elem - 1)) != 0; }

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// true if an output range overlaps an input range or another output range
inline bool any_alias(const Range* in, int n_in, const Range* out, int n_out) {
  for (int o = 0; o < n_out; ++o) {
    for (int i = 0; i < n_in; ++i)
      if (overlaps(out[o], in[i])) return true;
    for (int o2 = o + 1; o2 < n_out; ++o2)
      if (overlaps(out[o], out[o2])) return true;
  }
  return false;
}

inline Range opt_range(const void* p, size_t bytes) { return p ? range_of(p, bytes) : Range{0, 0}; }

}  // namespace npd
