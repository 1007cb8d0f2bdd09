// Host check of strided outputs (internal, not part of the ABI): whether slices
// that different CTAs write share memory.
#pragma once

#include <stdint.h>

namespace adt {

// Slice (i0, i1, i2) of a set starts at the sum of i_k * stride[k] and is `need`
// long; a second set of the same shape lies `delta` after it.  Whether a slice of
// the one meets a slice of the other; with delta = 0 the two are one set, of
// which different slices are compared.  Strides of dimensions of more than one
// are at least `need`, and all values small enough for sums in 64 bits.
inline bool slices_meet(const int64_t (&count)[3], const int64_t (&stride)[3], int64_t need, int64_t delta) {
  int64_t n[3], s[3], span = need;  // by count, the largest last
  for (int k = 0; k < 3; ++k) {
    n[k] = count[k];
    s[k] = count[k] > 1 ? stride[k] : 0;
    span += (n[k] - 1) * s[k];
    for (int j = k; j > 0 && n[j] < n[j - 1]; --j) {
      const int64_t a = n[j], b = s[j];
      n[j] = n[j - 1], s[j] = s[j - 1];
      n[j - 1] = a, s[j - 1] = b;
    }
  }
  if (delta >= span || -delta >= span) return false;
  if (delta == 0) {  // dimensions one within the other, as in all usual layouts
    int64_t extent = need, last = 0;
    bool nested = true;
    for (int k = 0; k < 3 && nested; ++k) {  // (smallest stride first)
      int64_t next = INT64_MAX, times = 1;
      for (int j = 0; j < 3; ++j)
        if (s[j] > last && s[j] < next) next = s[j], times = n[j];
      if (next == INT64_MAX) break;
      nested = next >= extent;
      extent += next * (times - 1);
      last = next;
    }
    for (int j = 0; j < 3; ++j)
      for (int k = 0; k < j; ++k) nested = nested && (s[j] == 0 || s[j] != s[k]);
    if (nested) return false;
  }
  // Any other: a difference of indices with |distance| < need.  Of the longest
  // dimension only the two that come nearest to the others' sum can give one.
  for (int64_t a = -(n[0] - 1); a < n[0]; ++a) {
    for (int64_t b = -(n[1] - 1); b < n[1]; ++b) {
      if (delta == 0 && a == 0 && b == 0) continue;
      const int64_t x = delta + a * s[0] + b * s[1];
      int64_t c = s[2] > 0 ? -x / s[2] - 1 : 0;
      for (int i = 0; i < 3; ++i, ++c) {
        const int64_t m = s[2] == 0 ? 0 : c < -(n[2] - 1) ? -(n[2] - 1) : c > n[2] - 1 ? n[2] - 1 : c;
        const int64_t d = x + m * s[2];
        if (d < need && -d < need) return true;
      }
    }
  }
  return false;
}

}  // namespace adt
