// Host check of strided outputs (internal, not part of the ABI): whether slices
// that different CTAs write share memory.
#pragma once

#include <stdint.h>

namespace adt {

// Indices differ by less than n[k] in dimension k: whether some differences sum
// up to a distance within `need` of -x.  For dimensions one within the other, the
// largest stride first: of each only the two multiples that come nearest can,
// since what the smaller ones add is less than a stride.
inline bool slices_near(const int64_t* n, const int64_t* s, int left, int64_t need, int64_t x) {
  if (left == 0) return x < need && -x < need;
  if (*n == 1) return slices_near(n + 1, s + 1, left - 1, need, x);
  int64_t m = -x / *s;
  if (m * *s > -x) --m;
  for (int i = 0; i < 2; ++i, ++m)
    if (m > -*n && m < *n && slices_near(n + 1, s + 1, left - 1, need, x + m * *s)) return true;
  return false;
}

// Slice (i0, i1, i2) of a set starts at the sum of i_k * stride[k] and is `need`
// long; a second set of the same shape lies `delta` after it.  Whether a slice of
// the one meets a slice of the other; with delta = 0 the two are one set, of
// which different slices are compared.  Strides of dimensions of more than one
// are at least `need`, and all values small enough for sums in 64 bits.
inline bool slices_meet(const int64_t (&count)[3], const int64_t (&stride)[3], int64_t need, int64_t delta) {
  int64_t n[3], s[3], span = need;  // by stride, the largest first
  for (int k = 0; k < 3; ++k) {
    n[k] = count[k];
    s[k] = count[k] > 1 ? stride[k] : 0;
    span += (n[k] - 1) * s[k];
    for (int j = k; j > 0 && s[j] > s[j - 1]; --j) {
      const int64_t a = n[j], b = s[j];
      n[j] = n[j - 1], s[j] = s[j - 1];
      n[j - 1] = a, s[j - 1] = b;
    }
  }
  if (delta >= span || -delta >= span) return false;
  int64_t extent = need;
  bool nested = true;  // dimensions one within the other, as in all usual layouts
  for (int k = 2; k >= 0; --k) {
    nested = nested && (n[k] == 1 || s[k] >= extent);
    extent += (n[k] - 1) * s[k];
  }
  if (nested) return delta != 0 && slices_near(n, s, 3, need, delta);
  // Any others: all differences of two dimensions, with those of the longest that
  // come nearest.
  int z = 0;
  for (int k = 1; k < 3; ++k)
    if (n[k] > n[z]) z = k;
  const int p = z == 0 ? 1 : 0, q = 3 - z - p;
  for (int64_t a = -(n[p] - 1); a < n[p]; ++a) {
    for (int64_t b = -(n[q] - 1); b < n[q]; ++b) {
      const int64_t x = delta + a * s[p] + b * s[q];
      if ((delta != 0 || a != 0 || b != 0) && slices_near(n + z, s + z, 1, need, x)) return true;
    }
  }
  return false;
}

}  // namespace adt
