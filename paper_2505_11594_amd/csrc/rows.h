// Whether two strided tensors have memory in common, for the C entry points' checks.
// Plain host code, in elements.
#pragma once
#include <stddef.h>

namespace sage {

// Rows of D elements each, at up to three dimensions of positive strides, the largest first.
struct RowSet {
  int dims = 0, D;
  long long stride[3], size[3], extent[4];   // extent[k]: from a row's first element on, over the dimensions from k on
  RowSet(int D_, long long sb, long long nb, long long sh, long long nh, long long sn, long long nn) : D(D_) {
    const long long s[3] = {sb, sh, sn}, n[3] = {nb, nh, nn};
    for (int i = 0; i < 3; ++i) {
      if (n[i] <= 1 || s[i] == 0) continue;  // the same rows again
      int at = dims++;
      for (; at > 0 && stride[at - 1] < s[i]; --at) { stride[at] = stride[at - 1]; size[at] = size[at - 1]; }
      stride[at] = s[i];
      size[at] = n[i];
    }
    extent[dims] = D;
    constexpr long long kMost = 1LL << 60;   // beyond any memory
    for (int k = dims; k-- > 0;) {
      const bool far = stride[k] > kMost / size[k] || extent[k + 1] >= kMost;
      extent[k] = far ? kMost : extent[k + 1] + stride[k] * (size[k] - 1);
    }
  }
};

inline long long floor_div(long long a, long long b) { return a / b - (a % b < 0); }   // b > 0

// Whether rows of a, from dimension ka on, and rows of b, from kb on, meet; b begins d elements behind a.
// Parts whose ranges are apart are left out at once, and of two dimensions with one stride (views of one
// buffer) only the differences of their indices are gone through: a few steps.  `steps` bounds the others;
// where they do not do, the answer is no.
inline bool rows_meet(const RowSet& a, int ka, const RowSet& b, int kb, long long d, int* steps) {
  if (d >= a.extent[ka] || d <= -b.extent[kb]) return false;
  const bool sa = ka < a.dims, sb = kb < b.dims;
  if (!sa && !sb) return true;
  const bool both = sa && sb && a.stride[ka] == b.stride[kb];
  const bool split_a = both || (sa && (!sb || a.stride[ka] > b.stride[kb])), split_b = both || !split_a;
  const int na = ka + split_a, nb = kb + split_b;
  const long long s = split_a ? a.stride[ka] : b.stride[kb];
  // the places of b's part behind a's, d + t s, at which the parts' ranges meet: in (-extent of b's, extent of a's)
  long long lo = floor_div(-b.extent[nb] - d, s) + 1, hi = floor_div(a.extent[na] - 1 - d, s);
  const long long first = split_a ? -(a.size[ka] - 1) : 0, last = split_b ? b.size[kb] - 1 : 0;
  lo = lo > first ? lo : first;
  hi = hi < last ? hi : last;
  for (long long t = lo; t <= hi; ++t) {
    if (--*steps < 0) return false;
    if (rows_meet(a, na, b, nb, d + t * s, steps)) return true;
  }
  return false;
}

}  // namespace sage
