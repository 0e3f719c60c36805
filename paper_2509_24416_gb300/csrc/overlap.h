// Whether an output's elements meet an input's: plain C++, for the C entries' checks.
#pragma once

#include <cstdint>

namespace clq {

// Two arrays of n[0] x n[1] runs of D 16-bit elements, one run at 0 or more elements' stride from
// the next in each dimension.  True if `out` has an element in common with `in` without being the very
// same places.  out's runs are apart, the ones of the dimension with the smaller stride inside a stride of
// the other.  in's strides are out's or 0 in each dimension (of more than one) where this is exact; with
// other strides arrays whose ranges of addresses meet count as overlapping.
inline bool overlaps(const void* out, const int64_t (&so)[2], const void* in, const int64_t (&si)[2],
                     const int64_t (&n)[2], int64_t D) {
  using wide = __int128;  // (strides are any 64-bit number)
  if (n[0] <= 0 || n[1] <= 0) return false;
  const wide d = (static_cast<wide>(reinterpret_cast<uintptr_t>(in)) -
                  static_cast<wide>(reinterpret_cast<uintptr_t>(out))) / 2;
  wide end_out = D, end_in = D;
  bool same = d == 0, alike = true;
  // in's elements less out's: d + q[0] S[0] + q[1] S[1] + c, |c| < D, q from lo to hi
  wide S[2], lo[2], hi[2];
  for (int i = 0; i < 2; ++i) {
    end_out += static_cast<wide>(n[i] - 1) * so[i];
    end_in += static_cast<wide>(n[i] - 1) * si[i];
    S[i] = lo[i] = hi[i] = 0;
    if (n[i] == 1) continue;
    same = same && si[i] == so[i];
    alike = alike && (si[i] == so[i] || si[i] == 0);
    S[i] = so[i];
    lo[i] = 1 - n[i];
    hi[i] = si[i] == 0 ? 0 : n[i] - 1;
  }
  if (same || d >= end_out || -d >= end_in) return false;
  if (!alike) return true;
  const int a = S[0] >= S[1] ? 0 : 1, b = 1 - a;  // outer and inner dimension
  // The multiple q of s, in its range, that takes v to the first value >= 0, and the one before it.
  auto nearest = [](wide v, wide s, wide low, wide high, int which) {
    if (s == 0) return wide{0};
    wide q = v <= 0 ? (-v + s - 1) / s : -(v / s);
    q -= which;
    return q < low ? low : q > high ? high : q;
  };
  for (int i = 0; i < 2; ++i)
    for (int j = 0; j < 2; ++j) {
      const wide v = d + nearest(d, S[a], lo[a], hi[a], i) * S[a];
      const wide w = v + nearest(v, S[b], lo[b], hi[b], j) * S[b];
      if (w < D && -w < D) return true;
    }
  return false;
}

}  // namespace clq
