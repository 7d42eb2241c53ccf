// Host-side checks of the calls that work on rows of matrices: types, strides, alignment, overlaps.
#pragma once
#include "host_checks.cuh"
#include "rows.cuh"

namespace absnt {

inline int bytes_of(int dtype) {
  switch (dtype) {
    case ABS_F32: return 4;
    case ABS_BF16: case ABS_F16: return 2;
    case ABS_E4M3: case ABS_E5M2: case ABS_E8M0: return 1;
    default: return 0;
  }
}
inline bool wide_float(int dtype) { return dtype == ABS_F32 || dtype == ABS_BF16 || dtype == ABS_F16; }

// n0 x n1 rows of h elements as a call gets them.  Strides of a dimension of one are not looked at.
struct Rows {
  const unsigned char* p;
  int64_t n0, n1, h;
  int64_t s0, s1;  // bytes
  int dtype, esz;
  bool given() const { return p != nullptr; }
  int64_t row_bytes() const { return h * esz; }
  int64_t bytes() const { return (n0 - 1) * s0 + (n1 - 1) * s1 + row_bytes(); }
  // as a kernel that reads `vec` values at once sees it (see rows_aligned)
  RowsArg arg(int vec = 1) const {
    const int64_t unit = static_cast<int64_t>(vec) * (esz ? esz : 1);
    return {const_cast<unsigned char*>(p), s0, s1, static_cast<uint32_t>(s0 / unit), static_cast<uint32_t>(s1 / unit),
            static_cast<uint32_t>(unit)};
  }
};

constexpr int64_t kMostElements = int64_t{1} << 46;  // between a tensor's first element and its last

// ABS_OK, or what is wrong with the description.  An absent one (data NULL) is fine.
inline int take_rows(const abs_rows& a, int64_t n0, int64_t n1, int64_t h, Rows& r) {
  r = Rows{static_cast<const unsigned char*>(a.data), n0, n1, h, 0, 0, a.dtype, bytes_of(a.dtype)};
  if (!r.given()) return ABS_OK;
  if (!r.esz) return ABS_ERR_DTYPE;
  if (a.reserved != 0) return ABS_ERR_RANGE;
  const int64_t s0 = n0 > 1 ? a.stride0 : 0, s1 = n1 > 1 ? a.stride1 : 0;
  if (s0 < 0 || s1 < 0 || s0 > kMostElements || s1 > kMostElements) return ABS_ERR_RANGE;
  if (static_cast<__int128>(n0 - 1) * s0 + static_cast<__int128>(n1 - 1) * s1 + h > kMostElements) return ABS_ERR_RANGE;
  if (misaligned(a.data, r.esz)) return ABS_ERR_ALIGN;
  r.s0 = s0 * r.esz;
  r.s1 = s1 * r.esz;
  return ABS_OK;
}

// whether rows of an output share no byte with one another
inline bool separate_rows(const Rows& r) {
  if (r.n0 == 1 && r.n1 == 1) return true;
  if (r.n0 == 1) return r.s1 >= r.row_bytes();
  if (r.n1 == 1) return r.s0 >= r.row_bytes();
  const bool outer = r.s0 >= r.s1;
  const int64_t small = outer ? r.s1 : r.s0, large = outer ? r.s0 : r.s1, n = outer ? r.n1 : r.n0;
  return small >= r.row_bytes() && large >= (n - 1) * small + r.row_bytes();
}

// every row of `a` lies where the same row of `b` does, element by element
inline bool same_rows(const Rows& a, const Rows& b) {
  return a.p == b.p && a.dtype == b.dtype && a.s0 == b.s0 && a.s1 == b.s1;
}

inline int64_t floor_div(int64_t a, int64_t b) { return a / b - ((a % b != 0) && ((a < 0) != (b < 0))); }

// Whether a row of `a` shares a byte with a row of `b`.  Exact for tensors of the same strides (columns of one
// matrix); others share one as soon as their address ranges do.
inline bool rows_touch(const Rows& a, const Rows& b) {
  if (!overlaps(a.p, a.bytes(), b.p, b.bytes())) return false;
  if (a.s0 != b.s0 || a.s1 != b.s1) return true;
  // b's row (i, j) is at distance d + i s0 + j s1 from a's row (0, 0), |i| < n0, |j| < n1
  const int64_t d = b.p - a.p, la = a.row_bytes(), lb = b.row_bytes();
  const bool outer_few = a.n0 <= a.n1;
  const int64_t n = outer_few ? a.n0 : a.n1, m = outer_few ? a.n1 : a.n0;
  const int64_t sn = outer_few ? a.s0 : a.s1, sm = outer_few ? a.s1 : a.s0;
  if (n > 4096) return true;
  for (int64_t i = -(n - 1); i <= n - 1; ++i) {
    // some j with -lb < d + i sn + j sm < la
    const int64_t low = -lb - d - i * sn, high = la - d - i * sn;
    if (sm == 0) {
      if (low < 0 && 0 < high) return true;
      continue;
    }
    int64_t j = floor_div(low, sm) + 1;  // the smallest with low < j sm
    if (j < -(m - 1)) j = -(m - 1);
    if (j <= m - 1 && j * sm < high && j * sm > low) return true;
  }
  return false;
}

// all rows begin on multiples of `vec` values, and at most 2^32 such multiples behind the first
inline bool rows_aligned(const Rows& r, int vec) {
  const int64_t a = static_cast<int64_t>(vec) * r.esz;
  return !r.given() || (!misaligned(r.p, a) && r.s0 % a == 0 && r.s1 % a == 0 && r.bytes() / a <= INT64_C(0xffffffff));
}

}  // namespace absnt
