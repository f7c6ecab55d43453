// What can be said of paac_rows arguments without a device: whether rows overlap, and how wide they may be accessed.  Plain C++.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "../../include/paac.h"

namespace paac {

// n0 x n1 rows of c elements of `size` bytes.  A stride that is never taken is made 0, so that it says nothing.
struct RowSet {
  uintptr_t at = 0;
  int64_t outer = 0, inner = 0, n0 = 1, n1 = 1, c = 0;
  int size = 1;

  RowSet() {}
  RowSet(const paac_rows& r, int64_t n0_, int64_t n1_, int64_t c_, int size_)
      : at(reinterpret_cast<uintptr_t>(r.data)), outer(n0_ > 1 ? r.outer : 0), inner(n1_ > 1 ? r.inner : 0), n0(n0_), n1(n1_), c(c_), size(size_) {}

  static int64_t magnitude(int64_t v) { return v < 0 ? -v : v; }
  // 2^56 bytes are beyond any address, so what reaches further is no array; the sums below are of 128 bits
  bool sane() const {
    constexpr int64_t most = int64_t(1) << 56;
    return outer > -most && outer < most && inner > -most && inner < most && low() > 0 && high() < most;
  }
  bool aligned() const { return at % size == 0; }
  // first and last byte that any row touches
  __int128 low() const {
    __int128 v = at;
    if (outer < 0) v += (__int128)outer * (n0 - 1) * size;
    if (inner < 0) v += (__int128)inner * (n1 - 1) * size;
    return v;
  }
  __int128 high() const {
    __int128 v = (__int128)at + (__int128)c * size - 1;
    if (outer > 0) v += (__int128)outer * (n0 - 1) * size;
    if (inner > 0) v += (__int128)inner * (n1 - 1) * size;
    return v;
  }
  // Whether the rows are certainly apart from one another: the smaller stride covers a row, the larger one all rows of the smaller.
  bool rows_apart() const {
    const int64_t a = magnitude(outer), b = magnitude(inner);
    if (n0 == 1) return n1 == 1 || b >= c;
    if (n1 == 1) return a >= c;
    if (b <= a) return b >= c && (__int128)a >= (__int128)b * (n1 - 1) + c;
    return a >= c && (__int128)b >= (__int128)a * (n0 - 1) + c;
  }
  // Whether two sets have no byte in common, the rows of this one being apart: one ends before the other begins, or they have as many rows of the
  // same strides, which cover the longer of the two's, and no row of one meets a row of the other (two parts of wider rows).  A row of the other is |i| larger and
  // |j| smaller strides away; the larger stride covers all rows of the smaller, which covers a row, so that only the multiples next to the
  // distance can meet.
  bool apart_from(const RowSet& o) const {
    if (high() < o.low() || o.high() < low()) return true;
    if (size != o.size || outer != o.outer || inner != o.inner || n0 != o.n0 || n1 != o.n1) return false;
    if (c != o.c) {
      RowSet longer = *this;
      longer.c = c > o.c ? c : o.c;
      if (!longer.rows_apart()) return false;
    }
    const bool first = magnitude(outer) >= magnitude(inner);
    const __int128 large = (__int128)magnitude(first ? outer : inner) * size, small = (__int128)magnitude(first ? inner : outer) * size;
    const int64_t n_large = first ? n0 : n1, n_small = first ? n1 : n0;
    const __int128 row = (__int128)c * size, others = (__int128)o.c * size, d = (__int128)o.at - (__int128)at;
    const __int128 i0 = large == 0 ? 0 : -(d / large);
    for (__int128 i = i0 - 1; i <= i0 + 1; ++i) {
      if (i <= -n_large || i >= n_large) continue;
      const __int128 e = d + i * large, j0 = small == 0 ? 0 : -(e / small);
      for (__int128 j = j0 - 1; j <= j0 + 1; ++j) {
        const __int128 off = e + j * small;
        if (j > -n_small && j < n_small && off > -others && off < row) return false;
      }
    }
    return true;
  }
  // Whether every row begins on a multiple of `bytes`, its length being one too.
  bool multiples_of(int bytes) const {
    return at % bytes == 0 && c * size % bytes == 0 && outer % bytes * size % bytes == 0 && inner % bytes * size % bytes == 0;
  }
  bool same_as(const RowSet& o) const { return at == o.at && size == o.size && outer == o.outer && inner == o.inner; }
};

// A plain array of `bytes` bytes as a set of one row.
inline RowSet array_set(const void* p, int64_t bytes) { return RowSet(paac_rows{const_cast<void*>(p), 0, 0}, 1, 1, bytes, 1); }

// The arrays of a call: whether each that is written is apart from all others.
class Arrays {
 public:
  bool apart = true;
  // (rows of `r` that are written are apart from one another)
  void keep(const RowSet& r, bool out) {
    if (count_ == MOST) apart = false;
    if (!apart) return;
    low_[count_] = r.low();
    high_[count_] = r.high();
    for (int i = 0; i < count_ && apart; ++i)
      if ((out || written_[i]) && low_[count_] <= high_[i] && low_[i] <= high_[count_])       // where one ends before the other begins they are apart
        if ((out && !r.apart_from(kept_[i])) || (written_[i] && !kept_[i].apart_from(r))) apart = false;
    kept_[count_] = r;
    written_[count_++] = out;
  }
  // one that may be absent
  void keep(const void* p, int64_t bytes, bool out) { if (p != nullptr) keep(array_set(p, bytes), out); }

 private:
  static constexpr int MOST = 24;
  RowSet kept_[MOST];
  __int128 low_[MOST], high_[MOST];      // first and last bytes, so that they are worked out once
  bool written_[MOST] = {};
  int count_ = 0;
};

}  // namespace paac
