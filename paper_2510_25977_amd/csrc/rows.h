// Do two matrices share memory?  Plain C++, so that it can be checked on the host against every byte.
#pragma once
#include <cstdint>
#include <initializer_list>

namespace svdmlp {

// `rows` rows of `bytes` bytes, `ld` >= bytes from the start of one to the next (of one row: not looked at), in the addresses begin ..
// end - 1; none where there is no matrix
struct Rows {
  int64_t begin = INT64_MAX, end = INT64_MIN, rows, bytes, ld;
  Rows(const void* at, int64_t rows, int64_t bytes, int64_t ld) : rows(rows), bytes(bytes), ld(ld) {
    if (!at || rows <= 0) return;
    begin = (int64_t)(uintptr_t)at;
    end = begin + (rows > 1 ? (rows - 1) * ld : 0) + bytes;
  }
};

inline int64_t floor_div(int64_t a, int64_t b) { return a / b - (a % b < 0); }

// Whether a row of one and a row of the other have a byte in common.  What lies between rows counts for nothing, so column ranges of
// one buffer are apart.  Constant time unless the ranges of addresses meet and the strides differ: then a step for every row of
// the matrix that has fewer.
inline bool overlap(const Rows& a, const Rows& b) {
  if (a.end <= b.begin || b.end <= a.begin) return false;
  const Rows &x = a.rows <= b.rows ? a : b, &y = a.rows <= b.rows ? b : a;
  if (y.rows == 1) return true;
  if (x.rows > 1 && x.ld == y.ld) {       // row j of y begins `rem` into row j + k of x and its gap
    const int64_t k = floor_div(y.begin - x.begin, x.ld), rem = y.begin - x.begin - k * x.ld;
    auto meet = [&](int64_t d) { return d < x.rows && d + y.rows > 0; };      // some row j of y has a row j + d of x
    return (rem < x.bytes && meet(k)) || (rem + y.bytes > x.ld && meet(k + 1));
  }
  for (int64_t i = 0; i < x.rows; ++i) {
    const int64_t at = x.begin + (i ? i * x.ld : 0) - y.begin;      // the rows of y that end behind this and begin before its end
    int64_t first = floor_div(at - y.bytes, y.ld) + 1, last = floor_div(at + x.bytes - 1, y.ld);
    if (first < 0) first = 0;
    if (last > y.rows - 1) last = y.rows - 1;
    if (first <= last) return true;
  }
  return false;
}

// ... one of the outputs with an input or with another output
inline bool outputs_overlap(std::initializer_list<Rows> outputs, std::initializer_list<Rows> inputs) {
  for (const Rows* o = outputs.begin(); o != outputs.end(); ++o) {
    for (const Rows& i : inputs)
      if (overlap(*o, i)) return true;
    for (const Rows* other = outputs.begin(); other != o; ++other)
      if (overlap(*o, *other)) return true;
  }
  return false;
}

}  // namespace svdmlp
