// rows_apart.hpp -- whether the rows of outputs overlap, each other or those of another tensor, looked at before a launch.
#ifndef ROWS_APART_HPP_
#define ROWS_APART_HPP_

#include <stdint.h>
#include <stdlib.h>

// Rows of `row` elements at these strides do not overlap if, in the order of their strides, each dimension steps over what the smaller ones cover.
inline bool rows_apart(const int64_t (&sizes)[3], const int64_t (&strides)[3], int64_t row) {
  int64_t covered = row;
  bool used[3] = {false, false, false};
  for (int k = 0; k < 3; ++k) {
    int least = -1;
    for (int d = 0; d < 3; ++d)
      if (!used[d] && (least < 0 || llabs(strides[d]) < llabs(strides[least]))) least = d;
    used[least] = true;
    if (sizes[least] == 1) continue;
    if (llabs(strides[least]) < covered) return false;
    covered += llabs(strides[least]) * (sizes[least] - 1);
  }
  return true;
}

struct Rows {   // of one tensor: row [i][t][h] at element i * strides[0] + t * strides[1] + h * strides[2]
  const void* p;
  int64_t sizes[3], strides[3];
};

// Whether a row of a and one of b, each of `row` elements of `bytes` bytes, share memory.  Two rows do if their distance, the bases' and a sum of whole multiples of the strides, is
// below a row.  Equal strides of the two count as one, over the differences of their indexes; then the largest stride's multiples that the others can still
// make up for are tried, in nested layouts one or two.  Layouts that need more than 2^14 trials (two sets of strides that do not nest, in the same memory) are taken to overlap.
class RowsMeet {
  struct Dim { __int128 stride, lo, hi; };   // multiples lo .. hi
  Dim dims_[6];
  __int128 least_[7], most_[7];              // what the dimensions from here on can add
  int n_ = 0, trials_ = 0;
  __int128 row_;

  static __int128 floor_div(__int128 a, __int128 b) { return a / b - (a % b < 0); }   // b > 0
  void add(int64_t stride, int64_t size, bool negative) {
    if (size <= 1 || stride == 0) return;
    if (stride < 0) negative = !negative;
    const __int128 s = stride < 0 ? -(__int128)stride : (__int128)stride, most = size - 1;
    int k = 0;
    while (k < n_ && dims_[k].stride > s) ++k;
    if (k == n_ || dims_[k].stride != s) {
      for (int m = n_++; m > k; --m) dims_[m] = dims_[m - 1];
      dims_[k] = Dim{s, 0, 0};
    }
    if (negative) dims_[k].lo -= most;
    else dims_[k].hi += most;
  }
  bool reach(int k, __int128 at) {   // whether the dimensions from k on bring `at` to within a row of 0
    if (k == n_) return at < row_ && -at < row_;
    const Dim& d = dims_[k];
    __int128 lo = -floor_div(row_ - 1 + most_[k + 1] + at, d.stride), hi = floor_div(row_ - 1 - least_[k + 1] - at, d.stride);
    lo = lo < d.lo ? d.lo : lo;
    hi = hi > d.hi ? d.hi : hi;
    for (; lo <= hi; ++lo) {
      if (k + 1 == n_ || ++trials_ > 1 << 14 || reach(k + 1, at + lo * d.stride)) return true;
    }
    return false;
  }

 public:
  bool operator()(const Rows& a, const Rows& b, int64_t row, int64_t bytes) {
    n_ = trials_ = 0;
    row_ = (__int128)row * bytes;
    for (int k = 0; k < 3; ++k) {
      add(a.strides[k], a.sizes[k], true);
      add(b.strides[k], b.sizes[k], false);
    }
    least_[n_] = most_[n_] = 0;
    for (int k = n_; k-- > 0;) {
      dims_[k].stride *= bytes;
      least_[k] = least_[k + 1] + dims_[k].lo * dims_[k].stride;
      most_[k] = most_[k + 1] + dims_[k].hi * dims_[k].stride;
    }
    return reach(0, (__int128)(intptr_t)b.p - (__int128)(intptr_t)a.p);
  }
};
// where the tensor's rows begin, at the least and at the most
inline void reach_of(const Rows& r, int64_t bytes, __int128* first, __int128* last) {
  *first = *last = (__int128)(intptr_t)r.p;
  for (int k = 0; k < 3; ++k) {
    const __int128 far = (__int128)(r.sizes[k] - 1) * r.strides[k] * bytes;
    *(far < 0 ? first : last) += far;
  }
}
inline bool rows_meet(const Rows& a, const Rows& b, int64_t row, int64_t bytes) {
  for (int k = 0; k < 3; ++k)
    if (a.sizes[k] <= 0 || b.sizes[k] <= 0) return false;
  __int128 a_first, a_last, b_first, b_last;
  reach_of(a, bytes, &a_first, &a_last);
  reach_of(b, bytes, &b_first, &b_last);
  if (a_last + row * bytes <= b_first || b_last + row * bytes <= a_first) return false;   // (most calls: tensors of their own; the five looks of a pair take 6 ns, without this 340)
  return RowsMeet()(a, b, row, bytes);
}

#endif  // ROWS_APART_HPP_
