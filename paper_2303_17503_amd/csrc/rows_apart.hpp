// rows_apart.hpp -- whether an output's rows overlap, looked at before a launch.
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

#endif  // ROWS_APART_HPP_
