// Whether two operands' rows share a byte, on the host (no CUDA: compiled alone by a test).
#pragma once

#include <algorithm>
#include <cstdint>

namespace fs {

// n rows of `width` bytes, `step` >= width apart (of a single row it is not used), from address `at` on; n, width > 0.
struct RowSpan {
  int64_t at, n, width, step;
};

// The sum of floor((a j + b) / m) over 0 <= j < rows; a, b >= 0, m > 0. (Euclid's steps: points under a line, counted by columns or,
// with both axes exchanged, by rows.)
inline __int128 floor_sum(__int128 rows, __int128 a, __int128 b, __int128 m) {
  __int128 sum = 0;
  while (rows > 0) {
    sum += (rows - 1) * rows / 2 * (a / m) + rows * (b / m);
    a %= m, b %= m;
    const __int128 top = a * rows + b;
    rows = top / m, b = top % m;
    std::swap(a, m);
  }
  return sum;
}

// Exactly: some row of one and some row of the other have a byte in common.
inline bool rows_overlap(RowSpan a, RowSpan b) {
  if (a.n == 1) a.step = a.width;
  if (b.n == 1) b.step = b.width;
  // b's rows j in [first, end) lie within a's reach: they end behind a's first byte and begin before its last row's end. Such a row meets a
  // row of a just where it meets one of rows without beginning or end at the same distance.
  using Wide = __int128;  // (rows that no memory holds are asked about too)
  const Wide reach = (Wide)(a.n - 1) * a.step + a.width;
  const Wide d = (Wide)a.at - b.at;  // from b's first byte to a's
  if (d + reach <= 0 || d >= (Wide)(b.n - 1) * b.step + b.width) return false;  // (usually, and without a division)
  const Wide first = d < b.width ? 0 : (d - b.width) / b.step + 1;
  const Wide end = std::min<Wide>(b.n, (d + reach - 1) / b.step + 1);
  if (first >= end) return false;
  // row j meets one where b.at + j b.step - a.at + b.width - 1, modulo a's step, is under both widths together less 1
  const int64_t both = a.width + b.width - 1;
  if (both >= a.step) return true;
  const Wide m = a.step, s = b.step % a.step, o = (first * b.step - d + b.width - 1) % m;  // (not below 0)
  return floor_sum(end - first, s, o + m, m) > floor_sum(end - first, s, o + m - both, m);
}

}  // namespace fs
