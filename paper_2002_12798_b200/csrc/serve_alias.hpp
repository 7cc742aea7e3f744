// Whether strided tensors share memory, for the checks of the serving operators' arguments.  Host code only.
#pragma once
#include <algorithm>
#include <cstdint>

namespace amap_serve {

// rows x heads runs of bytes, the first at `at`; strides in bytes, of any sign
struct Runs {
  int64_t at;
  int64_t rows, row;
  int64_t heads, head;
};

// Whether a run of a and a run of b, all of `width` bytes, share a byte.  Exact where the row strides are alike (views of one
// tensor); where they differ, or the heads of different strides are very many, tensors whose first and last bytes overlap
// are taken to share some.
inline bool share(const Runs &a, const Runs &b, int64_t width) {
  const auto low = [](const Runs &t) { return t.at + std::min<int64_t>(0, (t.rows - 1) * t.row) + std::min<int64_t>(0, (t.heads - 1) * t.head); };
  const auto high = [](const Runs &t) { return t.at + std::max<int64_t>(0, (t.rows - 1) * t.row) + std::max<int64_t>(0, (t.heads - 1) * t.head); };
  if (low(a) >= high(b) + width || low(b) >= high(a) + width) return false;
  if (a.rows > 1 && b.rows > 1 && a.row != b.row) return true;
  const bool one_head_stride = a.heads == 1 || b.heads == 1 || a.head == b.head;
  if (!one_head_stride && a.heads * b.heads > (1 << 20)) return true;
  // a run of each is `off` + m * row apart, m any difference of two rows
  const int64_t row = a.rows > 1 ? a.row : b.row, first = 1 - b.rows, last = a.rows - 1;
  const auto near = [&](int64_t off) {
    int64_t m = 0;
    if (row != 0) {
      m = -off / row;
      if (m * row > -off) m -= row > 0 ? 1 : -1;  // the multiple at or below -off
    }
    const int64_t up = row < 0 ? -1 : 1;
    for (const int64_t k : {m, m + up}) {
      const int64_t d = off + std::min(std::max(k, first), last) * row;
      if (d > -width && d < width) return true;
    }
    return false;
  };
  const int64_t apart = a.at - b.at;
  if (one_head_stride) {
    const int64_t head = a.heads > 1 ? a.head : b.head;
    for (int64_t n = 1 - b.heads; n < a.heads; ++n)
      if (near(apart + n * head)) return true;
    return false;
  }
  for (int64_t j = 0; j < a.heads; ++j)
    for (int64_t l = 0; l < b.heads; ++l)
      if (near(apart + j * a.head - l * b.head)) return true;
  return false;
}

}  // namespace amap_serve
