// Where strided operands lie in memory, for checks on the host.
#pragma once
#include <algorithm>
#include <cstdint>
#include <initializer_list>
#include <numeric>

namespace nc {

// The bytes of a strided operand: runs of `run` bytes, n[0] x n[1] x n[2] of them at
// these strides (bytes).  NULL or a count of 0: none.
struct Area {
  const void* base;
  int64_t run;
  int64_t n[3], stride[3];

  // one run of elements
  Area(const void* p, int64_t count, int64_t size) : base(count > 0 ? p : nullptr), run(count * size), n{1, 1, 1}, stride{} {}
  // up to three strided dimensions of 16-bit rows; a dimension of one entry, or of stride 0, adds nothing
  Area(const void* p, int64_t row, std::initializer_list<int64_t> dims) : base(p), run(2 * row), n{1, 1, 1}, stride{} {
    int i = 0;
    for (auto d = dims.begin(); d != dims.end(); d += 2) {
      if (d[0] < 1) base = nullptr;
      if (d[0] > 1 && d[1] > 0) {
        n[i] = d[0];
        stride[i++] = 2 * d[1];
      }
    }
  }
  // bytes from the first to past the last, of the dimensions whose stride is below `limit`
  __int128 extent(int64_t limit) const {
    __int128 e = run;
    for (int i = 0; i < 3; ++i)
      if (stride[i] < limit) e += (__int128)(n[i] - 1) * stride[i];
    return e;
  }
};

// Whether two operands are seen to share no byte: they lie one behind the other, or
// inside different parts of a common period, as the columns of one buffer do.
inline bool apart(const Area& a, const Area& b) {
  if (!a.base || !b.base) return true;
  const __int128 delta = (__int128)(uintptr_t)b.base - (__int128)(uintptr_t)a.base;
  if (delta >= a.extent(INT64_MAX) || -delta >= b.extent(INT64_MAX)) return true;
  for (const Area* from : {&a, &b})
    for (const int64_t limit : from->stride) {  // the dimensions from this stride on make the period
      if (limit == 0) continue;
      int64_t period = 0;
      for (const Area* x : {&a, &b})
        for (const int64_t s : x->stride)
          if (s >= limit) period = std::gcd(period, s);
      const __int128 r = (delta % period + period) % period;
      if (r >= a.extent(limit) && r + b.extent(limit) <= period) return true;
    }
  return false;
}
inline bool all_apart(const Area& out, std::initializer_list<Area> others) {
  return std::all_of(others.begin(), others.end(), [&](const Area& x) { return apart(out, x); });
}

}  // namespace nc
