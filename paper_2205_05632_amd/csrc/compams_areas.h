// What a call reads and writes, and whether two such areas share memory.  Plain host functions.
#pragma once

#include <numeric>

#include <stddef.h>
#include <stdint.h>

namespace compams {

// Rows of `bytes` bytes, `ld` bytes apart: what a call reads or writes.
struct Area {
  const void* p;
  int64_t rows, bytes, ld;
};
inline Area area(const void* p, int64_t rows, int64_t cols, int64_t ld, size_t size) {
  return {p, rows, cols * static_cast<int64_t>(size), ld * static_cast<int64_t>(size)};
}
// Whether two areas share a byte: if their extents do, and the places of their rows within the distance from row to row.  (Of
// two distances, within the largest that divides both: areas that meet nowhere there are apart.)  What is empty, and a null
// pointer, shares nothing.
inline bool meet(const Area& a, const Area& b) {
  typedef __int128 Wide;
  if (!a.p || !b.p || a.rows <= 0 || b.rows <= 0 || a.bytes <= 0 || b.bytes <= 0) return false;
  const auto extent = [](const Area& v) { return static_cast<Wide>(v.rows - 1) * v.ld + v.bytes; };
  // b's first byte, from a's
  const Wide from = reinterpret_cast<intptr_t>(b.p) - static_cast<Wide>(reinterpret_cast<intptr_t>(a.p));
  if (from >= extent(a) || -from >= extent(b)) return false;
  if (a.rows == 1 && b.rows == 1) return true;
  const int64_t ld = a.rows == 1 ? b.ld : b.rows == 1 ? a.ld : std::gcd(a.ld, b.ld);
  if (ld <= 0) return true;
  const int64_t at = static_cast<int64_t>((from % ld + ld) % ld);
  return at < a.bytes || at + b.bytes > ld;
}
// The same place: what may be written over what is read there.
inline bool same(const Area& a, const Area& b) { return a.p == b.p && (a.rows <= 1 || a.ld == b.ld); }

// A weight's gradients, for n workers a matrix of floats each: as an area, a worker's extent to a row.
struct Gradients {
  const float* p;
  int64_t n, rows, cols, ld, stride;
  Area extents() const { return area(p, n, (rows - 1) * (rows > 1 ? ld : 0) + cols, stride, sizeof(float)); }
  Area of(int64_t worker) const { return area(p + worker * stride, rows, cols, ld, sizeof(float)); }
};
// Whether the gradients of two weights share memory, as far as a worker's and its neighbour's show.
inline bool meet(const Gradients& a, const Gradients& b) {
  if (!a.p || !b.p) return false;
  if (meet(a.of(0), b.of(0))) return true;
  return a.n > 1 && (meet(a.of(0), b.of(1)) || meet(a.of(1), b.of(0)));
}

}  // namespace compams
