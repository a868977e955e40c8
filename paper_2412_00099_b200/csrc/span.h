// Host: where the rows of a tensor lie in memory, and whether two tensors share a byte.
#pragma once
#include <stdint.h>

#include <initializer_list>

namespace mcce {

// `rows` rows of `width` bytes, `step` bytes apart (step >= width), in [lo, hi); or `count` such blocks, `far` bytes apart (no less than a block
// takes).  Strides and counts that a caller got wrong are cut to what fits.  No address: not part of the call.
struct Span {
  uintptr_t lo, hi;
  int64_t rows, step, width;
  int64_t count = 1, far = 0;
};
inline int64_t bytes_of(int64_t n, int64_t each) {
  int64_t r;
  return __builtin_mul_overflow(n, each, &r) ? INT64_MAX : r;
}
inline Span span(const void* p, int64_t rows, int64_t step, int64_t width) {
  Span s{(uintptr_t)p, (uintptr_t)p, rows, step, width};
  if (p && rows > 0) {
    const unsigned __int128 end = (unsigned __int128)s.lo + (unsigned __int128)(rows - 1) * (uint64_t)step + (uint64_t)width;
    s.hi = end > UINTPTR_MAX ? UINTPTR_MAX : (uintptr_t)end;
  }
  return s;
}
inline Span row_span(const void* p, int64_t rows, int64_t ld, int64_t d, int elem_bytes) {
  return span(p, rows, bytes_of(rows > 1 ? ld : d, elem_bytes), d * elem_bytes);
}
// `count` matrices of `rows` rows
inline Span stack_span(const void* p, int64_t count, int64_t step, int64_t rows, int64_t ld, int64_t d, int elem_bytes) {
  Span s = row_span(p, rows, ld, d, elem_bytes);
  if (!p || count <= 1) return s;
  s.count = count, s.far = bytes_of(step, elem_bytes);
  const unsigned __int128 end = (unsigned __int128)s.hi + (unsigned __int128)(count - 1) * (uint64_t)s.far;
  s.hi = end > UINTPTR_MAX ? UINTPTR_MAX : (uintptr_t)end;
  return s;
}
inline Span flat_span(const void* p, int64_t n, int64_t each = 1) { return span(p, 1, bytes_of(n, each), bytes_of(n, each)); }

// Rows of two tensors may lie between one another (column ranges of one buffer), so their first and last bytes decide only
// where the whole ranges are apart.  Else every row of a is cut to the range of b and compared with b's rows by its place
// in a step of b alone; that place repeats after step_b / gcd(step_a, step_b) rows of a.
inline bool rows_disjoint(const Span& a, const Span& b) {
  typedef __int128 Wide;
  const Wide at = (Wide)a.lo - (Wide)b.lo;   // of a's first row in b
  const Wide b_end = (Wide)b.hi - (Wide)b.lo;
  if (a.rows > 1 && b.rows > 1 && a.step % b.step && a.rows > b.rows) return rows_disjoint(b, a);
  // the rows of a that reach into b's range
  const Wide first = at + a.width > 0 ? 0 : (-at - a.width) / a.step + 1;
  const Wide last_start = (b_end - 1 - at) / a.step, last = last_start < a.rows - 1 ? last_start : (Wide)(a.rows - 1);
  auto meets = [&](Wide i) {
    Wide lo = at + i * a.step, hi = lo + a.width;
    if (lo < 0) lo = 0;
    if (hi > b_end) hi = b_end;
    if (lo >= hi) return false;
    const Wide in = lo % b.step;
    return in < b.width || in + (hi - lo) > b.step;
  };
  if (first > last) return true;
  if (meets(first) || meets(last)) return false;   // the others are not cut
  int64_t divisor = a.step, rest = b.step;
  while (rest) {
    const int64_t r = divisor % rest;
    divisor = rest, rest = r;
  }
  const int64_t period = b.step / divisor;
  for (Wide i = first + 1; i < last && i <= first + period; ++i)
    if (meets(i)) return false;
  return true;
}
// Block i of a span of several
inline Span block_of(const Span& s, int64_t i) {
  return span((const void*)(s.lo + (uintptr_t)i * (uintptr_t)s.far), s.rows, s.step, s.width);
}
inline bool disjoint(const Span& a, const Span& b) {
  if (a.lo >= b.hi || b.lo >= a.hi) return true;
  if (a.count == 1 && b.count == 1) return rows_disjoint(a, b);
  if (a.count > 1 && b.count > 1 && a.far == b.far) {   // only how many blocks apart two are matters, and three such differences are near enough
    typedef __int128 Wide;
    const Wide near = ((Wide)a.lo - (Wide)b.lo) / a.far;
    for (Wide d = near - 1; d <= near + 1; ++d) {       // block i + d of b
      const Wide i = d < 0 ? -d : 0;
      if (i >= a.count || i + d >= b.count) continue;
      if (!disjoint(block_of(a, (int64_t)i), block_of(b, (int64_t)(i + d)))) return false;
    }
    return true;
  }
  // Blocks of either lie one behind the other, so that walking both in the order of their addresses meets every pair that overlaps.
  for (int64_t i = 0, j = 0; i < a.count && j < b.count;) {
    const Span x = block_of(a, i), y = block_of(b, j);
    if (x.lo < y.hi && y.lo < x.hi && !rows_disjoint(x, y)) return false;
    if (x.hi <= y.hi) ++i;
    else ++j;
  }
  return true;
}

// An output that shares no byte with these tensors.
inline bool apart(const Span& out, std::initializer_list<const Span*> others) {
  for (const Span* o : others)
    if (!disjoint(out, *o)) return false;
  return true;
}
// The same for an output that may be this input: row for row the same addresses, or none.
inline bool same_or_apart(const Span& out, const Span& in) {
  return (out.lo == in.lo && out.rows == in.rows && out.step == in.step && out.width == in.width && out.count == in.count && out.far == in.far) ||
         disjoint(out, in);
}

}  // namespace mcce
