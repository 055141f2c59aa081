// Whether arrays of a call share memory, where each may be a part of wider rows.
#pragma once
#include <algorithm>
#include <numeric>
#include <stdint.h>
#include <utility>

namespace {

// Rows in memory: `bytes` each, `step` bytes from one to the next (step >= bytes)
struct Rows {
  const void *p; // NULL: there are none
  int64_t rows, bytes, step;
};

// bytes from the first to the last (2^62 are more than there are)
inline int64_t span(const Rows &x) { return x.rows - 1 > ((1ll << 62) - x.bytes) / x.step ? 1ll << 62 : (x.rows - 1) * x.step + x.bytes; }

inline bool share(Rows a, Rows b) {
  if (!a.p || !b.p || a.rows < 1 || b.rows < 1 || a.bytes < 1 || b.bytes < 1) return false;
  const int64_t to_a = span(a), to_b = span(b);
  const int64_t d = (int64_t)((uintptr_t)b.p - (uintptr_t)a.p); // where b begins, from a's beginning on
  if (d >= to_a || d + to_b <= 0) return false;
  for (auto [x, to] : {std::pair(&a, to_a), std::pair(&b, to_b)})
    if (x->rows == 1 || x->step == x->bytes) *x = Rows{x->p, 1, to, to}; // nothing between its rows
  // From the first row of a that ends behind b's beginning on, as many as it takes until rows lie to each other as before
  const int64_t first = d < a.bytes ? 0 : (d - a.bytes) / a.step + 1, after = std::min(a.rows, first + b.step / std::gcd(a.step, b.step));
  for (int64_t i = first; i < after; ++i) {
    const int64_t from = i * a.step - d, to = from + a.bytes; // from b's beginning on
    if (from >= to_b) return false;
    const int64_t j = std::min((to - 1) / b.step, b.rows - 1); // the last of b's rows that begins before `to`
    if (j * b.step + b.bytes > from) return true;
  }
  return false;
}
inline bool same_place(const Rows &a, const Rows &b) { return a.p == b.p && a.rows == b.rows && a.bytes == b.bytes && (a.rows <= 1 || a.step == b.step); }

} // namespace
