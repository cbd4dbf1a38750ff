// Operands of the operators around a layer's products and the checks their ABI
// makes of them (host side).
#pragma once

#include <stdint.h>

#include <initializer_list>
#include <utility>

#include "tcu.h"
#include "tcu_host.h"

namespace tcu {

inline int64_t elem_size(int elem) { return elem == TCU_ELEM_F32 ? 4 : 2; }
inline bool elem_ok(int elem) { return elem >= TCU_ELEM_F32 && elem <= TCU_ELEM_BF16; }
inline bool dim_ok(int64_t n) { return n >= 0 && n <= TCU_MAX_RECT_DIM; }

// One operand: rows x cols elements of es bytes with pitch ld, its base at a
// multiple of `align` bytes.  Of a row's columns those of `runs` runs of `run` elements
// `step` apart, if there are several.
struct Operand {
  const void *p;
  int64_t rows, cols, ld, es;
  int align = 16;
  bool out = false;
  int64_t runs = 1, run = 0, step = 0;
  bool empty() const { return rows <= 0 || cols <= 0; }
  int64_t extent() const { return view_extent(rows, cols, ld, es); }
};

inline bool same_view(const Operand &a, const Operand &b) {
  return a.p == b.p && (a.ld == b.ld || a.rows <= 1) && a.es == b.es;
}

// Whether two operands whose rows meet share no byte all the same, as rows of runs: in
// bytes, w of every run, `step` apart, n of a row, rows `ld` apart.  Exact where their rows
// have one pitch; else found where all pitches are multiples of the smallest.
inline bool runs_apart(const Operand &a, const Operand &b) {
  if (a.runs == 1 && b.runs == 1) return false;
  struct Runs {
    int64_t rows, ld, n, step, w;
  };
  const auto in_bytes = [](const Operand &o) {
    return Runs{o.rows, o.ld * o.es, o.runs, o.step * o.es, (o.runs > 1 ? o.run : o.cols) * o.es};
  };
  Runs x = in_bytes(a), y = in_bytes(b);
  const int64_t d = (int64_t)(reinterpret_cast<uintptr_t>(b.p) - reinterpret_cast<uintptr_t>(a.p));
  // every run of x begins at one place modulo the smallest pitch, every run of y d behind it
  const int64_t pitches[] = {x.rows > 1 ? x.ld : 0, x.n > 1 ? x.step : 0, y.rows > 1 ? y.ld : 0,
                             y.n > 1 ? y.step : 0};
  int64_t least = kMaxExtent;
  for (const int64_t p : pitches)
    if (p > 0 && p < least) least = p;
  bool whole = true;
  for (const int64_t p : pitches) whole = whole && p % least == 0;
  const int64_t at = (d % least + least) % least;
  if (whole && at >= x.w && at + y.w <= least) return true;
  // one pitch of rows: y's first row begins `off` behind row k of x.  (rows of single runs
  // as far apart as the other's runs are: a single row)
  const auto one_row = [](Runs &r, const Runs &other) {
    if (r.n == 1 && r.ld == other.step && r.ld != other.ld) r = Runs{1, other.ld, r.rows, r.ld, r.w};
  };
  one_row(x, y);
  one_row(y, x);
  const int64_t ld = x.rows > 1 ? x.ld : y.ld;
  const auto fits = [&](const Runs &r) {
    return (r.rows == 1 || r.ld == ld) && (r.n - 1) * r.step + r.w <= ld;
  };
  if (!fits(x) || !fits(y)) return false;
  const int64_t off = (d % ld + ld) % ld, k = (d - off) / ld;
  // (rows of y beside rows of x, and those that begin in the row before)
  const auto meet = [&](int64_t k, int64_t off) {
    const void *row = reinterpret_cast<const void *>(reinterpret_cast<uintptr_t>(a.p) + off);
    return k < x.rows && k + y.rows > 0 &&
           views_overlap(a.p, x.n, x.w, x.step, row, y.n, y.w, y.step);
  };
  return !meet(k, off) && !meet(k + 1, off - ld);
}

// The checks every operator makes of its operands: pointers, pitches and
// extents, alignment, and that an output shares no byte with another operand
// (`in_place`: it may be exactly the same view as the input it is paired with).
template <size_t n>
int check_operands(const Operand (&ops)[n],
                   std::initializer_list<std::pair<int, int>> in_place = {}) {
  for (const Operand &o : ops)
    if (!o.p && !o.empty()) return TCU_ERR_NULL;
  for (const Operand &o : ops)
    if (!o.empty() && (o.ld < o.cols || o.ld >= kMaxExtent || o.extent() >= kMaxExtent))
      return TCU_ERR_SHAPE;
  for (const Operand &o : ops)
    if ((reinterpret_cast<uintptr_t>(o.p) & (uintptr_t)(o.align - 1)) != 0) return TCU_ERR_ALIGN;
  for (size_t i = 0; i < n; ++i) {
    if (!ops[i].out || ops[i].empty()) continue;
    for (size_t j = 0; j < n; ++j) {
      if (j == i || ops[j].empty() || (ops[j].out && j < i)) continue;
      bool paired = false;
      for (const auto &pr : in_place)
        if (pr.first == (int)i && pr.second == (int)j && same_view(ops[i], ops[j])) paired = true;
      if (paired) continue;
      const Operand &a = ops[i], &b = ops[j];
      if (views_overlap(a.p, a.rows, a.cols * a.es, a.ld * a.es, b.p, b.rows, b.cols * b.es,
                        b.ld * b.es) &&
          !runs_apart(a, b))
        return TCU_ERR_OVERLAP;
    }
  }
  return TCU_OK;
}

// With pointer checks on, every operand's whole extent.
template <size_t n>
int check_device(const Operand (&ops)[n]) {
  if (!checks_on()) return TCU_OK;
  for (const Operand &o : ops) {
    const int rc = device_range(o.p, o.extent());
    if (rc != TCU_OK) return rc;
  }
  return TCU_OK;
}

// A vector of n elements as an operand.
inline Operand vec(const void *p, int64_t n, int64_t es, int align, bool out = false) {
  return Operand{p, 1, n, n, es, align, out};
}

inline int64_t blocks(int64_t n, int64_t s) { return (n + s - 1) / s; }

}  // namespace tcu
