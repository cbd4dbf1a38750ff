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
// multiple of `align` bytes.
struct Operand {
  const void *p;
  int64_t rows, cols, ld, es;
  int align = 16;
  bool out = false;
  bool empty() const { return rows <= 0 || cols <= 0; }
  int64_t extent() const { return view_extent(rows, cols, ld, es); }
};

inline bool same_view(const Operand &a, const Operand &b) {
  return a.p == b.p && (a.ld == b.ld || a.rows <= 1) && a.es == b.es;
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
                        b.ld * b.es))
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
