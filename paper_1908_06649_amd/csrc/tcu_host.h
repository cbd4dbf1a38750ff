// Host-side helpers of the ABI layers: device query, argument checks and cost
// accounting (defined in tcu_abi.cpp).
#pragma once

#include <stdint.h>

#include <initializer_list>
#include <utility>

#include "tcu.h"

namespace tcu {

// Extents from here on are refused.
constexpr int64_t kMaxExtent = (int64_t)1 << 40;

inline bool misaligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

// Resolve the current device and check it is a gfx950; fills its CU count.
int device_ready(int *num_cus);

// With pointer checks on, every operand extent (pointer, bytes) in turn.
int check_ranges(std::initializer_list<std::pair<const void *, int64_t>> ranges);
int device_range(const void *p, int64_t bytes);
bool checks_on();

// Bytes from the base of an R x C view with row pitch ld (elements of es
// bytes) to one past its last element, saturated at 2^62; 0 for an empty view.
int64_t view_extent(int64_t rows, int64_t cols, int64_t ld, int64_t es);

// Whether two row-major views (base, rows, bytes per row, byte pitch) share a
// byte.
bool views_overlap(const void *a, int64_t ar, int64_t aw, int64_t ap, const void *b, int64_t br,
                   int64_t bw, int64_t bp);

// Count `calls` tall calls of M rows each with unit size s.
void count_tall(int64_t calls, int64_t M, int s);

// The calling thread's unit size (tcu_set_unit).
int unit_size();

}  // namespace tcu
