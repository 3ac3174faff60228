// Argument checks shared by the host sides of the C entry points.
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace cts {

struct Range { const void* p; size_t bytes; };

// Every float array is read or written in 16-byte vectors: its address must be
// a multiple of 16 (ids: of 4).
inline bool misaligned(const void* ptr, uintptr_t a) {
  return (reinterpret_cast<uintptr_t>(ptr) & (a - 1)) != 0;
}

inline bool overlap(Range a, Range b) {
  if (!a.p || !b.p || !a.bytes || !b.bytes) return false;
  const uintptr_t a0 = reinterpret_cast<uintptr_t>(a.p), b0 = reinterpret_cast<uintptr_t>(b.p);
  return a0 < b0 + b.bytes && b0 < a0 + a.bytes;
}

// `rows` rows of `width` bytes, `ld` bytes apart.
struct Rows { const void* p; uint64_t rows, width, ld; };

inline Range extent(Rows a) { return {a.p, a.p && a.rows ? (a.rows - 1) * a.ld + a.width : 0}; }

// Rows of the same stride may interleave without meeting (the slices of one
// packed array); other strides count as meeting where their extents do.
inline bool overlap(Rows a, Rows b) {
  if (!overlap(extent(a), extent(b))) return false;
  if (a.ld != b.ld || !a.ld) return true;
  const uintptr_t a0 = reinterpret_cast<uintptr_t>(a.p), b0 = reinterpret_cast<uintptr_t>(b.p);
  const uint64_t d = b0 >= a0 ? (b0 - a0) % a.ld : (a.ld - (a0 - b0) % a.ld) % a.ld;   // b's column in a's rows
  return d < a.width || d + b.width > a.ld;
}

inline bool same(Rows a, Rows b) { return a.p == b.p && a.ld == b.ld; }

}  // namespace cts
