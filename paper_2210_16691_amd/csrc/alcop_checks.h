// Checks of arguments that the host code of the operators shares.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "../../include/alcop.h"

namespace alcop {

inline int size_of(alcop_dtype t) { return t == ALCOP_F32 ? 4 : t == ALCOP_E4M3 ? 1 : 2; }
inline bool is_half(alcop_dtype t) { return t == ALCOP_F16 || t == ALCOP_BF16; }
inline bool aligned(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) == 0; }

// A matrix in memory, in bytes.
struct Span {
  const char* p;
  double rows, row, pitch;
  Span(const void* ptr, int rows_, int cols, long ld, int size)
      : p((const char*)ptr), rows(rows_), row((double)cols * size), pitch((double)ld * size)
  {
  }
};
// Whether two matrices share bytes.  Column ranges of one buffer, rows equally far apart, do not.
inline bool meet(const Span& a, const Span& b)
{
  if (!a.p || !b.p) return false;
  const double ea = (a.rows - 1) * a.pitch + a.row, eb = (b.rows - 1) * b.pitch + b.row;
  if (!(a.p < b.p + (size_t)eb && b.p < a.p + (size_t)ea)) return false;
  if (a.pitch != b.pitch || a.rows < 2 || b.rows < 2) return true;
  const long pitch = (long)a.pitch;
  const long d = (long)((((b.p - a.p) % pitch) + pitch) % pitch);      // b's columns start d bytes behind a's
  return !(d >= (long)a.row && d + (long)b.row <= pitch);
}
inline bool same(const Span& a, const Span& b) { return a.p == b.p && (a.rows < 2 || a.pitch == b.pitch) && a.row == b.row; }

inline size_t r256(double bytes) { return ((size_t)bytes + 255) & ~(size_t)255; }

}  // namespace alcop
