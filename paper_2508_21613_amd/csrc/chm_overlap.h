// Whether two operands of a call share memory.  The kernels read inputs while others of their workgroups store results, so the entry points
// refuse results that lie over an input or over each other.
#ifndef CHM_OVERLAP_H
#define CHM_OVERLAP_H
#include <stdint.h>

namespace chm_overlap {

struct Rows { const void *p; int64_t rows, bytes, pitch; };      // rows of `bytes` bytes, pitch >= bytes from one to the next

inline Rows stretch(const void *p, int64_t bytes) { return Rows{p, 1, bytes, bytes}; }

// Exact: columns side by side in the same rows of memory share nothing
inline bool share(Rows a, Rows b) {
  if (!a.p || !b.p || a.rows < 1 || b.rows < 1 || a.bytes < 1 || b.bytes < 1) return false;
  if ((uintptr_t)b.p < (uintptr_t)a.p) { const Rows c = a; a = b; b = c; }
  const int64_t d = (int64_t)((uintptr_t)b.p - (uintptr_t)a.p);
  if (d >= (a.rows - 1) * a.pitch + a.bytes) return false;
  if (a.rows == 1) return true;                                  // b starts within a's only row
  if (a.pitch == b.pitch || b.rows == 1) {
    // b's first row starts in row q of a or in the gap behind it
    const int64_t q = d / a.pitch, r = d - q * a.pitch;
    return r < a.bytes || (r + b.bytes > a.pitch && q + 1 < a.rows);
  }
  // rows of different lengths that start among each other: each row of a against the last one of b that starts before its end
  for (int64_t i = d / a.pitch; i < a.rows; ++i) {
    const int64_t first = i * a.pitch - d, end = first + a.bytes;          // from b's start on
    if (end <= 0) continue;
    int64_t j = (end - 1) / b.pitch;
    if (j >= b.rows) j = b.rows - 1;
    if (j * b.pitch + b.bytes > first) return true;
    if (first >= (b.rows - 1) * b.pitch + b.bytes) break;
  }
  return false;
}

// Whether one of `results` lies over another one or over one of `inputs`
template <int R, int I>
bool clash(const Rows (&results)[R], const Rows (&inputs)[I]) {
  for (int r = 0; r < R; ++r) {
    for (int i = 0; i < I; ++i)
      if (share(results[r], inputs[i])) return true;
    for (int o = 0; o < r; ++o)
      if (share(results[r], results[o])) return true;
  }
  return false;
}

}  // namespace chm_overlap
#endif
