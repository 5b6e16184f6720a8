// Tensors of several strided dimensions around a run of consecutive elements: whether their elements are apart, and whether two of them share memory.
#ifndef CHM_STRIDED_H
#define CHM_STRIDED_H
#include <stdint.h>

#include "chm_overlap.h"

namespace chm_strided {

struct Dim { int64_t n, stride; };

// whether n elements `stride` elements apart (up to 8 bytes each) end within what 64 bits count of bytes
inline bool countable(int64_t stride, int64_t n) { return stride >= 0 && (n < 2 || stride <= (1ll << 58) / n); }

// `outer` times (a multiple of `step` bytes apart) some rows
struct Block { const void *p; int64_t outer, step; chm_overlap::Rows rows; };

// Up to three dimensions (sizes and strides in elements) around `width` elements of `size` bytes; strides >= 0
struct Tensor {
  const void *p;
  int64_t run;               // bytes of a run of consecutive elements
  Dim dim[3];                // the others, in bytes, smallest stride first; those of stride 0 (the same elements again) are left out
  int dims;
  bool empty, repeats;       // repeats: a dimension of stride 0

  Tensor(const void *p_, int64_t width, int size, const Dim (&d)[3]) : p(p_), run(width * size), dims(0), empty(width < 1), repeats(false) {
    for (const Dim &x : d) {
      if (x.n < 1) empty = true;
      if (x.n < 2) continue;               // its stride says nothing
      if (x.stride == 0) { repeats = true; continue; }
      int at = dims++;
      for (; at > 0 && dim[at - 1].stride > x.stride * size; --at) dim[at] = dim[at - 1];
      dim[at] = Dim{x.n, x.stride * size};
    }
    while (dims && dim[0].stride == run) {                   // dimensions that follow on one another are one
      run *= dim[0].n;
      drop(0);
    }
    for (int i = 0; i + 1 < dims;)
      if (dim[i + 1].stride == dim[i].n * dim[i].stride) {
        dim[i].n *= dim[i + 1].n;
        drop(i + 1);
      } else {
        ++i;
      }
  }
  void drop(int i) {
    for (--dims; i < dims; ++i) dim[i] = dim[i + 1];
  }
  // whether no two of its elements lie over each other: every dimension steps over all that the smaller ones reach
  bool apart() const {
    if (empty) return true;
    if (repeats) return false;
    int64_t reach = run;
    for (int i = 0; i < dims; ++i) {
      if (dim[i].stride < reach) return false;
      reach += (dim[i].n - 1) * dim[i].stride;
    }
    return true;
  }
  // As rows, or several blocks of rows; with three dimensions left the two smaller ones become one, of all places in between as well
  Block block() const {
    using chm_overlap::Rows;
    if (empty) return Block{nullptr, 0, 0, Rows{nullptr, 0, 0, 0}};
    if (dims == 0) return Block{p, 1, 0, Rows{p, 1, run, run}};
    if (dims == 1) return Block{p, 1, 0, rows(dim[0].n, run, dim[0].stride)};
    if (dims == 2) return Block{p, dim[1].n, dim[1].stride, rows(dim[0].n, run, dim[0].stride)};
    const int64_t reach = (dim[0].n - 1) * dim[0].stride + run;
    if (dim[1].stride % dim[0].stride == 0)
      return Block{p, dim[2].n, dim[2].stride, rows((dim[1].n - 1) * (dim[1].stride / dim[0].stride) + dim[0].n, run, dim[0].stride)};
    return Block{p, dim[2].n, dim[2].stride, rows(dim[1].n, reach, dim[1].stride)};
  }
  // rows that reach into the next (inputs may) are one stretch
  chm_overlap::Rows rows(int64_t n, int64_t bytes, int64_t pitch) const {
    return bytes <= pitch ? chm_overlap::Rows{p, n, bytes, pitch} : chm_overlap::stretch(p, (n - 1) * pitch + bytes);
  }
};

inline bool share(const Tensor &x, const Tensor &y) {
  using chm_overlap::Rows;
  if (!x.p || !y.p || x.empty || y.empty) return false;
  Block a = x.block(), b = y.block();
  const auto reach = [](const Block &t) { return (t.rows.rows - 1) * t.rows.pitch + t.rows.bytes; };
  const auto whole = [&](Block &t) {                         // blocks that reach into each other are one stretch
    if (t.outer > 1 && t.step < reach(t)) t = Block{t.p, 1, 0, chm_overlap::stretch(t.p, (t.outer - 1) * t.step + reach(t))};
  };
  whole(a);
  whole(b);
  const int64_t ra = reach(a), rb = reach(b);
  const char *pa = (const char *)a.p, *pb = (const char *)b.p;
  for (int64_t i = 0, j = 0; i < a.outer && j < b.outer;) {  // both go up in memory
    Rows s = a.rows, t = b.rows;
    s.p = pa + i * a.step;
    t.p = pb + j * b.step;
    if (chm_overlap::share(s, t)) return true;
    const uintptr_t ea = (uintptr_t)s.p + (uintptr_t)ra, eb = (uintptr_t)t.p + (uintptr_t)rb;
    if (ea <= eb) {                                          // skip what ends before the other begins
      const int64_t gap = (int64_t)((uintptr_t)t.p - ea);
      i += a.step > 0 && gap > a.step ? gap / a.step : 1;
    } else {
      const int64_t gap = (int64_t)((uintptr_t)s.p - eb);
      j += b.step > 0 && gap > b.step ? gap / b.step : 1;
    }
  }
  return false;
}

}  // namespace chm_strided
#endif
