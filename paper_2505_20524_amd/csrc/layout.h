// Where strided tensors lie, and whether two of them are seen to lie apart.  Host code.
#pragma once
#include <stdint.h>

#include "../../include/fog.h"

// Rows of `row` bytes: bytes between neighbours, largest first, of the dimensions that have more than one.
struct FogBox {
  uintptr_t base;
  int dims;
  int64_t n[3], stride[3], row;
  int64_t extent(int from) const {
    int64_t e = row;
    for (int i = from; i < dims; ++i) e += (n[i] - 1) * stride[i];
    return e;
  }
};

// Rows of `elements` elements of `size` bytes; strides in elements.
static inline fog_status fog_make_box(const void* p, int dims, const int64_t* n, const int64_t* stride, int64_t elements, int size, FogBox* box) {
  if (!p) return FOG_ERR_NULL;
  box->base = reinterpret_cast<uintptr_t>(p);
  if (box->base & (uintptr_t)(size - 1)) return FOG_ERR_ALIGN;
  box->dims = 0;
  box->row = elements * size;
  for (int i = 0; i < dims; ++i) {
    if (n[i] <= 1) continue;
    if (stride[i] < 0) return FOG_ERR_SHAPE;
    if ((double)(n[i] - 1) * (double)stride[i] * size > 140737488355328.0) return FOG_ERR_UNSUPPORTED;      // 2^47 bytes: more than an address space holds
    int at = box->dims++;
    for (; at > 0 && box->stride[at - 1] < stride[i] * size; --at) {
      box->n[at] = box->n[at - 1];
      box->stride[at] = box->stride[at - 1];
    }
    box->n[at] = n[i];
    box->stride[at] = stride[i] * size;
  }
  return FOG_OK;
}

// Whether no row of a box lies on another of it.
static inline bool fog_injective(const FogBox& a) {
  for (int i = 0; i < a.dims; ++i)
    if (a.stride[i] < a.extent(i + 1)) return false;
  return true;
}

// Whether two boxes are seen to lie apart, b's first row `off` bytes behind a's: one ends before the other begins, or both step by the same
// distance and lie apart within a step.  (A step of a has two neighbours of b: the one at `off` modulo the distance and the one before.)
static inline bool fog_apart_from(const FogBox& a, int ia, const FogBox& b, int ib, int64_t off) {
  if (off >= a.extent(ia) || -off >= b.extent(ib)) return true;
  if (ia >= a.dims || ib >= b.dims || a.stride[ia] != b.stride[ib] || a.stride[ia] <= 0) return false;
  const int64_t s = a.stride[ia], r = ((off % s) + s) % s;
  return fog_apart_from(a, ia + 1, b, ib + 1, r) && fog_apart_from(a, ia + 1, b, ib + 1, r - s);
}
static inline bool fog_apart(const FogBox& a, const FogBox& b) { return fog_apart_from(a, 0, b, 0, (int64_t)(b.base - a.base)); }
static inline bool fog_apart_as_spans(const FogBox& a, const FogBox& b) {
  return a.base + (uintptr_t)a.extent(0) <= b.base || b.base + (uintptr_t)b.extent(0) <= a.base;
}

// The matrices of a call: what it writes has to lie apart from everything else, but for results in the place of an input.
struct FogMatrices {
  static constexpr int MOST = 8;
  FogBox box[MOST];
  bool written[MOST];
  int count = 0;
  // A matrix that may be left out (NULL): nothing to look at.
  fog_status add(const void* p, int64_t rows, int64_t cols, int64_t ld, int size, bool is_written) {
    if (!p) return FOG_OK;
    if (ld < cols) return FOG_ERR_SHAPE;
    const fog_status st = fog_make_box(p, 1, &rows, &ld, cols, size, &box[count]);
    if (st != FOG_OK) return st;
    written[count++] = is_written;
    return FOG_OK;
  }
  bool fine() const {
    for (int i = 0; i < count; ++i)
      for (int k = 0; k < i; ++k) {
        if (!written[i] && !written[k]) continue;
        const FogBox &a = box[i], &b = box[k];
        const bool same = written[i] != written[k] && a.base == b.base && a.row == b.row && a.dims == b.dims && (a.dims == 0 || a.stride[0] == b.stride[0]);
        if (!same && !fog_apart(a, b)) return false;
      }
    return true;
  }
};
