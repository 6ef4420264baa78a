// Argument checks that the entry points of sva_cache_api.hip and sva_layer_api.hip share.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <algorithm>

#include "../../include/sva.h"
#include "overlap.h"
#include "sva_internal.h"

namespace sva {
namespace api {

inline bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) % n) == 0; }

inline int hip_status(hipError_t e) { return e == hipSuccess ? SVA_OK : SVA_ERR_HIP; }

// One strided tensor [B, heads, N, D]: its view, and the bytes from its first
// element to behind its last.
struct Tensor {
  HeadsView v;
  size_t span;
  int align;                     // what data and strides are multiples of: 16, 8, 4 or 2 bytes
  RowSet rows;
};

inline int check_heads(const sva_heads* h, int64_t B, int64_t N, int64_t D, size_t item, bool wide, bool output, Tensor* t) {
  if (!h || !h->data || h->heads < 1) return SVA_ERR_INVALID_ARG;
  if (h->stride_b < 0 || h->stride_h < 0 || h->stride_n < 0) return SVA_ERR_INVALID_ARG;
  struct Dim {
    int64_t size, stride;
  };
  // a dimension of one has no stride
  Dim dims[3] = {{B, B > 1 ? h->stride_b : 0}, {h->heads, h->heads > 1 ? h->stride_h : 0}, {N, N > 1 ? h->stride_n : 0}};
  int64_t span = D;
  for (const Dim& d : dims) {
    int64_t x;
    if (__builtin_mul_overflow(d.size - 1, d.stride, &x) || __builtin_add_overflow(span, x, &span)) return SVA_ERR_SHAPE;
  }
  if (span > ((int64_t)1 << 58)) return SVA_ERR_SHAPE;
  int align = 16;
  auto fits = [&](int n) {
    bool all = aligned(h->data, n);
    for (const Dim& d : dims) all = all && d.stride * (int64_t)item % n == 0;
    return all;
  };
  while (align > (int)item && !fits(align)) align /= 2;
  if (!aligned(h->data, item) || (wide && align < 16)) return SVA_ERR_ALIGNMENT;
  if (output) {                  // rows must not overlap
    std::sort(dims, dims + 3, [](const Dim& a, const Dim& b) { return a.stride < b.stride; });
    int64_t reach = D;
    for (const Dim& d : dims) {
      if (d.size == 1) continue;
      if (d.stride < reach) return SVA_ERR_INVALID_ARG;
      reach += (d.size - 1) * d.stride;
    }
  }
  t->v.p = h->data;
  t->v.sb = h->stride_b;
  t->v.sh = h->stride_h;
  t->v.sn = h->stride_n;
  t->v.heads = h->heads;
  t->span = (size_t)span * item;
  t->align = align;
  t->rows.at = reinterpret_cast<uintptr_t>(h->data);
  t->rows.row = D * (int64_t)item;
  for (int i = 0; i < 3; ++i) {
    t->rows.size[i] = dims[i].size;
    t->rows.stride[i] = dims[i].stride * (int64_t)item;
  }
  return SVA_OK;
}

inline bool apart(const Tensor& x, const Tensor& y) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(x.v.p), b = reinterpret_cast<uintptr_t>(y.v.p);
  return a + x.span <= b || b + y.span <= a;
}

// `rows` runs of `row` bytes as a tensor.
inline Tensor runs_of(const void* p, int64_t rows, int64_t stride, int64_t row) {
  Tensor t{};
  t.v.p = const_cast<void*>(p);
  t.span = (size_t)((rows - 1) * stride + row);
  t.rows = {reinterpret_cast<uintptr_t>(p), row, {rows, 1, 1}, {stride, 0, 0}};
  return t;
}

// Whether they share a byte: apart() by rows, not by spans.
inline bool meet(const Tensor& x, const Tensor& y) { return !apart(x, y) && rows_meet(x.rows, y.rows); }

inline bool same(const Tensor& x, const Tensor& y, int64_t B, int64_t N) {
  return x.v.p == y.v.p && (B == 1 || x.v.sb == y.v.sb) && (x.v.heads == 1 || x.v.sh == y.v.sh) &&
         (N == 1 || x.v.sn == y.v.sn);
}

inline bool good_dtype(int32_t t) { return t == SVA_BF16 || t == SVA_F32; }
inline size_t item_of(int32_t t) { return t == SVA_F32 ? 4 : 2; }

}  // namespace api
}  // namespace sva
