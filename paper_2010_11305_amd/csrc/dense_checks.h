// What the host sides of the dense operators check and convert alike: alignment, element types, sizes, overlap.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "dense_internal.h"

namespace embd {

constexpr size_t kAlign = 256;
inline size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
inline hipStream_t S(void* s) { return reinterpret_cast<hipStream_t>(s); }
inline int status(hipError_t e) { return e == hipSuccess ? EMB_OK : EMB_EHIP; }
inline bool aligned(const void* p) { return reinterpret_cast<uintptr_t>(p) % kAlign == 0; }

inline int type_bytes(int32_t type) { return type == EMB_TYPE_FP32 ? 4 : 2; }
inline bool type_ok(int32_t type) { return type == EMB_TYPE_FP32 || type == EMB_TYPE_BF16 || type == EMB_TYPE_FP16; }
inline bool rounding_ok(int32_t r) { return r == EMB_ROUND_NEAREST || r == EMB_ROUND_STOCHASTIC; }

// Sizes an MX4 matrix may have: below 2^31 each way, and a buffer that can exist.
inline bool dims_ok(int64_t rows, int64_t cols) {
  if (rows < 0 || cols < 0 || rows >= kMaxDim || cols >= kMaxDim) return false;
  const Mx4 q(nullptr, rows, cols);   // at most 2^27 row tiles of 2^24 column tiles: no overflow of 64 bits
  return (double)q.bytes() <= kMaxBytes;
}

// The operands of a product.
inline bool product_ok(int64_t m, int64_t n, int64_t k) { return dims_ok(m, k) && dims_ok(n, k) && k <= kMaxDepth; }

// A full-precision matrix: element-aligned, rows not overlapping, inside the address space.
inline bool matrix_ok(const void* x, int32_t type, int64_t rows, int64_t cols, int64_t ld) {
  if (!x || reinterpret_cast<uintptr_t>(x) % type_bytes(type) || ld < cols) return false;
  return (double)rows * (double)ld * type_bytes(type) <= 4.0 * kMaxBytes;
}

// Whether two matrices share an element; row by row where their strides differ.
inline bool share_elements(const void* x, int64_t x_rows, int64_t x_cols, int64_t x_ld, const void* y, int64_t y_rows,
                           int64_t y_cols, int64_t y_ld, int64_t bytes) {
  if (!x_rows || !x_cols || !y_rows || !y_cols) return false;
  const int64_t to = (int64_t)(reinterpret_cast<uintptr_t>(y) - reinterpret_cast<uintptr_t>(x));
  const int64_t xw = x_cols * bytes, xs = x_ld * bytes, yw = y_cols * bytes, ys = y_ld * bytes;
  if (to >= (x_rows - 1) * xs + xw || to + (y_rows - 1) * ys + yw <= 0) return false;
  if (xs == ys && xs > 0) {   // rows i of x and k of y do where to - xw < (i - k) xs < to + yw
    const int64_t low = to - xw, above = low < 0 ? -(-low / xs) : low / xs;        // low / xs cut towards zero
    int64_t q = low < 0 && -low % xs ? above : above + 1;                           // the least with q xs > low
    if (q < -(y_rows - 1)) q = -(y_rows - 1);
    return q <= x_rows - 1 && q * xs < to + yw;
  }
  for (int64_t i = 0; i < x_rows; ++i) {
    const int64_t before = i * xs - to - yw;                 // rows of y that start there or earlier end before row i of x
    const int64_t k = before < 0 ? 0 : before / ys + 1;
    if (k < y_rows && to + k * ys < i * xs + xw) return true;
  }
  return false;
}

}  // namespace embd
