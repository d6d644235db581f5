// The root-mean-square norm of rows with the residual's addition, its output in 8 bits, and its gradients.
//
// Rows of any width: a workgroup takes a row and goes over it as often as it has to, a thread always over the same 8
// columns at a time, so that what it wrote in one pass it reads in the next.
#include "dense_device.h"

namespace embd {

namespace {

constexpr int kThreads = 256;
constexpr int kPer = 8;

// The sum, and the largest, of a value over the workgroup, for every thread.  `part` is LDS of a wave's
// number of values; it may be used again after a barrier.
template <class T, int THREADS>
__device__ __forceinline__ T block_sum(T v, T* part) {
#pragma unroll
  for (int m = 32; m; m >>= 1) v += __shfl_xor(v, m);
  if constexpr (THREADS > 64) {
    __syncthreads();
    if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w) v += part[w];
  }
  return v;
}
template <int THREADS>
__device__ __forceinline__ uint32_t block_max(uint32_t v, uint32_t* part) {
#pragma unroll
  for (int m = 32; m; m >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, m));
  if constexpr (THREADS > 64) {
    __syncthreads();
    if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w) v = max(v, part[w]);
  }
  return v;
}

__device__ __forceinline__ float inverse_of(double squares, int64_t cols, float eps) {
  return (float)(1.0 / sqrt(squares / (double)cols + (double)eps));
}

// 8 codes of 8-bit rows at any address.
struct __attribute__((packed, aligned(1))) Codes8 {
  uint32_t w[2];
};

// What 127 stands for, over 127: not below the normal numbers, so that its reciprocal is finite.
__device__ __forceinline__ float scale8(uint32_t amax) {
  return fmaxf(__uint_as_float(amax) / 127.0f, 0x1p-126f);
}

// 8 values to codes.  |v| <= 127.00003 scale, so nothing passes 127.
__device__ __forceinline__ Codes8 codes8(const float (&v)[kPer], float per) {
  Codes8 c = {{0, 0}};
#pragma unroll
  for (int j = 0; j < kPer; ++j) c.w[j / 4] |= ((uint32_t)(int)rintf(v[j] * per) & 0xFFu) << (8 * (j % 4));
  return c;
}

__device__ __forceinline__ void store_codes(int8_t* p, int n, const Codes8& c) {
  if (n == kPer) {
    *reinterpret_cast<Codes8*>(p) = c;
    return;
  }
#pragma unroll
  for (int j = 0; j < kPer; ++j)
    if (j < n) p[j] = (int8_t)(c.w[j / 4] >> (8 * (j % 4)));
}

template <int T>
__device__ __forceinline__ typename Elem<T>::type* row_of(const Rows& r, int64_t row) {
  return static_cast<typename Elem<T>::type*>(const_cast<void*>(r.p)) + row * r.ld;
}

// h of 8 columns: x, or x + residual rounded to the type.
template <int T>
__device__ __forceinline__ Raw<T, kPer> load_h(const NormForward& a, int64_t row, int64_t c, int n) {
  Raw<T, kPer> h;
  load_values(row_of<T>(a.x, row) + c, n, h);
  if (a.residual.p) {
    Raw<T, kPer> r;
    load_values(row_of<T>(a.residual, row) + c, n, r);
#pragma unroll
    for (int j = 0; j < kPer; ++j) h.put(j, to_bits<T>(h.get(j) + r.get(j)));
  }
  return h;
}

// gain of 8 columns, ones where there is none.
template <int GT>
__device__ __forceinline__ void load_gain(const void* gain, int64_t c, int n, float (&g)[kPer]) {
  if (!gain) {
#pragma unroll
    for (int j = 0; j < kPer; ++j) g[j] = 1.0f;
    return;
  }
  Raw<GT, kPer> r;
  load_values(static_cast<const typename Elem<GT>::type*>(gain) + c, n, r);
#pragma unroll
  for (int j = 0; j < kPer; ++j) g[j] = r.get(j);
}

template <int T, int GT, bool BITS8>
__global__ __launch_bounds__(kThreads) void k_norm(NormForward a, int64_t first) {
  __shared__ double sums[kThreads / 64];
  __shared__ uint32_t tops[kThreads / 64];
  const int64_t row = first + blockIdx.x;
  double squares = 0.0;
  for (int64_t c = (int64_t)threadIdx.x * kPer; c < a.cols; c += kThreads * kPer) {
    const int n = a.cols - c < kPer ? (int)(a.cols - c) : kPer;
    const Raw<T, kPer> h = load_h<T>(a, row, c, n);
    if (a.sum.p) store_values(row_of<T>(a.sum, row) + c, n, h);
#pragma unroll
    for (int j = 0; j < kPer; ++j) squares = fma((double)h.get(j), (double)h.get(j), squares);
  }
  const float inverse = inverse_of(block_sum<double, kThreads>(squares, sums), a.cols, a.eps);
  if (a.inverse && threadIdx.x == 0) a.inverse[row] = inverse;
  const auto again = [&](int64_t c, int n, float (&v)[kPer]) {
    Raw<T, kPer> h;
    if (a.sum.p)
      load_values(row_of<T>(a.sum, row) + c, n, h);
    else
      h = load_h<T>(a, row, c, n);
    float g[kPer];
    load_gain<GT>(a.gain, c, n, g);
#pragma unroll
    for (int j = 0; j < kPer; ++j) v[j] = h.get(j) * inverse * g[j];
  };
  float v[kPer];
  if constexpr (!BITS8) {
    for (int64_t c = (int64_t)threadIdx.x * kPer; c < a.cols; c += kThreads * kPer) {
      const int n = a.cols - c < kPer ? (int)(a.cols - c) : kPer;
      again(c, n, v);
      Raw<T, kPer> y;
#pragma unroll
      for (int j = 0; j < kPer; ++j) y.put(j, to_bits<T>(v[j]));
      store_values(row_of<T>(a.y, row) + c, n, y);
    }
  } else {
    uint32_t top = 0;
    for (int64_t c = (int64_t)threadIdx.x * kPer; c < a.cols; c += kThreads * kPer) {
      const int n = a.cols - c < kPer ? (int)(a.cols - c) : kPer;
      again(c, n, v);
#pragma unroll
      for (int j = 0; j < kPer; ++j)
        if (j < n) top = max(top, __float_as_uint(v[j]) & 0x7FFFFFFFu);
    }
    top = block_max<kThreads>(top, tops);
    const bool fine = top < 0x7F800000u;
    const float scale = scale8(top), per = fine ? 1.0f / scale : 0.0f;
    if (threadIdx.x == 0) a.scales[row] = fine ? scale : __uint_as_float(0x7FC00000u);
    int8_t* out = static_cast<int8_t*>(const_cast<void*>(a.y.p)) + row * a.y.ld;
    for (int64_t c = (int64_t)threadIdx.x * kPer; c < a.cols; c += kThreads * kPer) {
      const int n = a.cols - c < kPer ? (int)(a.cols - c) : kPer;
      again(c, n, v);
      store_codes(out + c, n, fine ? codes8(v, per) : Codes8{{0, 0}});
    }
  }
}

// The gradient of h, a workgroup a row.
template <int T, int GT>
__global__ __launch_bounds__(kThreads) void k_norm_dx(NormBackward a, int64_t first) {
  __shared__ double sums[kThreads / 64];
  const int64_t row = first + blockIdx.x;
  const float inverse = a.inverse[row];
  double along = 0.0;
  const auto part = [&](int64_t c, int n, float (&dn)[kPer], float (&u)[kPer]) {
    Raw<T, kPer> d, h;
    load_values(row_of<T>(a.dy, row) + c, n, d);
    load_values(row_of<T>(a.h, row) + c, n, h);
    float g[kPer];
    load_gain<GT>(a.gain, c, n, g);
#pragma unroll
    for (int j = 0; j < kPer; ++j) dn[j] = d.get(j) * g[j], u[j] = h.get(j) * inverse;
  };
  float dn[kPer], u[kPer];
  for (int64_t c = (int64_t)threadIdx.x * kPer; c < a.cols; c += kThreads * kPer) {
    const int n = a.cols - c < kPer ? (int)(a.cols - c) : kPer;
    part(c, n, dn, u);
#pragma unroll
    for (int j = 0; j < kPer; ++j)
      if (j < n) along += (double)(dn[j] * u[j]);
  }
  const float mean = (float)(block_sum<double, kThreads>(along, sums) / (double)a.cols);
  for (int64_t c = (int64_t)threadIdx.x * kPer; c < a.cols; c += kThreads * kPer) {
    const int n = a.cols - c < kPer ? (int)(a.cols - c) : kPer;
    part(c, n, dn, u);
    Raw<T, kPer> s = {}, out;
    if (a.dsum.p) load_values(row_of<T>(a.dsum, row) + c, n, s);
#pragma unroll
    for (int j = 0; j < kPer; ++j) out.put(j, to_bits<T>((dn[j] - u[j] * mean) * inverse + s.get(j)));
    store_values(row_of<T>(a.dx, row) + c, n, out);
  }
}

// A slab's part of the gain's gradient: a thread a column.  It runs before k_norm_dx, which may write over dy and h.
template <int T>
__global__ __launch_bounds__(kThreads) void k_norm_gain(NormBackward a, int64_t first) {
  const int64_t wide = ceil_div(a.cols, kThreads), block = first + blockIdx.x;
  const int64_t slab = block / wide, c = block % wide * kThreads + threadIdx.x;
  if (c >= a.cols) return;
  const int64_t row0 = slab * kNormSlabRows, row1 = row0 + kNormSlabRows < a.rows ? row0 + kNormSlabRows : a.rows;
  float sum = 0.0f;
  for (int64_t row = row0; row < row1; ++row) {
    Raw<T, 4 / Elem<T>::kBytes> d, h;
    d.w[0] = load_bits<T>(row_of<T>(a.dy, row) + c);
    h.w[0] = load_bits<T>(row_of<T>(a.h, row) + c);
    sum += d.get(0) * (h.get(0) * a.inverse[row]);
  }
  a.partial[slab * a.cols + c] = sum;
}

template <int GT>
__global__ __launch_bounds__(kThreads) void k_norm_gain_join(const float* __restrict__ partial, int64_t slabs, int64_t cols,
                                                             typename Elem<GT>::type* __restrict__ out, int64_t first) {
  const int64_t c = (first + blockIdx.x) * kThreads + threadIdx.x;
  if (c >= cols) return;
  double sum = 0.0;
  for (int64_t s = 0; s < slabs; ++s) sum += (double)partial[s * cols + c];
  if constexpr (GT == EMB_TYPE_FP32)
    out[c] = (float)sum;
  else
    out[c] = (uint16_t)to_bits<GT>((float)sum);
}

template <int T>
__global__ __launch_bounds__(kThreads) void k_rows8_dequantize(const int8_t* __restrict__ codes, int64_t rows, int64_t cols,
                                                               int64_t ldc, const float* __restrict__ scales,
                                                               typename Elem<T>::type* __restrict__ x, int64_t ldx,
                                                               int64_t first) {
  const int64_t wide = ceil_div(cols, kPer), i = (first + blockIdx.x) * kThreads + threadIdx.x;
  const int64_t row = i / wide, c = i % wide * kPer;
  if (row >= rows) return;
  const int n = cols - c < kPer ? (int)(cols - c) : kPer;
  const int8_t* p = codes + row * ldc + c;
  Codes8 q = {{0, 0}};
  if (n == kPer) {
    q = *reinterpret_cast<const Codes8*>(p);
  } else {
#pragma unroll
    for (int j = 0; j < kPer; ++j)
      if (j < n) q.w[j / 4] |= (uint32_t)(uint8_t)p[j] << (8 * (j % 4));
  }
  const float scale = scales[row];
  Raw<T, kPer> out;
#pragma unroll
  for (int j = 0; j < kPer; ++j) out.put(j, to_bits<T>((float)(int8_t)(q.w[j / 4] >> (8 * (j % 4))) * scale));
  store_values(x + row * ldx + c, n, out);
}

template <int T, int GT>
hipError_t norm_as(const NormForward& a, hipStream_t s) {
  return in_launches(a.rows, kThreads, [&](int64_t first, unsigned n) {
    if (a.scales)
      k_norm<T, GT, true><<<n, kThreads, 0, s>>>(a, first);
    else
      k_norm<T, GT, false><<<n, kThreads, 0, s>>>(a, first);
    return hipGetLastError();
  });
}

template <int T, int GT>
hipError_t backward_as(const NormBackward& a, hipStream_t s) {
  if (a.dgain) {
    const int64_t slabs = norm_slabs(a.rows, a.cols);
    hipError_t e = hipSuccess;
    if (slabs)
      e = in_launches(slabs * ceil_div(a.cols, kThreads), kThreads, [&](int64_t first, unsigned n) {
        k_norm_gain<T><<<n, kThreads, 0, s>>>(a, first);
        return hipGetLastError();
      });
    if (e != hipSuccess) return e;
    e = in_launches(ceil_div(a.cols, kThreads), kThreads, [&](int64_t first, unsigned n) {
      k_norm_gain_join<GT><<<n, kThreads, 0, s>>>(a.partial, slabs, a.cols, static_cast<typename Elem<GT>::type*>(a.dgain), first);
      return hipGetLastError();
    });
    if (e != hipSuccess) return e;
  }
  if (!a.rows) return hipSuccess;
  return in_launches(a.rows, kThreads, [&](int64_t first, unsigned n) {
    k_norm_dx<T, GT><<<n, kThreads, 0, s>>>(a, first);
    return hipGetLastError();
  });
}

}  // namespace

int64_t norm_slabs(int64_t rows, int64_t cols) { return ceil_div(rows, kNormSlabRows); }

#define EMBD_NORM_TYPES(F)                                                                \
  switch (type) {                                                                         \
    case EMB_TYPE_FP32:                                                                   \
      return F<EMB_TYPE_FP32, EMB_TYPE_FP32>(a, s);                                       \
    case EMB_TYPE_BF16:                                                                   \
      return gain_wide ? F<EMB_TYPE_BF16, EMB_TYPE_FP32>(a, s) : F<EMB_TYPE_BF16, EMB_TYPE_BF16>(a, s); \
    default:                                                                              \
      return gain_wide ? F<EMB_TYPE_FP16, EMB_TYPE_FP32>(a, s) : F<EMB_TYPE_FP16, EMB_TYPE_FP16>(a, s); \
  }

hipError_t launch_norm(const NormForward& a, int type, bool gain_wide, hipStream_t s) { EMBD_NORM_TYPES(norm_as) }
hipError_t launch_norm_backward(const NormBackward& a, int type, bool gain_wide, hipStream_t s) { EMBD_NORM_TYPES(backward_as) }
#undef EMBD_NORM_TYPES

hipError_t launch_rows8_dequantize(const int8_t* codes, int64_t rows, int64_t cols, int64_t ldc, const float* scales, void* x,
                                   int type, int64_t ldx, hipStream_t s) {
  return in_launches(ceil_div(rows * ceil_div(cols, kPer), kThreads), kThreads, [&](int64_t first, unsigned n) {
#define EMBD_OUT(T)                                                                                                       \
  k_rows8_dequantize<T><<<n, kThreads, 0, s>>>(codes, rows, cols, ldc, scales, static_cast<typename Elem<T>::type*>(x), ldx, first)
    if (type == EMB_TYPE_FP32)
      EMBD_OUT(EMB_TYPE_FP32);
    else if (type == EMB_TYPE_BF16)
      EMBD_OUT(EMB_TYPE_BF16);
    else
      EMBD_OUT(EMB_TYPE_FP16);
#undef EMBD_OUT
    return hipGetLastError();
  });
}

}  // namespace embd
