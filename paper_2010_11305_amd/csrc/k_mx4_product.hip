// Products of MX4 matrices on the scaled matrix instruction v_mfma_scale_f32_16x16x128_f8f6f4.
#include "dense_device.h"

namespace embd {

namespace {

using v8i = int __attribute__((ext_vector_type(8)));
using f32x4 = float __attribute__((ext_vector_type(4)));

__device__ __forceinline__ v8i operand(const uint4& q) {
  v8i r = {(int)q.x, (int)q.y, (int)q.z, (int)q.w, 0, 0, 0, 0};
  return r;
}

// D += A B for one 16x16 tile over 128 columns.  The rows of C are the columns of D (the
// weight is the first operand), so that a lane holds four consecutive columns of a row of C.
__device__ __forceinline__ f32x4 mma(const v8i& b, const v8i& a, f32x4 c, uint32_t sb, uint32_t sa) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, c, 4, 4, 0, (int)sb, 0, (int)sa);
}

// Columns [col, col + 4) of one row of C.
template <int TYPE>
__device__ __forceinline__ void store4(typename Elem<TYPE>::type* row, int64_t col, int64_t n, const f32x4& v) {
  if (col + 4 <= n) {
    if constexpr (TYPE == EMB_TYPE_FP32) {
      Bytes16 b;
#pragma unroll
      for (int i = 0; i < 4; ++i) b.w[i] = __float_as_uint(v[i]);
      *reinterpret_cast<Bytes16*>(row + col) = b;
    } else {
      Bytes8 b;
#pragma unroll
      for (int i = 0; i < 2; ++i) b.w[i] = to_bits<TYPE>(v[2 * i]) | to_bits<TYPE>(v[2 * i + 1]) << 16;
      *reinterpret_cast<Bytes8*>(row + col) = b;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (col + i >= n) continue;
      if constexpr (TYPE == EMB_TYPE_FP32)
        row[col + i] = v[i];
      else
        row[col + i] = (uint16_t)to_bits<TYPE>(v[i]);
    }
  }
}

// A wave computes 32 x 32 of C, its operands straight from memory.
template <int TYPE>
__global__ __launch_bounds__(256) void k_product(Mx4 a, Mx4 b, typename Elem<TYPE>::type* __restrict__ c, int64_t ldc) {
  const int64_t wide = (b.row_tiles + 3) / 4;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t mt = (int64_t)blockIdx.x / wide * 4 + (wave >> 1) * 2, nt = (int64_t)blockIdx.x % wide * 4 + (wave & 1) * 2;
  if (mt >= a.row_tiles || nt >= b.row_tiles) return;
  const int64_t ms[2] = {mt, mt + 1 < a.row_tiles ? mt + 1 : mt}, ns[2] = {nt, nt + 1 < b.row_tiles ? nt + 1 : nt};
  f32x4 acc[2][2] = {};
  for (int64_t kt = 0; kt < a.col_tiles; ++kt) {
    v8i fa[2], fb[2];
    uint32_t sa[2], sb[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      fa[i] = operand(*reinterpret_cast<const uint4*>(a.base + a.tile(ms[i], kt) + 16 * lane));
      fb[i] = operand(*reinterpret_cast<const uint4*>(b.base + b.tile(ns[i], kt) + 16 * lane));
      sa[i] = a.base[a.scale(ms[i], kt, lane)];
      sb[i] = b.base[b.scale(ns[i], kt, lane)];
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) acc[i][j] = mma(fb[j], fa[i], acc[i][j], sb[j], sa[i]);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int64_t row = (mt + i) * kTileRows + (lane & 15), col = (nt + j) * kTileRows + (lane >> 4) * 4;
      if (row < a.rows && col < b.rows) store4<TYPE>(c + row * ldc, col, b.rows, acc[i][j]);
    }
}

// C = 0 (a product over no columns).
template <int TYPE>
__global__ __launch_bounds__(256) void k_zero(int64_t m, int64_t n, typename Elem<TYPE>::type* __restrict__ c, int64_t ldc) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < m * n; i += (int64_t)gridDim.x * 256) c[i / n * ldc + i % n] = 0;
}

template <int TYPE>
hipError_t matmul_as(const void* a, const void* b, int64_t m, int64_t n, int64_t k, void* cv, int64_t ldc,
                     hipStream_t s) {
  auto* c = static_cast<typename Elem<TYPE>::type*>(cv);
  if (!k) {
    const int64_t blocks = (m * n + 255) / 256;
    k_zero<TYPE><<<(unsigned)(blocks < 65536 ? blocks : 65536), 256, 0, s>>>(m, n, c, ldc);
    return hipGetLastError();
  }
  const Mx4 qa(a, m, k), qb(b, n, k);
  const int64_t grid = ((qa.row_tiles + 3) / 4) * ((qb.row_tiles + 3) / 4);
  k_product<TYPE><<<(unsigned)grid, 256, 0, s>>>(qa, qb, c, ldc);
  return hipGetLastError();
}

}  // namespace

size_t matmul_workspace(int64_t, int64_t, int64_t) { return 0; }

hipError_t launch_matmul(const void* a, const void* b, int64_t m, int64_t n, int64_t k, void* c, int type, int64_t ldc,
                         void* workspace, hipStream_t s) {
  if (type == EMB_TYPE_FP32) return matmul_as<EMB_TYPE_FP32>(a, b, m, n, k, c, ldc, s);
  if (type == EMB_TYPE_BF16) return matmul_as<EMB_TYPE_BF16>(a, b, m, n, k, c, ldc, s);
  return matmul_as<EMB_TYPE_FP16>(a, b, m, n, k, c, ldc, s);
}

size_t linear_workspace(int64_t m, int64_t n, int64_t k) {
  return ((size_t)Mx4(nullptr, m, k).bytes() + 255) / 256 * 256 + matmul_workspace(m, n, k);
}

hipError_t launch_linear(const void* x, int type, int64_t m, int64_t k, int64_t ldx, const void* w, int64_t n, void* y,
                         int64_t ldy, void* workspace, hipStream_t s) {
  if (k) {
    const hipError_t e = launch_quantize(x, type, m, k, ldx, workspace, nullptr, EMB_ROUND_NEAREST, 0, 0, s);
    if (e != hipSuccess) return e;
  }
  const size_t q = k ? ((size_t)Mx4(nullptr, m, k).bytes() + 255) / 256 * 256 : 0;
  return launch_matmul(workspace, w, m, n, k, y, type, ldy, static_cast<uint8_t*>(workspace) + q, s);
}

}  // namespace embd
