// Products of few rows with a W4 weight, y = x w^T, on the 16x16 matrix instructions.
//
// w = bias + scale q over a group, so y is the sum over the groups of scale * sum(q x) + bias * sum(x).  The codes become the
// instruction's first operand as they are, small whole numbers that every type here holds exactly; the sums of x come from
// the same instruction with ones in their place, in the registers where the sums of products lie.  FP32 rows go
// in as three BF16 parts that add up to them exactly.
#include "dense_device.h"

namespace embd {

namespace {

using bf16x8 = __bf16 __attribute__((ext_vector_type(8)));
using f16x8 = _Float16 __attribute__((ext_vector_type(8)));
using f32x4 = float __attribute__((ext_vector_type(4)));
using i32x4 = int __attribute__((ext_vector_type(4)));
using u32x4 = uint32_t __attribute__((ext_vector_type(4)));
using u32x2 = uint32_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float f16_low(uint32_t w) { return __half2float(__ushort_as_half((uint16_t)w)); }
__device__ __forceinline__ float f16_high(uint32_t w) { return __half2float(__ushort_as_half((uint16_t)(w >> 16))); }

// 8 codes of a dword as bytes, columns in order.
__device__ __forceinline__ u32x2 code_bytes(uint32_t w) { return u32x2{w & 0x0F0F0F0Fu, w >> 4 & 0x0F0F0F0Fu}; }

// The same as 16-bit floating point: a byte q below 16 is q 2^-9 as an E4M3 element, subnormal or not.
template <int T>
__device__ __forceinline__ u32x4 code_values(uint32_t w) {
  const u32x2 b = code_bytes(w);
  u32x4 v;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if constexpr (T == EMB_TYPE_FP16) {
      v[2 * h] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b[h], 512.0f, false));
      v[2 * h + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b[h], 512.0f, true));
    } else {
      v[2 * h] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b[h], 512.0f, false));
      v[2 * h + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b[h], 512.0f, true));
    }
  }
  return v;
}

template <int T>
__device__ __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (T == EMB_TYPE_FP16)
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// The operand of 32 columns of 16 rows: PARTS registers sets of 8 values a lane.
template <int T>
struct Operand {
  static constexpr int kParts = T == EMB_TYPE_FP32 ? 3 : 1;
  static constexpr uint32_t kOnes = T == EMB_TYPE_FP16 ? 0x3C003C00u : 0x3F803F80u;
  using Acc = f32x4;
  u32x4 part[kParts];

  __device__ __forceinline__ void load(const void* x, int64_t at, int n) {
    Raw<T, 8> r;
    load_values(static_cast<const typename Elem<T>::type*>(x) + at, n, r);
    if constexpr (T == EMB_TYPE_FP32) {
#pragma unroll
      for (int p = 0; p < 3; ++p) {
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
          const uint32_t lo = r.w[j] & 0xFFFF0000u, hi = r.w[j + 1] & 0xFFFF0000u;
          part[p][j / 2] = lo >> 16 | hi;
          r.w[j] = __float_as_uint(__uint_as_float(r.w[j]) - __uint_as_float(lo));
          r.w[j + 1] = __float_as_uint(__uint_as_float(r.w[j + 1]) - __uint_as_float(hi));
        }
      }
    } else {
      part[0] = u32x4{r.w[0], r.w[1], r.w[2], r.w[3]};
    }
  }
  __device__ __forceinline__ void sums(uint32_t w, Acc& codes, Acc& ones) const {
    const u32x4 a = code_values<T>(w), one = {kOnes, kOnes, kOnes, kOnes};
#pragma unroll
    for (int p = kParts - 1; p >= 0; --p) {
      codes = mma<T>(a, part[p], codes);
      ones = mma<T>(one, part[p], ones);
    }
  }
};

template <>
struct Operand<EMB_TYPE_INT8> {
  using Acc = i32x4;
  u32x2 part;

  __device__ __forceinline__ void load(const void* x, int64_t at, int n) {
    const uint8_t* p = static_cast<const uint8_t*>(x) + at;
    part = u32x2{0, 0};
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < n) part[j / 4] |= (uint32_t)p[j] << (8 * (j % 4));
  }
  __device__ __forceinline__ void sums(uint32_t w, Acc& codes, Acc& ones) const {
    const long b = __builtin_bit_cast(long, part);
    codes = __builtin_amdgcn_mfma_i32_16x16x32_i8(__builtin_bit_cast(long, code_bytes(w)), b, codes, 0, 0, 0);
    ones = __builtin_amdgcn_mfma_i32_16x16x32_i8(0x0101010101010101l, b, ones, 0, 0, 0);
  }
};

template <int T>
__device__ __forceinline__ void store_one(void* y, int64_t at, float v) {
  if constexpr (T == EMB_TYPE_FP32)
    static_cast<float*>(y)[at] = v;
  else
    static_cast<uint16_t*>(y)[at] = (uint16_t)to_bits<T>(v);
}

constexpr int kWaves = 4;

// A workgroup computes 16 outputs of 16 rows, its waves sharing the columns.
template <int T, int G>
__global__ __launch_bounds__(64 * kWaves) void k_w4_linear(W4Linear a, W4 w, int64_t first) {
  __shared__ f32x4 meet[kWaves][64];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, b = lane / 16;
  const int64_t block = first + blockIdx.x, rt = block % w.row_tiles, row = block / w.row_tiles * 16 + lane % 16;
  constexpr int kSame = G / 32, kPer = kTileCols / G;
  f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int64_t kt = wave; kt < w.col_tiles; kt += kWaves) {
    const u32x4 codes = reinterpret_cast<const u32x4*>(w.base + w.tile(rt, kt))[lane];
#pragma unroll
    for (int g = 0; g < kPer; ++g) {
      typename Operand<T>::Acc c = {}, o = {};
#pragma unroll
      for (int i = g * kSame; i < (g + 1) * kSame; ++i) {
        const int64_t col = kt * kTileCols + 32 * i + 8 * b;
        const int64_t left = row < a.m ? w.cols - col : 0;
        const int n = left >= 8 ? 8 : left > 0 ? (int)left : 0;
        Operand<T> x;
        x.load(a.x, n ? row * a.ldx + col : 0, n);
        x.sums(codes[i], c, o);
      }
      const u32x4 pairs = reinterpret_cast<const u32x4*>(w.base + w.pairs(rt, kt * kPer + g))[b];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        sum[r] = fmaf(f16_low(pairs[r]), (float)c[r], sum[r]);
        sum[r] = fmaf(f16_high(pairs[r]), (float)o[r], sum[r]);
      }
    }
  }
  meet[wave][lane] = sum;
  __syncthreads();
  if (wave || row >= a.m) return;
#pragma unroll
  for (int v = 1; v < kWaves; ++v) sum += meet[v][lane];
  const float scale = a.scales ? a.scales[row] : 1.0f;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int64_t n = rt * 16 + 4 * b + r;
    if (n >= w.rows) continue;
    float v = sum[r] * scale;
    if (a.bias) v += a.bias[n];
    if (a.relu && v < 0.0f) v = 0.0f;
    const int64_t at = row * a.ldy + n;
    if (a.y_type == EMB_TYPE_FP32)
      store_one<EMB_TYPE_FP32>(a.y, at, v);
    else if (a.y_type == EMB_TYPE_BF16)
      store_one<EMB_TYPE_BF16>(a.y, at, v);
    else
      store_one<EMB_TYPE_FP16>(a.y, at, v);
  }
}

template <int T>
hipError_t linear_as(const W4Linear& a, const W4& w, hipStream_t s) {
  return in_launches(w.row_tiles * ceil_div(a.m, 16), 64 * kWaves, [&](int64_t first, unsigned n) {
    if (w.group == 32)
      k_w4_linear<T, 32><<<n, 64 * kWaves, 0, s>>>(a, w, first);
    else if (w.group == 64)
      k_w4_linear<T, 64><<<n, 64 * kWaves, 0, s>>>(a, w, first);
    else
      k_w4_linear<T, 128><<<n, 64 * kWaves, 0, s>>>(a, w, first);
    return hipGetLastError();
  });
}

}  // namespace

size_t w4_linear_workspace(int type, int64_t m, int64_t n, int64_t k, int group) { return 0; }

hipError_t launch_w4_linear(const W4Linear& a, int type, const W4& w, void* workspace, hipStream_t s) {
  if (type == EMB_TYPE_FP32) return linear_as<EMB_TYPE_FP32>(a, w, s);
  if (type == EMB_TYPE_BF16) return linear_as<EMB_TYPE_BF16>(a, w, s);
  if (type == EMB_TYPE_FP16) return linear_as<EMB_TYPE_FP16>(a, w, s);
  return linear_as<EMB_TYPE_INT8>(a, w, s);
}

}  // namespace embd
