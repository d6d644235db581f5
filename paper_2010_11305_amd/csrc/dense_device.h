// Device helpers of the dense operators: element types, Philox uniforms, and the quantisation
// of one MX4 block held by one lane.
#pragma once

#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "dense_internal.h"
#include "embc_device.h"

namespace embd {

using bf16x2 = __bf16 __attribute__((ext_vector_type(2)));
using f16x2 = _Float16 __attribute__((ext_vector_type(2)));
using f32x2 = float __attribute__((ext_vector_type(2)));

// 16 bytes at any alignment of the element type (the memory system takes unaligned vector
// accesses; only the type's own alignment is promised by callers).
struct __attribute__((packed, aligned(2))) Bytes16 {
  uint32_t w[4];
};
struct __attribute__((packed, aligned(2))) Bytes8 {
  uint32_t w[2];
};

template <int TYPE>
struct Elem;
template <>
struct Elem<EMB_TYPE_FP32> {
  static constexpr int kBytes = 4;
  using type = float;
};
template <>
struct Elem<EMB_TYPE_BF16> {
  static constexpr int kBytes = 2;
  using type = uint16_t;
};
template <>
struct Elem<EMB_TYPE_FP16> {
  static constexpr int kBytes = 2;
  using type = uint16_t;
};

// N consecutive values as they lie in memory, N even: dwords of one FP32 value or of two 16-bit ones.
template <int TYPE, int N>
struct Raw {
  static constexpr int kPer = 4 / Elem<TYPE>::kBytes;  // values per dword
  static constexpr int kWords = N / kPer;
  uint32_t w[kWords];

  __device__ __forceinline__ float get(int j) const {
    if constexpr (TYPE == EMB_TYPE_FP32) return __uint_as_float(w[j]);
    const uint32_t h = j % 2 ? w[j / 2] >> 16 : w[j / 2] & 0xFFFFu;
    if constexpr (TYPE == EMB_TYPE_BF16) return __uint_as_float(h << 16);
    return __half2float(__ushort_as_half((uint16_t)h));
  }
  // element j from its bits
  __device__ __forceinline__ void put(int j, uint32_t v) {
    if constexpr (kPer == 1)
      w[j] = v;
    else if (j % 2)
      w[j / 2] = (w[j / 2] & 0xFFFFu) | v << 16;
    else
      w[j / 2] = (w[j / 2] & 0xFFFF0000u) | v;
  }
};

template <int TYPE>
__device__ __forceinline__ uint32_t load_bits(const typename Elem<TYPE>::type* p) {
  if constexpr (TYPE == EMB_TYPE_FP32) return __float_as_uint(*p);
  return *p;
}

// Values [0, n) of p, n <= N; zeros beyond.  Whole 16-byte pieces are loaded at once.
template <int TYPE, int N>
__device__ __forceinline__ void load_values(const typename Elem<TYPE>::type* p, int n, Raw<TYPE, N>& r) {
  constexpr int kPiece = 16 / Elem<TYPE>::kBytes;
#pragma unroll
  for (int q = 0; q < N / kPiece; ++q) {
    if ((q + 1) * kPiece <= n) {
      const Bytes16 b = *reinterpret_cast<const Bytes16*>(p + q * kPiece);
#pragma unroll
      for (int i = 0; i < 4; ++i) r.w[4 * q + i] = b.w[i];
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) r.w[4 * q + i] = 0;
#pragma unroll
      for (int j = 0; j < kPiece; ++j)
        if (q * kPiece + j < n) r.put(q * kPiece + j, load_bits<TYPE>(p + q * kPiece + j));
    }
  }
}

// FP32 to 16-bit types, nearest even (NaN stays NaN).
__device__ __forceinline__ uint32_t bf16_bits(float x) {
  const __bf16 b = (__bf16)x;
  return __builtin_bit_cast(uint16_t, b);
}
__device__ __forceinline__ uint32_t f16_bits(float x) {
  return __half_as_ushort(__float2half(embc::as_f32_value(x)));
}
template <int TYPE>
__device__ __forceinline__ uint32_t to_bits(float x) {
  if constexpr (TYPE == EMB_TYPE_FP32) return __float_as_uint(x);
  if constexpr (TYPE == EMB_TYPE_BF16) return bf16_bits(x);
  return f16_bits(x);
}

// The first n values of r to p, n <= N, whole 16-byte pieces at once.
template <int TYPE, int N>
__device__ __forceinline__ void store_values(typename Elem<TYPE>::type* p, int n, const Raw<TYPE, N>& r) {
  constexpr int kPiece = 16 / Elem<TYPE>::kBytes;
#pragma unroll
  for (int q = 0; q < N / kPiece; ++q) {
    if ((q + 1) * kPiece <= n) {
      *reinterpret_cast<Bytes16*>(p + q * kPiece) = Bytes16{{r.w[4 * q], r.w[4 * q + 1], r.w[4 * q + 2], r.w[4 * q + 3]}};
    } else {
#pragma unroll
      for (int j = 0; j < kPiece; ++j) {
        const int e = q * kPiece + j;
        if (e >= n) continue;
        if constexpr (TYPE == EMB_TYPE_FP32)
          p[e] = __uint_as_float(r.w[e]);
        else
          p[e] = (uint16_t)(e % 2 ? r.w[e / 2] >> 16 : r.w[e / 2]);
      }
    }
  }
}

// 2^(byte - 127), byte 0 .. 254 (the lowest is a subnormal number)
__device__ __forceinline__ float power_of(uint32_t byte) {
  return __uint_as_float(byte ? byte << 23 : 0x00400000u);
}

// |x| bits of the largest magnitude among the values of a lane; NaN and infinity have exponent 255.
template <int TYPE, int N>
__device__ __forceinline__ uint32_t max_magnitude(const Raw<TYPE, N>& r) {
  if constexpr (TYPE == EMB_TYPE_FP32) {
    uint32_t a = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) a = max(a, r.w[j] & 0x7FFFFFFFu);
    return a;
  } else {
    using u16x2 = uint16_t __attribute__((ext_vector_type(2)));
    u16x2 a = {0, 0};
#pragma unroll
    for (int i = 0; i < N / 2; ++i)
      a = __builtin_elementwise_max(a, __builtin_bit_cast(u16x2, r.w[i] & 0x7FFF7FFFu));
    const uint16_t m = a.x > a.y ? a.x : a.y;
    if constexpr (TYPE == EMB_TYPE_BF16) return (uint32_t)m << 16;
    return __float_as_uint(__half2float(__ushort_as_half(m)));
  }
}

// The scale byte of a block whose largest magnitude has these FP32 bits.
__device__ __forceinline__ uint32_t mx4_scale(uint32_t amax) {
  const uint32_t e = amax >> 23;
  return e == 255 ? 255u : e > 2 ? e - 2 : 0u;
}

// embc::philox4x32_10 with the three-way exclusive or as one instruction.
__device__ __forceinline__ uint4 philox(uint4 c, uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t p0 = (uint64_t)0xD2511F53u * c.x, p1 = (uint64_t)0xCD9E8D57u * c.z;
    c = make_uint4(__builtin_amdgcn_bitop3_b32((uint32_t)(p1 >> 32), c.y, k0, 0x96), (uint32_t)p1,
                   __builtin_amdgcn_bitop3_b32((uint32_t)(p0 >> 32), c.w, k1, 0x96), (uint32_t)p0);
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return c;
}

// Where a block lies in the random stream: key, and the counter of its first 8 values.
struct Mx4Random {
  uint32_t k0, k1, step, tag;
};

// The 8 values at p of a block: their codes in one dword.
template <int TYPE, int N>
__device__ __forceinline__ uint32_t codes8_nearest(const Raw<TYPE, N>& r, int j0, float scale) {
  uint32_t c = 0;
#define EMBD_PAIR(SEL)                                                                                              \
  if constexpr (TYPE == EMB_TYPE_FP32)                                                                              \
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, r.get(j0 + 2 * SEL), r.get(j0 + 2 * SEL + 1), scale, SEL);      \
  else if constexpr (TYPE == EMB_TYPE_BF16)                                                                         \
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, r.w[j0 / 2 + SEL]), scale, SEL);    \
  else                                                                                                              \
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(f16x2, r.w[j0 / 2 + SEL]), scale, SEL);
  EMBD_PAIR(0)
  EMBD_PAIR(1)
  EMBD_PAIR(2)
  EMBD_PAIR(3)
#undef EMBD_PAIR
  return c;
}

// Stochastic codes of 8 values.  The conversion adds the top 22 bits r of its random word to the fraction of
// |x| / 2^s between two neighbours, cut to 22 bits, and takes the upper one on a carry (for the low value of
// its pair; the high one, here 0, would see other bits).  With r = 2^22 - 1 - 64 u that is a fraction above
// u / 2^16, exactly, if the fraction has no bits beyond 22: |x| / 2^s, a multiple of 2^-23 where it is
// 1 or more, is made one below 1 by rounding it up, which moves no fraction across a multiple of 2^-16.
// 6 operations a value where the comparison written out takes 18.
template <int TYPE, int N>
__device__ __forceinline__ uint32_t codes8_stochastic(const Raw<TYPE, N>& r, int j0, uint32_t scale, uint32_t col8,
                                                      uint32_t row, const Mx4Random& q) {
  const uint4 w = philox(make_uint4(col8, row, q.step, q.tag), q.k0, q.k1);
  const uint32_t rest[4] = {~w.x, ~w.y, ~w.z, ~w.w};   // 2^16 - 1 - u, two a word
  const int up = 150 - (int)scale;
  uint32_t c[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float x = r.get(j0 + j);
    const f32x2 y = {copysignf(ceilf(ldexpf(fabsf(x), up)), x), 0.0f};
    // each into a register of its own: this builtin does not keep the other bytes of the first argument
    c[j] = __builtin_amdgcn_cvt_scalef32_sr_pk_fp4_f32(0, y, j % 2 ? rest[j / 2] | 0xFFFFu : rest[j / 2] << 16 | 0xFFFFu,
                                                       0x1p23f, 0);
  }
  // the low bytes of c[0], c[2], c[4], c[6]; with those of the odd ones shifted between their halves
  const uint32_t even = __builtin_amdgcn_perm(c[2], c[0], 0x0C0C0400u) | __builtin_amdgcn_perm(c[6], c[4], 0x0C0C0400u) << 16;
  const uint32_t odd = __builtin_amdgcn_perm(c[3], c[1], 0x0C0C0400u) | __builtin_amdgcn_perm(c[7], c[5], 0x0C0C0400u) << 16;
  return even | odd << 4;
}

// One block held by a lane: 32 values to 16 bytes of codes and the scale byte.
template <int TYPE, bool STOCHASTIC>
__device__ __forceinline__ uint4 quantize_block(const Raw<TYPE, kBlock>& r, uint32_t col8, uint32_t row,
                                                const Mx4Random& q, uint32_t* scale) {
  const uint32_t s = mx4_scale(max_magnitude(r));
  *scale = s;
  if (s == 255u) return make_uint4(0, 0, 0, 0);
  uint32_t c[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (STOCHASTIC)
      c[i] = codes8_stochastic(r, 8 * i, s, col8 + i, row, q);
    else
      c[i] = codes8_nearest(r, 8 * i, power_of(s));
  }
  return make_uint4(c[0], c[1], c[2], c[3]);
}

}  // namespace embd
