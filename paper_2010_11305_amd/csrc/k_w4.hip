// Matrices in 4-bit integer codes with a scale and a bias per group ("W4"): quantisation, expansion, and the plain form.
//
// A wave takes a tile of 16 rows x 128 columns; lane 16 b + r holds columns 32 i + 8 b + (0 .. 7) of row r for i = 0 .. 3,
// so a group of 32 columns is four lanes' values of one i, one of 64 or 128 of two or four.
//
// 8192 x 12800, groups of 128 (BF16 210 MB, the matrix 55.7 MB): quantisation 78 us (3.4 TB/s; an IEEE division a value, as the
// tables' rows have it), expansion 45 us (5.9 TB/s), plain form to tiles and back 36 and 37 us, 3 TB/s.
#include "dense_device.h"

namespace embd {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

__device__ __forceinline__ float f16_value(uint32_t bits) { return __half2float(__ushort_as_half((uint16_t)bits)); }

// The tile of a wave, and the lane's place in it.
struct Place {
  int64_t rt, kt, row;
  int b, r, lane;
  bool inside;
};
__device__ __forceinline__ Place place_of(const W4& q, int64_t first) {
  Place p;
  p.lane = threadIdx.x % 64;
  p.b = p.lane / 16, p.r = p.lane % 16;
  const int64_t tile = (first + blockIdx.x) * kWaves + threadIdx.x / 64;
  p.rt = tile / q.col_tiles, p.kt = tile % q.col_tiles;
  p.inside = p.rt < q.row_tiles;
  p.row = p.rt * kTileRows + p.r;
  return p;
}

// Columns of the matrix among the 8 of dword i of a lane.
__device__ __forceinline__ int columns(const W4& q, const Place& p, int i, int64_t* c) {
  *c = p.kt * kTileCols + 32 * i + 8 * p.b;
  const int64_t left = q.cols - *c;
  return p.row >= q.rows || left <= 0 ? 0 : left < 8 ? (int)left : 8;
}

// Codes (0 .. 15 each) of 8 columns to a dword of a tile, and back.
__device__ __forceinline__ int shift_of(int j) { return j < 4 ? 8 * j : 8 * (j - 4) + 4; }

// 8 plain codes, column j in nibble j, to a dword of a tile, and back: columns 0 .. 3 in the even nibbles, 4 .. 7 in the odd.
__device__ __forceinline__ uint32_t spread(uint32_t x) {
  x = (x | x << 8) & 0x00FF00FFu;
  return (x | x << 4) & 0x0F0F0F0Fu;
}
__device__ __forceinline__ uint32_t tiled(uint32_t plain) { return spread(plain & 0xFFFFu) | spread(plain >> 16) << 4; }
__device__ __forceinline__ uint32_t gathered(uint32_t x) {
  x &= 0x0F0F0F0Fu;
  x = (x | x >> 4) & 0x00FF00FFu;
  return (x | x >> 8) & 0xFFFFu;
}
__device__ __forceinline__ uint32_t plain(uint32_t tile) { return gathered(tile) | gathered(tile >> 4) << 16; }

// Four bytes at any address.
struct __attribute__((packed, aligned(1))) Bytes4 {
  uint32_t w;
};

template <int TYPE, int G>
__global__ __launch_bounds__(kThreads) void k_w4_quantize(const typename Elem<TYPE>::type* __restrict__ x, int64_t ld, W4 q,
                                                          uint8_t* __restrict__ out, int64_t first) {
  constexpr int kSame = G / 32;   // dwords of a lane in one group
  const Place p = place_of(q, first);
  if (!p.inside) return;
  Raw<TYPE, 8> v[4];
  int n[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    int64_t c;
    n[i] = columns(q, p, i, &c);
    load_values(n[i] ? x + p.row * ld + c : x, n[i], v[i]);
  }
  uint32_t word[4];
#pragma unroll
  for (int g = 0; g < 4 / kSame; ++g) {
    float lo = __uint_as_float(0x7F800000u), hi = -lo;
    uint32_t top = 0;
    int any = 0;
#pragma unroll
    for (int i = g * kSame; i < (g + 1) * kSame; ++i) {
      any |= n[i];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (j >= n[i]) continue;
        const float w = v[i].get(j);
        lo = fminf(lo, w), hi = fmaxf(hi, w);
        top = max(top, __float_as_uint(w) & 0x7FFFFFFFu);
      }
    }
#pragma unroll
    for (int m = 16; m < 64; m *= 2) {
      lo = fminf(lo, __shfl_xor(lo, m)), hi = fmaxf(hi, __shfl_xor(hi, m));
      top = max(top, (uint32_t)__shfl_xor((int)top, m));
      any |= __shfl_xor(any, m);
    }
    uint32_t sb = 0, bb = 0;
    const bool fine = top < __float_as_uint(65520.0f);
    float s = 0.0f, b = 0.0f;
    if (any) {
      sb = fine ? f16_bits((hi - lo) / 15.0f) : 0x7E00u;
      bb = fine ? f16_bits(lo + 0.0f) : 0x7E00u;   // -0 as +0
      s = f16_value(sb), b = f16_value(bb);
    }
#pragma unroll
    for (int i = g * kSame; i < (g + 1) * kSame; ++i) {
      word[i] = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (j >= n[i] || !fine || s == 0.0f) continue;
        const float c = fminf(fmaxf(rintf((v[i].get(j) - b) / s), 0.0f), 15.0f);
        word[i] |= (uint32_t)c << shift_of(j);
      }
    }
    if (p.b == 0) {
      uint32_t* pair = reinterpret_cast<uint32_t*>(out + q.pairs(p.rt, p.kt * (kTileCols / G) + g)) + p.r;
      *pair = sb | bb << 16;
    }
  }
  reinterpret_cast<uint4*>(out + q.tile(p.rt, p.kt))[p.lane] = make_uint4(word[0], word[1], word[2], word[3]);
}

template <int TYPE>
__global__ __launch_bounds__(kThreads) void k_w4_dequantize(W4 q, typename Elem<TYPE>::type* __restrict__ x, int64_t ld,
                                                            int64_t first) {
  const Place p = place_of(q, first);
  if (!p.inside) return;
  const uint4 w4 = reinterpret_cast<const uint4*>(q.base + q.tile(p.rt, p.kt))[p.lane];
  const uint32_t word[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    int64_t c;
    const int n = columns(q, p, i, &c);
    if (!n) continue;
    const uint32_t pair = reinterpret_cast<const uint32_t*>(q.base + q.pairs(p.rt, p.kt * (kTileCols / q.group) + 32 * i / q.group))[p.r];
    const float s = f16_value(pair & 0xFFFFu), b = f16_value(pair >> 16);
    Raw<TYPE, 8> v = {};
#pragma unroll
    for (int j = 0; j < 8; ++j) v.put(j, to_bits<TYPE>(b + s * (float)(word[i] >> shift_of(j) & 15u)));
    store_values(x + p.row * ld + c, n, v);
  }
}

// Plain codes to tiles: a dword of a tile is four bytes of a row.
__global__ __launch_bounds__(kThreads) void k_w4_pack(const uint8_t* __restrict__ codes, const uint16_t* __restrict__ scales,
                                                      const uint16_t* __restrict__ biases, W4 q, uint8_t* __restrict__ out,
                                                      int64_t first) {
  const Place p = place_of(q, first);
  if (!p.inside) return;
  const int64_t pitch = (q.cols + 1) / 2, groups = ceil_div(q.cols, q.group);
  uint32_t word[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    int64_t c;
    const int n = columns(q, p, i, &c);
    const uint8_t* from = codes + p.row * pitch + c / 2;
    word[i] = 0;
    if (n == 8) {
      word[i] = tiled(reinterpret_cast<const Bytes4*>(from)->w);
    } else {
      for (int j = 0; j < n; ++j) word[i] |= (uint32_t)(from[j / 2] >> (4 * (j % 2)) & 15) << shift_of(j);
    }
  }
  reinterpret_cast<uint4*>(out + q.tile(p.rt, p.kt))[p.lane] = make_uint4(word[0], word[1], word[2], word[3]);
  const int per = kTileCols / q.group;
  if (p.b < per) {
    const int64_t g = p.kt * per + p.b;
    const bool there = p.row < q.rows && g < groups;
    reinterpret_cast<uint32_t*>(out + q.pairs(p.rt, g))[p.r] =
        there ? (uint32_t)scales[p.row * groups + g] | (uint32_t)biases[p.row * groups + g] << 16 : 0u;
  }
}

__global__ __launch_bounds__(kThreads) void k_w4_unpack(W4 q, uint8_t* __restrict__ codes, uint16_t* __restrict__ scales,
                                                        uint16_t* __restrict__ biases, int64_t first) {
  const Place p = place_of(q, first);
  if (!p.inside || p.row >= q.rows) return;
  const int64_t pitch = (q.cols + 1) / 2, groups = ceil_div(q.cols, q.group);
  const uint4 w4 = reinterpret_cast<const uint4*>(q.base + q.tile(p.rt, p.kt))[p.lane];
  const uint32_t word[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    int64_t c;
    const int n = columns(q, p, i, &c);
    uint8_t* to = codes + p.row * pitch + c / 2;
    if (n == 8) {
      reinterpret_cast<Bytes4*>(to)->w = plain(word[i]);
    } else {
      for (int j = 0; j < n; j += 2)
        to[j / 2] = (uint8_t)((word[i] >> shift_of(j) & 15u) | (j + 1 < n ? (word[i] >> shift_of(j + 1) & 15u) << 4 : 0u));
    }
  }
  const int per = kTileCols / q.group;
  const int64_t g = p.kt * per + p.b;
  if (p.b < per && g < groups) {
    const uint32_t pair = reinterpret_cast<const uint32_t*>(q.base + q.pairs(p.rt, g))[p.r];
    scales[p.row * groups + g] = (uint16_t)pair;
    biases[p.row * groups + g] = (uint16_t)(pair >> 16);
  }
}

int64_t workgroups(const W4& q) { return ceil_div(q.row_tiles * q.col_tiles, kWaves); }

template <int T>
hipError_t quantize_as(const void* x, int64_t ld, const W4& q, hipStream_t s) {
  const auto* p = static_cast<const typename Elem<T>::type*>(x);
  uint8_t* out = const_cast<uint8_t*>(q.base);
  return in_launches(workgroups(q), kThreads, [&](int64_t first, unsigned n) {
    if (q.group == 32)
      k_w4_quantize<T, 32><<<n, kThreads, 0, s>>>(p, ld, q, out, first);
    else if (q.group == 64)
      k_w4_quantize<T, 64><<<n, kThreads, 0, s>>>(p, ld, q, out, first);
    else
      k_w4_quantize<T, 128><<<n, kThreads, 0, s>>>(p, ld, q, out, first);
    return hipGetLastError();
  });
}

template <int T>
hipError_t dequantize_as(const W4& q, void* x, int64_t ld, hipStream_t s) {
  return in_launches(workgroups(q), kThreads, [&](int64_t first, unsigned n) {
    k_w4_dequantize<T><<<n, kThreads, 0, s>>>(q, static_cast<typename Elem<T>::type*>(x), ld, first);
    return hipGetLastError();
  });
}

}  // namespace

hipError_t launch_w4_quantize(const void* x, int type, int64_t ld, const W4& q, hipStream_t s) {
  if (type == EMB_TYPE_FP32) return quantize_as<EMB_TYPE_FP32>(x, ld, q, s);
  if (type == EMB_TYPE_BF16) return quantize_as<EMB_TYPE_BF16>(x, ld, q, s);
  return quantize_as<EMB_TYPE_FP16>(x, ld, q, s);
}

hipError_t launch_w4_dequantize(const W4& q, void* x, int type, int64_t ld, hipStream_t s) {
  if (type == EMB_TYPE_FP32) return dequantize_as<EMB_TYPE_FP32>(q, x, ld, s);
  if (type == EMB_TYPE_BF16) return dequantize_as<EMB_TYPE_BF16>(q, x, ld, s);
  return dequantize_as<EMB_TYPE_FP16>(q, x, ld, s);
}

hipError_t launch_w4_pack(const uint8_t* codes, const uint16_t* scales, const uint16_t* biases, const W4& q, hipStream_t s) {
  return in_launches(workgroups(q), kThreads, [&](int64_t first, unsigned n) {
    k_w4_pack<<<n, kThreads, 0, s>>>(codes, scales, biases, q, const_cast<uint8_t*>(q.base), first);
    return hipGetLastError();
  });
}

hipError_t launch_w4_unpack(const W4& q, uint8_t* codes, uint16_t* scales, uint16_t* biases, hipStream_t s) {
  return in_launches(workgroups(q), kThreads, [&](int64_t first, unsigned n) {
    k_w4_unpack<<<n, kThreads, 0, s>>>(q, codes, scales, biases, first);
    return hipGetLastError();
  });
}

}  // namespace embd
