// Products of few rows with a W4 weight, y = x w^T, on the 16x16 matrix instructions.
//
// w = bias + scale q over a group, so y is the sum over the groups of scale * sum(q x) + bias * sum(x).  The codes become the
// instruction's first operand as they are, small whole numbers that every type here holds exactly; the sums of x come from
// the same instruction with ones in their place, in the registers where the sums of products lie.  FP32 rows go
// in as three BF16 parts that add up to them exactly.
//
// Few rows (k_w4_few) are bound by memory and by what every launch costs.  us a call in a graph, and of the kernel by its trace: 1 row,
// 4096 x 12800, groups of 128 8.0 and 8.4 (27.9 MB, 3.5 TB/s), of which 3.3 are left without the loop over the columns; one 8-bit row
// against 8192 x 8192 8.4 and 8.5 (35.7 MB, 4.2 TB/s).  Code runs once or twice in such a call, and its way from memory counts as
// much as the data's: with the loop unrolled over 7 tiles, whose loads were all under way at once, the same took 3.0 and 4.5 us
// more.  So loops stay short, and what is rare goes value by value.
// Up to 64 rows (k_w4_more): 64 rows, 8192 x 12800, 31.7 us a call in a graph with groups of 32 and 29.1 with groups of 128 (423 and 461
// TFLOP/s); by the trace 28.3 for groups of 32, and 5.0 for k_w4_rows.  No one thing bounds it: of the 57 thousand clocks of its waves
// (24 us) the matrix pipe is busy for 34%, by the counters, vector instructions other than its own issue for 40% (groups of 128:
// 25 and 31%), with three waves a SIMD that do not cover for each other: each waits for data 37% of its time and for its turn
// at a pipe 40%.  Reads out of the L2 are 515 MB, 420 of them x; conflicts of LDS banks are 5 thousand clocks.  Without the loads of x it took 28 us (groups of 128: 21), without those of w 27 (25), without matrix
// instructions 32 (20).
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

// 16 rows x 128 columns of x as the second operand: lane 16 b + r holds columns 32 i + 8 b + (0 .. 7) of row r, in kSets sets
// of 16 bytes: one for each i = 0 .. 3 (and each part of FP32 rows), or for i = 0, 1 and i = 2, 3 of 8-bit rows.
template <int T>
struct Tile {
  static constexpr int kParts = T == EMB_TYPE_FP32 ? 3 : 1;
  static constexpr int kSets = 4 * kParts;
  static constexpr uint32_t kOne = T == EMB_TYPE_FP16 ? 0x3C003C00u : 0x3F803F80u;
  using E = typename Elem<T>::type;
  using Codes = u32x4[4];
  Raw<T, 8> v[4];

  __device__ __forceinline__ void load(const E* p) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int q = 0; q < Raw<T, 8>::kWords / 4; ++q) {
        const Bytes16 w = *reinterpret_cast<const Bytes16*>(p + 32 * i + q * (16 / Elem<T>::kBytes));
#pragma unroll
        for (int j = 0; j < 4; ++j) v[i].w[4 * q + j] = w.w[j];
      }
  }
  __device__ __forceinline__ void load_part(const E* p, int n) {   // n columns from p on are there
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int left = n - 32 * i;
      load_values(left > 0 ? p + 32 * i : p, left > 8 ? 8 : left > 0 ? left : 0, v[i]);
    }
  }
  // 8 values of columns 32 i + .. into LDS: their parts, where `to` is set 0 and each set `pitch` (of 16 bytes) behind the one
  // before, or as they are, the second half of FP32 ones 4 pitches behind the first
  template <bool RAW>
  static __device__ __forceinline__ void stage_whole(const E* p, u32x4* to, int i, int pitch) {
    Raw<T, 8> r;
#pragma unroll
    for (int q = 0; q < Raw<T, 8>::kWords / 4; ++q) {
      const Bytes16 w = *reinterpret_cast<const Bytes16*>(p + q * (16 / Elem<T>::kBytes));
#pragma unroll
      for (int j = 0; j < 4; ++j) r.w[4 * q + j] = w.w[j];
    }
    if constexpr (RAW) {
#pragma unroll
      for (int q = 0; q < Raw<T, 8>::kWords / 4; ++q) to[4 * q * pitch] = u32x4{r.w[4 * q], r.w[4 * q + 1], r.w[4 * q + 2], r.w[4 * q + 3]};
    } else {
      u32x4 s[kParts];
      split(r, s);
#pragma unroll
      for (int q = 0; q < kParts; ++q) to[(4 * q + i) * pitch] = s[q];
    }
  }
  // the first n of them, zeros for the others: value by value, as it runs once
  template <bool RAW>
  static __device__ __forceinline__ void stage_part(const E* p, int n, u32x4* to, int i, int pitch) {
#pragma unroll 1
    for (int j = 0; j < 8; ++j) {
      Raw<T, 8> r = {};
      r.w[0] = j < n ? load_bits<T>(p + j) : 0;
      if constexpr (RAW) {
        reinterpret_cast<uint32_t*>(to + j / 4 * 4 * pitch)[j % 4] = r.w[0];
      } else {
        u32x4 s[kParts];
        split(r, s);
#pragma unroll
        for (int q = 0; q < kParts; ++q) reinterpret_cast<uint16_t*>(&to[(4 * q + i) * pitch])[j] = (uint16_t)s[q][0];
      }
    }
  }
  // the operand of 8 values, its parts
  static __device__ __forceinline__ void split(const Raw<T, 8>& v, u32x4 (&s)[kParts]) {
    if constexpr (T == EMB_TYPE_FP32) {
      // cut to the 8 bits of BF16 twice; what is left has 8
      float x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = __uint_as_float(v.w[j]);
#pragma unroll
      for (int p = 0; p < 3; ++p)
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
          const uint32_t lo = __float_as_uint(x[j]), hi = __float_as_uint(x[j + 1]);
          s[p][j / 2] = __builtin_amdgcn_perm(hi, lo, 0x07060302u);
          x[j] -= __uint_as_float(lo & 0xFFFF0000u);
          x[j + 1] -= __uint_as_float(hi & 0xFFFF0000u);
        }
    } else {
      s[0] = u32x4{v.w[0], v.w[1], v.w[2], v.w[3]};
    }
  }
  __device__ __forceinline__ void operand(u32x4 (&s)[kSets]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      u32x4 p[kParts];
      split(v[i], p);
#pragma unroll
      for (int q = 0; q < kParts; ++q) s[4 * q + i] = p[q];
    }
  }
};

template <>
struct Tile<EMB_TYPE_INT8> {
  static constexpr int kSets = 2;
  using E = uint8_t;
  using Codes = u32x4[2];
  u32x2 v[4];

  __device__ __forceinline__ void load(const E* p) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const Bytes w = *reinterpret_cast<const Bytes*>(p + 32 * i);
      v[i] = u32x2{w.w[0], w.w[1]};
    }
  }
  struct __attribute__((packed, aligned(1))) Bytes {
    uint32_t w[2];
  };
  template <bool RAW>
  static __device__ __forceinline__ void stage_whole(const E* p, u32x4* to, int i, int pitch) {
    const Bytes w = *reinterpret_cast<const Bytes*>(p);
    reinterpret_cast<u32x2*>(to + i / 2 * pitch)[i % 2] = u32x2{w.w[0], w.w[1]};
  }
  template <bool RAW>
  static __device__ __forceinline__ void stage_part(const E* p, int n, u32x4* to, int i, int pitch) {
#pragma unroll 1
    for (int j = 0; j < 8; ++j) reinterpret_cast<uint8_t*>(reinterpret_cast<u32x2*>(to + i / 2 * pitch) + i % 2)[j] = j < n ? p[j] : 0;
  }
  __device__ __forceinline__ void load_part(const E* p, int n) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[i] = u32x2{0, 0};
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (32 * i + j < n) v[i][j / 4] |= (uint32_t)p[32 * i + j] << (8 * (j % 4));
    }
  }
  __device__ __forceinline__ void operand(u32x4 (&s)[kSets]) const {
#pragma unroll
    for (int i = 0; i < 2; ++i) s[i] = u32x4{v[2 * i][0], v[2 * i][1], v[2 * i + 1][0], v[2 * i + 1][1]};
  }
};

// The first operand for a lane's 16 bytes of codes.
template <int T>
__device__ __forceinline__ void codes_of(const u32x4& w, typename Tile<T>::Codes& a) {
  if constexpr (T == EMB_TYPE_INT8) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const u32x2 lo = code_bytes(w[2 * i]), hi = code_bytes(w[2 * i + 1]);
      a[i] = u32x4{lo[0], lo[1], hi[0], hi[1]};
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = code_values<T>(w[i]);
  }
}

template <int T>
__device__ __forceinline__ f32x4 mma(const u32x4& a, const u32x4& b, const f32x4& c) {
  if constexpr (T == EMB_TYPE_FP16)
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// sum(a x) over group g of a tile, as FP32 values; ONES: sum(x).
template <int T, int G, bool ONES>
__device__ __forceinline__ f32x4 group_sum(const typename Tile<T>::Codes& a, const u32x4 (&x)[Tile<T>::kSets], int g) {
  if constexpr (T == EMB_TYPE_INT8) {
    i32x4 c = {0, 0, 0, 0};
    const u32x4 one = {0x01010101u, 0x01010101u, 0x01010101u, 0x01010101u};
    if constexpr (G == 32) {
      const u32x4 f = ONES ? one : a[g / 2];
      const u32x2 p = g % 2 ? u32x2{f[2], f[3]} : u32x2{f[0], f[1]};
      const u32x2 q = g % 2 ? u32x2{x[g / 2][2], x[g / 2][3]} : u32x2{x[g / 2][0], x[g / 2][1]};
      c = __builtin_amdgcn_mfma_i32_16x16x32_i8(__builtin_bit_cast(long, p), __builtin_bit_cast(long, q), c, 0, 0, 0);
    } else {
#pragma unroll
      for (int i = g * (G / 64); i < (g + 1) * (G / 64); ++i)
        c = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, ONES ? one : a[i]), __builtin_bit_cast(i32x4, x[i]), c, 0, 0, 0);
    }
    // Where one value of a sum of ones is used, the other registers of it count as free, and the compiler (ROCm 7.2)
    // converts that value into a register of x that is still to be written to LDS: all four are kept.
    if constexpr (ONES) asm volatile("" : "+v"(c));
    return f32x4{(float)c[0], (float)c[1], (float)c[2], (float)c[3]};   // below 2^24: exact
  } else {
    f32x4 c = {0.0f, 0.0f, 0.0f, 0.0f};
    constexpr uint32_t o = Tile<T>::kOne;
    const u32x4 one = {o, o, o, o};
#pragma unroll
    for (int p = Tile<T>::kParts - 1; p >= 0; --p)
#pragma unroll
      for (int i = g * (G / 32); i < (g + 1) * (G / 32); ++i) c = mma<T>(ONES ? one : a[i], x[4 * p + i], c);
    if constexpr (ONES) asm volatile("" : "+v"(c));   // as above
    return c;
  }
}

// Reads of a row tile's codes, or of its pairs, through a buffer descriptor: an offset past its end reads nothing and
// gives 0, so that loops may run ahead without a branch around their loads (the compiler would wait for more than it
// has to behind one).  Sizes stay below 2^31: at most 2^17 column tiles of 1 KB.
struct Strip {
  __amdgpu_buffer_rsrc_t at;
  __device__ __forceinline__ Strip(const uint8_t* p, int bytes)
      : at(__builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p), 0, bytes, 0x00020000)) {}
  __device__ __forceinline__ u32x4 load4(int offset) const {
    return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(at, offset, 0, 0));
  }
  __device__ __forceinline__ uint32_t load1(int offset) const { return __builtin_amdgcn_raw_buffer_load_b32(at, offset, 0, 0); }
};
__device__ __forceinline__ Strip codes_strip(const W4& w, int64_t rt) { return Strip(w.base + w.tile(rt, 0), (int)(w.col_tiles * kTileBytes)); }
__device__ __forceinline__ Strip pairs_strip(const W4& w, int64_t rt) { return Strip(w.base + w.pairs(rt, 0), (int)(w.groups * kTileRows * 4)); }

// What follows the sums of one output: the row's scale, bias, activation, the type.
__device__ __forceinline__ void finish(const W4Linear& a, int64_t row, int64_t n, float v) {
  if (a.scales) v *= a.scales[row];
  if (a.bias) v += a.bias[n];
  if (a.relu && v < 0.0f) v = 0.0f;
  const int64_t at = row * a.ldy + n;
  if (a.y_type == EMB_TYPE_FP32)
    static_cast<float*>(a.y)[at] = v;
  else
    static_cast<uint16_t*>(a.y)[at] = (uint16_t)(a.y_type == EMB_TYPE_BF16 ? bf16_bits(v) : f16_bits(v));
}

// ---- up to 16 rows -----------------------------------------------------------------------------
// A workgroup computes 16 outputs of up to 16 rows; its waves (up to 16) share the column tiles.  All of the rows are in
// LDS, in the order of the operand; FP32 ones as they are (RAW) where their three parts would not fit.
constexpr int kFewWaves = 16;
constexpr int kFewLds = 65536;       // two workgroups to a CU
constexpr int kFewLdsRaw = 131072;   // one
template <int T, int G, bool RAW>
__global__ __launch_bounds__(64 * kFewWaves) void k_w4_few(W4Linear a, W4 w, int64_t first) {
  constexpr int kPer = kTileCols / G, kSets = Tile<T>::kSets;
  using X = Tile<T>;
  extern __shared__ u32x4 lds[];
  const int lane = threadIdx.x % 64, b = lane / 16, waves = blockDim.x / 64;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int64_t block = first + blockIdx.x, rt = block % w.row_tiles, row0 = block / w.row_tiles * 16;
  const int rows = a.m - row0 < 16 ? (int)(a.m - row0) : 16, tiles = (int)w.col_tiles;
  const int row = lane % 16 < rows ? lane % 16 : rows - 1;   // rows past the last one repeat it and are not stored
  const auto* x = static_cast<const typename X::E*>(a.x) + row0 * a.ldx;
  const Strip codes = codes_strip(w, rt), pairs = pairs_strip(w, rt);
  u32x4 c, pair[kPer];
  const auto load_w = [&](int kt) {
    c = codes.load4(kt * kTileBytes + lane * 16);
#pragma unroll
    for (int g = 0; g < kPer; ++g) pair[g] = pairs.load4((kt * kPer + g) * (kTileRows * 4) + b * 16);
  };
  f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
  const auto add = [&](const u32x4 (&s)[kSets], int next) {
    typename X::Codes q;
    codes_of<T>(c, q);
    u32x4 now[kPer];
#pragma unroll
    for (int g = 0; g < kPer; ++g) now[g] = pair[g];
    load_w(next);
#pragma unroll
    for (int g = 0; g < kPer; ++g) {
      const f32x4 p = group_sum<T, G, false>(q, s, g), o = group_sum<T, G, true>(q, s, g);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        sum[r] = fmaf(f16_low(now[g][r]), p[r], sum[r]);
        sum[r] = fmaf(f16_high(now[g][r]), o[r], sum[r]);
      }
    }
  };
  load_w(wave);
  // pieces of 8 columns that are whole, several loads at once; then the rest of the last tile
  const uint32_t whole = (uint32_t)(w.cols / 8), rest = (uint32_t)tiles * 16 - whole;
  const auto place = [&](uint32_t piece, uint32_t r) {   // of RAW, the first half of its 8 values
    return RAW ? lds + ((piece / 16 * 8 + piece / 4 % 4) * rows + r) * 4 + piece % 4 : lds + (piece / 16 * kSets * rows + r) * 4 + piece % 4;
  };
#pragma unroll 4
  for (uint32_t i = threadIdx.x; i < whole * rows; i += blockDim.x) {
    const uint32_t r = i / whole, piece = i % whole;
    X::template stage_whole<RAW>(x + r * a.ldx + 8 * piece, place(piece, r), piece / 4 % 4, rows * 4);
  }
#pragma unroll 1
  for (uint32_t i = threadIdx.x; i < rest * rows; i += blockDim.x) {
    const uint32_t r = i / rest, piece = whole + i % rest;
    X::template stage_part<RAW>(x + r * a.ldx + 8 * piece, (int)w.cols - 8 * (int)piece, place(piece, r), piece / 4 % 4, rows * 4);
  }
  __syncthreads();
#pragma unroll 1
  for (int kt = wave; kt < tiles; kt += waves) {
    u32x4 s[kSets];
    if constexpr (RAW) {
      X v;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const u32x4 l = lds[((kt * 8 + h * 4 + i) * rows + row) * 4 + b];
#pragma unroll
          for (int j = 0; j < 4; ++j) v.v[i].w[4 * h + j] = l[j];
        }
      v.operand(s);
    } else {
#pragma unroll
      for (int i = 0; i < kSets; ++i) s[i] = lds[((kt * kSets + i) * rows + row) * 4 + b];
    }
    add(s, kt + waves);
  }
  __syncthreads();   // x has been read
  f32x4* meet = reinterpret_cast<f32x4*>(lds);
  meet[wave * 64 + lane] = sum;
  __syncthreads();
  // 16 outputs of a row are neighbours
  for (int t = threadIdx.x; t < 256; t += blockDim.x) {
    const int n = t % 16, r = t / 16;
    float v = 0.0f;
    for (int k = 0; k < waves; ++k) v += meet[k * 64 + n / 4 * 16 + r][n % 4];
    if (r < rows && rt * 16 + n < w.rows) finish(a, row0 + r, rt * 16 + n, v);
  }
}

// ---- more rows -----------------------------------------------------------------------------------
// x first goes through the workspace: tiles of 16 rows x 128 columns in the order of the operand, zeros past the last
// column, and the sums of their groups.  Every workgroup reads all of them, whole lines at a time.  Read as they lie, rows a
// power of two apart are in one channel of the L2 (48 x 4096 x 8192 in 8 bits: 26 us, so 12.5); tiles in LDS that 128 outputs
// share make all waves wait for each other, and shares of the columns another launch (17 us).
struct Prepared {
  u32x4* x;       // [column tile][tile of 16 rows][set][lane]
  float* sums;    // [column tile][tile of 16 rows][lane]: of group b and row r at 16 b + r
  int64_t tiles;  // of 16 rows
};
template <int T>
Prepared prepared(void* workspace, int64_t m, const W4& w) {
  const int64_t tiles = ceil_div(m, 16);
  uint8_t* p = static_cast<uint8_t*>(workspace);
  return {reinterpret_cast<u32x4*>(p), reinterpret_cast<float*>(p + w.col_tiles * tiles * Tile<T>::kSets * 1024), tiles};
}

template <int T, int G>
__global__ __launch_bounds__(256) void k_w4_rows(W4Linear a, W4 w, Prepared out, int64_t first) {
  constexpr int kPer = kTileCols / G, kSets = Tile<T>::kSets;
  using X = Tile<T>;
  const int lane = threadIdx.x % 64, b = lane / 16;
  const int64_t i = (first + blockIdx.x) * 4 + threadIdx.x / 64;   // a wave a tile
  const int64_t kt = i / out.tiles, t = i % out.tiles, row = t * 16 + lane % 16;
  if (kt >= w.col_tiles) return;
  // rows past the last one repeat it
  const auto* x = static_cast<const typename X::E*>(a.x) + (row < a.m ? row : a.m - 1) * a.ldx + kt * kTileCols + 8 * b;
  X tile;
  if ((kt + 1) * kTileCols <= w.cols)
    tile.load(x);
  else
    tile.load_part(x, (int)(w.cols - kt * kTileCols) - 8 * b);
  u32x4 s[kSets];
  tile.operand(s);
#pragma unroll
  for (int k = 0; k < kSets; ++k) out.x[(i * kSets + k) * 64 + lane] = s[k];
  float total = 0.0f;
  typename X::Codes none = {};
#pragma unroll
  for (int g = 0; g < kPer; ++g) {
    const float o = group_sum<T, G, true>(none, s, g)[0];   // the same for every lane of a row
    total = g == b ? o : total;
  }
  out.sums[i * 64 + lane] = total;
}

// A workgroup computes 16 RT outputs of 16 MT rows; its waves share the column tiles.  No wave waits for another before the
// end, and no sums leave the workgroup.
template <int T>
constexpr int kMostTiles = T == EMB_TYPE_FP32 ? 2 : 4;   // of 16 rows: an operand of FP32 rows takes three times the registers
template <int RT>
constexpr int kMoreWaves = RT == 4 ? 8 : RT == 2 ? 12 : 16;   // 256 registers a wave, 168 or 128

constexpr int64_t kCus = 256;

struct WavePairs {       // scales and biases of a wave's tile, in LDS
  uint16_t scales[64];   // of group g of the tile and row r of w at 16 g + r
  uint16_t biases[64];
};

template <int T, int G, int MT, int RT>
__global__ __launch_bounds__(64 * kMoreWaves<RT>) void k_w4_more(W4Linear a, W4 w, Prepared in, int64_t first) {
  constexpr int kPer = kTileCols / G, kSets = Tile<T>::kSets;
  constexpr int kRing = kSets <= 4 && MT > 1 ? 2 : 1;   // operands under way
  constexpr bool kBiasByMatrix = G < 128;   // up to four groups are one FP32 matrix instruction; one is less by itself
  extern __shared__ u32x4 lds[];
  const int lane = threadIdx.x % 64, b = lane / 16, waves = blockDim.x / 64;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int64_t block = first + blockIdx.x, wide = ceil_div(w.row_tiles, RT), rt0 = block % wide * RT, t0 = block / wide * MT;
  const int tiles = (int)w.col_tiles;
  WavePairs* mine = reinterpret_cast<WavePairs*>(lds) + wave * RT;
  // tiles past the last one repeat it and are not stored, of x and of w
  int64_t at[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) at[t] = t0 + t < in.tiles ? t0 + t : in.tiles - 1;
  u32x4 c[RT];
  uint32_t p[RT];
  const auto strip_of = [&](int i) { return rt0 + i < w.row_tiles ? rt0 + i : w.row_tiles - 1; };
  const auto load_w = [&](int kt) {
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      p[i] = pairs_strip(w, strip_of(i)).load1((kt * kPer * 16 + lane % (16 * kPer)) * 4);
      c[i] = codes_strip(w, strip_of(i)).load4(kt * kTileBytes + lane * 16);
    }
  };
  f32x4 sum[RT][MT] = {};
  load_w(wave);
#pragma unroll 1
  for (int kt = wave; kt < tiles; kt += waves) {
    u32x4 s[kRing][kSets];
    float ones[MT];
    const auto load_x = [&](int t) {
      const int64_t i = kt * in.tiles + at[t];
#pragma unroll
      for (int k = 0; k < kSets; ++k) s[t % kRing][k] = in.x[(i * kSets + k) * 64 + lane];
    };
#pragma unroll
    for (int t = 0; t < MT; ++t) ones[t] = in.sums[(kt * in.tiles + at[t]) * 64 + (kBiasByMatrix ? lane : lane % 16)];
#pragma unroll
    for (int t = 0; t < kRing; ++t) load_x(t);
    typename Tile<T>::Codes q[RT];
    float bias[RT];
    u32x2 scale[RT][kPer], one_bias[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      mine[i].scales[lane] = (uint16_t)p[i];
      mine[i].biases[lane] = (uint16_t)(p[i] >> 16);
      bias[i] = b < kPer ? f16_high(p[i]) : 0.0f;
      codes_of<T>(c[i], q[i]);
    }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < RT; ++i) {
#pragma unroll
      for (int g = 0; g < kPer; ++g) scale[i][g] = *reinterpret_cast<const u32x2*>(&mine[i].scales[16 * g + 4 * b]);
      one_bias[i] = *reinterpret_cast<const u32x2*>(&mine[i].biases[4 * b]);
    }
    __builtin_amdgcn_wave_barrier();
    if constexpr (MT <= kRing) load_w(kt + waves);
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      // loads return in order: those of w, from farther away, go last
      const auto next = [&] {
        if (t + kRing < MT) load_x(t + kRing);
        if (t + kRing == MT - 1) load_w(kt + waves);
        __builtin_amdgcn_sched_barrier(0);
      };
#pragma unroll
      for (int i = 0; i < RT; ++i) {
        if constexpr (kBiasByMatrix) {
          sum[i][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(bias[i], ones[t], sum[i][t], 0, 0, 0);
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k)
            sum[i][t][k] = fmaf(k % 2 ? f16_high(one_bias[i][k / 2]) : f16_low(one_bias[i][k / 2]), ones[t], sum[i][t][k]);
        }
#pragma unroll
        for (int g = 0; g < kPer; ++g) {
          const f32x4 v = group_sum<T, G, false>(q[i], s[t % kRing], g);
#pragma unroll
          for (int k = 0; k < 4; ++k)
            sum[i][t][k] = fmaf(k % 2 ? f16_high(scale[i][g][k / 2]) : f16_low(scale[i][g][k / 2]), v[k], sum[i][t][k]);
        }
      }
      next();
    }
  }
  __syncthreads();   // scales and biases have been read
  f32x4* meet = reinterpret_cast<f32x4*>(lds);
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int t = 0; t < MT; ++t) meet[((wave * RT + i) * MT + t) * 64 + lane] = sum[i][t];
  __syncthreads();
  // 16 RT outputs of a row are neighbours
  for (int i = threadIdx.x; i < 256 * RT * MT; i += blockDim.x) {
    const int n = i % (16 * RT), m = i / (16 * RT);
    const f32x4* from = meet + ((n / 16) * MT + m / 16) * 64 + n % 16 / 4 * 16 + m % 16;
    float v = 0.0f;
    for (int k = 0; k < waves; ++k) v += from[k * RT * MT * 64][n % 4];
    if (t0 * 16 + m < a.m && rt0 * 16 + n < w.rows) finish(a, t0 * 16 + m, rt0 * 16 + n, v);
  }
}

// ---- which of them -----------------------------------------------------------------------------
template <int T, int G, int MT, int RT>
hipError_t more_as(const W4Linear& a, const W4& w, const Prepared& in, hipStream_t s) {
  int waves = 4;   // of those that have a column tile
  while (waves < kMoreWaves<RT> && waves < w.col_tiles) waves += 4;
  return in_launches(ceil_div(w.row_tiles, RT) * ceil_div(in.tiles, MT), 64 * waves, [&](int64_t first, unsigned n) {
    k_w4_more<T, G, MT, RT><<<n, 64 * waves, waves * RT * MT * 1024, s>>>(a, w, in, first);
    return hipGetLastError();
  });
}

template <int T, int G, int MT>
hipError_t more_of(const W4Linear& a, const W4& w, const Prepared& in, hipStream_t s) {
  // A workgroup fills a CU.  Of 32 outputs, it takes less than twice the time, as it reads x half as often: taken where there are more
  // than CUs.  Of 64, it takes four thirds of that and halves the rounds of the CUs, to which an odd one counts in full: two
  // rounds for three take as long.  64 BF16 rows of 4096, groups of 32 (and 128), us, with 16 and 32 outputs a workgroup: to 4096
  // outputs 12.8 and 15.4 (12.0 and 14.3), 5120 18.9 and 15.5 (18.5 and 14.4); with 32 and 64: to 8192 17.5 and 23.5 (15.9 and 18.4),
  // 12800 27.3 and 23.7 (25.3 and 19.1), 20480 39.7 and 41.6 (36.3 and 33.2), 32768 53.7 and 43.8 (48.1 and 36.2).  20 FP32 rows to
  // 4352 with 16 and 32: 22.1 and 15.6 (21.4 and 15.3); they have no registers for 64.
  const int64_t blocks = ceil_div(in.tiles, MT), rounds2 = ceil_div(ceil_div(w.row_tiles, 2) * blocks, kCus);
  if constexpr (MT >= 2 && T != EMB_TYPE_FP32)
    if (3 * ceil_div(ceil_div(w.row_tiles, 4) * blocks, kCus) < 2 * rounds2) return more_as<T, G, MT, 4>(a, w, in, s);
  return w.row_tiles * blocks > kCus ? more_as<T, G, MT, 2>(a, w, in, s) : more_as<T, G, MT, 1>(a, w, in, s);
}

// Bytes of LDS that x takes in k_w4_few (of a block of 16 rows where there are more); as it is: of FP32 rows.
template <int T>
int64_t few_bytes(int64_t m, int64_t k, bool raw) {
  return (m < 16 ? m : 16) * ceil_div(k, kTileCols) * (raw ? 512 : Tile<T>::kSets * 64);
}
template <int T>
bool few_raw(int64_t m, int64_t k) { return T == EMB_TYPE_FP32 && few_bytes<T>(m, k, false) > kFewLds; }
// Whether k_w4_few takes a product.
template <int T>
bool few(int64_t m, int64_t n, int64_t k) {
  const bool raw = few_raw<T>(m, k);
  if (few_bytes<T>(m, k, raw) > (raw ? kFewLdsRaw : kFewLds)) return false;
  // the weight is read for each 16 rows; us (BF16, the other way): 64 x 2048 x 2048 7.5 (9.3), 64 x 8192 x 512 7.7 (9.4),
  // 32 x 8192 x 2048 15.1 (9.0)
  return m <= 16 || ceil_div(m, 16) * ceil_div(n, 16) * ceil_div(k, kTileCols) <= 8192;
}

template <int T, int G>
hipError_t few_as(const W4Linear& a, const W4& w, hipStream_t s) {
  int waves = 4;   // enough to fill the CUs, of those that have a column tile
  const int64_t blocks = w.row_tiles * ceil_div(a.m, 16);
  while (waves < kFewWaves && waves < w.col_tiles && waves * blocks < 256 * kFewWaves) waves *= 2;
  const bool raw = few_raw<T>(a.m, w.cols);
  const int64_t x_bytes = few_bytes<T>(a.m, w.cols, raw), meet = waves * 1024;
  const size_t bytes = (size_t)(x_bytes > meet ? x_bytes : meet);
  return in_launches(blocks, 64 * waves, [&](int64_t first, unsigned n) {
    if constexpr (T == EMB_TYPE_FP32) {
      if (raw) {
        k_w4_few<T, G, true><<<n, 64 * waves, bytes, s>>>(a, w, first);
        return hipGetLastError();
      }
    }
    k_w4_few<T, G, false><<<n, 64 * waves, bytes, s>>>(a, w, first);
    return hipGetLastError();
  });
}

template <int T, int G>
hipError_t linear_as(const W4Linear& a, const W4& w, void* workspace, hipStream_t s) {
  if (few<T>(a.m, w.rows, w.cols)) return few_as<T, G>(a, w, s);
  const Prepared in = prepared<T>(workspace, a.m, w);
  const hipError_t e = in_launches(ceil_div(w.col_tiles * in.tiles, 4), 256, [&](int64_t first, unsigned n) {
    k_w4_rows<T, G><<<n, 256, 0, s>>>(a, w, in, first);
    return hipGetLastError();
  });
  if (e != hipSuccess) return e;
  if (in.tiles == 1) return more_of<T, G, 1>(a, w, in, s);
  if (in.tiles == 2 || kMostTiles<T> == 2) return more_of<T, G, 2>(a, w, in, s);
  if constexpr (kMostTiles<T> > 2) return in.tiles == 3 ? more_of<T, G, 3>(a, w, in, s) : more_of<T, G, 4>(a, w, in, s);
  return hipErrorInvalidValue;
}

template <int T>
hipError_t linear_of(const W4Linear& a, const W4& w, void* workspace, hipStream_t s) {
  if (w.group == 32) return linear_as<T, 32>(a, w, workspace, s);
  if (w.group == 64) return linear_as<T, 64>(a, w, workspace, s);
  return linear_as<T, 128>(a, w, workspace, s);
}

template <int T>
size_t workspace_of(int64_t m, int64_t n, int64_t k) {
  return few<T>(m, n, k) ? 0 : (size_t)(ceil_div(k, kTileCols) * ceil_div(m, 16)) * (Tile<T>::kSets * 1024 + 256);
}

}  // namespace

size_t w4_linear_workspace(int type, int64_t m, int64_t n, int64_t k, int group) {
  if (type == EMB_TYPE_FP32) return workspace_of<EMB_TYPE_FP32>(m, n, k);
  if (type == EMB_TYPE_INT8) return workspace_of<EMB_TYPE_INT8>(m, n, k);
  return workspace_of<EMB_TYPE_BF16>(m, n, k);
}

hipError_t launch_w4_linear(const W4Linear& a, int type, const W4& w, void* workspace, hipStream_t s) {
  if (type == EMB_TYPE_FP32) return linear_of<EMB_TYPE_FP32>(a, w, workspace, s);
  if (type == EMB_TYPE_BF16) return linear_of<EMB_TYPE_BF16>(a, w, workspace, s);
  if (type == EMB_TYPE_FP16) return linear_of<EMB_TYPE_FP16>(a, w, workspace, s);
  return linear_of<EMB_TYPE_INT8>(a, w, workspace, s);
}

}  // namespace embd
