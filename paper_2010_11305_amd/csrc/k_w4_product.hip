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

// 16 rows x 128 columns of x as the second operand: lane 16 b + r holds columns 32 i + 8 b + (0 .. 7) of row r.
// kSets registers sets of 16 bytes: for i = 0 .. 3 of each part of FP32 rows, or i = 0, 1 and 2, 3 of 8-bit rows.
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
  __device__ __forceinline__ void operand(u32x4 (&s)[kSets]) const {
    if constexpr (T == EMB_TYPE_FP32) {
      // cut to the 8 bits of BF16 twice; what is left has 8
      float x[4][8];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) x[i][j] = __uint_as_float(v[i].w[j]);
#pragma unroll
      for (int p = 0; p < 3; ++p)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 8; j += 2) {
            const uint32_t lo = __float_as_uint(x[i][j]), hi = __float_as_uint(x[i][j + 1]);
            s[4 * p + i][j / 2] = __builtin_amdgcn_perm(hi, lo, 0x07060302u);
            x[i][j] -= __uint_as_float(lo & 0xFFFF0000u);
            x[i][j + 1] -= __uint_as_float(hi & 0xFFFF0000u);
          }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) s[i] = u32x4{v[i].w[0], v[i].w[1], v[i].w[2], v[i].w[3]};
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
    struct __attribute__((packed, aligned(1))) Bytes {
      uint32_t w[2];
    };
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const Bytes w = *reinterpret_cast<const Bytes*>(p + 32 * i);
      v[i] = u32x2{w.w[0], w.w[1]};
    }
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
// A workgroup computes 16 outputs of 16 rows; its waves (up to 16) share the column tiles.
constexpr int kFewWaves = 16;
// Column tiles whose loads a wave has under way at once.
template <int T, int G>
constexpr int kAhead = T == EMB_TYPE_FP32 || G == 32 ? 2 : G == 64 ? 3 : 4;

template <int T, int G>
__global__ __launch_bounds__(64 * kFewWaves) void k_w4_few(W4Linear a, W4 w, int64_t first) {
  constexpr int kPer = kTileCols / G, D = kAhead<T, G>;
  using X = Tile<T>;
  __shared__ f32x4 meet[kFewWaves][64];
  const int lane = threadIdx.x % 64, b = lane / 16, waves = blockDim.x / 64;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int64_t block = first + blockIdx.x, rt = block % w.row_tiles, row0 = block / w.row_tiles * 16;
  const int64_t row = row0 + lane % 16;
  // rows past the last one repeat it and are not stored
  const typename X::E* x = static_cast<const typename X::E*>(a.x) + (row < a.m ? row : a.m - 1) * a.ldx + 8 * b;
  const u32x4* codes = reinterpret_cast<const u32x4*>(w.base + w.tile(rt, 0)) + lane;
  const u32x4* pairs = reinterpret_cast<const u32x4*>(w.base + w.pairs(rt, 0)) + b;
  const int whole = (int)(w.cols / kTileCols), tail = (int)(w.cols % kTileCols);
  f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
  const auto add = [&](const u32x4& c, const u32x4 (&pair)[kPer], const X& rows) {
    typename X::Codes q;
    u32x4 s[X::kSets];
    codes_of<T>(c, q);
    rows.operand(s);
#pragma unroll
    for (int g = 0; g < kPer; ++g) {
      const f32x4 p = group_sum<T, G, false>(q, s, g), o = group_sum<T, G, true>(q, s, g);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        sum[r] = fmaf(f16_low(pair[g][r]), p[r], sum[r]);
        sum[r] = fmaf(f16_high(pair[g][r]), o[r], sum[r]);
      }
    }
  };
  for (int kt = wave; kt < whole; kt += D * waves) {
    u32x4 c[D], pair[D][kPer];
    X rows[D];
#pragma unroll
    for (int d = 0; d < D; ++d) {
      const int64_t at = kt + d * waves < whole ? kt + d * waves : kt;   // beyond the last: loaded and not used
      c[d] = codes[at * 64];
#pragma unroll
      for (int g = 0; g < kPer; ++g) pair[d][g] = pairs[(at * kPer + g) * 4];
      rows[d].load(x + at * kTileCols);
    }
#pragma unroll
    for (int d = 0; d < D; ++d)
      if (kt + d * waves < whole) add(c[d], pair[d], rows[d]);
  }
  if (tail && wave == whole % waves) {
    u32x4 pair[kPer];
#pragma unroll
    for (int g = 0; g < kPer; ++g) pair[g] = pairs[((int64_t)whole * kPer + g) * 4];
    X rows;
    rows.load_part(x + (int64_t)whole * kTileCols, tail - 8 * b);
    add(codes[(int64_t)whole * 64], pair, rows);
  }
  meet[wave][lane] = sum;
  __syncthreads();
  if (threadIdx.x >= 256) return;
  // 16 outputs of a row are neighbours
  for (int t = threadIdx.x; t < 256; t += blockDim.x) {
    const int n = t % 16, r = t / 16;
    float v = 0.0f;
    for (int k = 0; k < waves; ++k) v += meet[k][n / 4 * 16 + r][n % 4];
    if (row0 + r < a.m && rt * 16 + n < w.rows) finish(a, row0 + r, rt * 16 + n, v);
  }
}

// ---- up to 64 rows -----------------------------------------------------------------------------
// A workgroup computes 128 outputs of 16 MT rows over a share of the column tiles: two halves of four waves take them in
// turn, each wave two row tiles of w.  A half's waves put a tile of x into LDS in the order of the operand, and with it the
// sums of its groups, which one matrix instruction makes of the registers that are on their way there.  The halves
// meet in LDS, the shares of the columns in the workspace.
constexpr int kBatchWaves = 4, kBatchRows = 2, kBatchThreads = 2 * 64 * kBatchWaves;
constexpr int kBatchOut = kBatchWaves * kBatchRows * kTileRows;   // 128
constexpr int kCodesAhead = 3;   // iterations that the loads of codes, scales and biases run ahead

template <int T>
constexpr int kMostTiles = T == EMB_TYPE_FP32 ? 2 : 4;   // of 16 rows: FP32 rows take three times the LDS

template <int T, int G, int MT>
struct BatchStage {
  u32x4 x[MT][Tile<T>::kSets][64];
  float sums[MT][64];                            // of group b of the tile and row r at 16 b + r
  uint32_t pairs[kBatchWaves][kBatchRows][64];   // (scale, bias) of group b, row r of w
};

template <int T, int G, int MT>
__global__ __launch_bounds__(kBatchThreads) void k_w4_batch(W4Linear a, W4 w, float* __restrict__ partial, int shares, int64_t first) {
  constexpr int kPer = kTileCols / G, kSets = Tile<T>::kSets;
  using X = Tile<T>;
  using Stage = BatchStage<T, G, MT>;
  __shared__ Stage stages[2][2];
  static_assert(sizeof(stages) >= sizeof(f32x4) * kBatchWaves * kBatchRows * MT * 64);
  const int lane = threadIdx.x % 64, b = lane / 16, r = lane % 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), half = wave / kBatchWaves, own = wave % kBatchWaves;
  // shares of the same rows of w are far apart, workgroups of the same share of the columns and rows of x near: they
  // read the same part of x
  const int64_t block = first + blockIdx.x, wide = ceil_div(w.row_tiles, kBatchWaves * kBatchRows);
  const int64_t nb = block % wide, share = block / wide % shares, mb = block / wide / shares;
  const int64_t row0 = mb * MT * 16;
  const int tiles = (int)w.col_tiles;
  const int kt0 = (int)((int64_t)tiles * share / shares), kt1 = (int)((int64_t)tiles * (share + 1) / shares);
  const int steps = (kt1 - kt0 + 1) / 2;
  const int whole = (int)(w.cols / kTileCols);

  // what this wave reads of w
  int64_t rt[kBatchRows];
#pragma unroll
  for (int i = 0; i < kBatchRows; ++i) {
    rt[i] = (nb * kBatchWaves + own) * kBatchRows + i;
    if (rt[i] >= w.row_tiles) rt[i] = w.row_tiles - 1;   // read again, not stored
  }
  u32x4 codes[kCodesAhead][kBatchRows];
  uint32_t pairs[kCodesAhead][kBatchRows];
  const auto tile_of = [&](int step) {
    const int kt = kt0 + 2 * step + half;
    return kt < kt1 ? kt : kt1 - 1;   // beyond the last: loaded and not used
  };
  const auto load_w = [&](int step, u32x4 (&c)[kBatchRows], uint32_t (&p)[kBatchRows]) {
    const int kt = tile_of(step);
#pragma unroll
    for (int i = 0; i < kBatchRows; ++i) {
      c[i] = reinterpret_cast<const u32x4*>(w.base + w.tile(rt[i], kt))[lane];
      p[i] = reinterpret_cast<const uint32_t*>(w.base + w.pairs(rt[i], (int64_t)kt * kPer))[lane % (16 * kPer)];
    }
  };
  // the tile of x that this wave puts into LDS, of rows own, own + 4, .. (MT is at most 4: one, or none)
  const bool brings = own < MT;
  const int64_t row = row0 + own * 16 + r;
  const typename X::E* x = static_cast<const typename X::E*>(a.x) + (row < a.m ? row : a.m - 1) * a.ldx + 8 * b;
  X rows;
  const auto load_x = [&](int step) {
    if (!brings) return;
    const int kt = tile_of(step);
    if (kt < whole)
      rows.load(x + (int64_t)kt * kTileCols);
    else
      rows.load_part(x + (int64_t)kt * kTileCols, (int)(w.cols - (int64_t)kt * kTileCols) - 8 * b);
  };
  f32x4 sum[kBatchRows][MT] = {};
  load_x(0);
#pragma unroll
  for (int s = 0; s < kCodesAhead; ++s) load_w(s, codes[s], pairs[s]);
  const auto step = [&](int it, u32x4 (&c)[kBatchRows], uint32_t (&p)[kBatchRows]) {
    Stage& st = stages[half][it % 2];
    if (brings) {
      u32x4 s[kSets];
      rows.operand(s);
#pragma unroll
      for (int i = 0; i < kSets; ++i) st.x[own][i][lane] = s[i];
      float total = 0.0f;
      typename X::Codes none = {};
#pragma unroll
      for (int g = 0; g < kPer; ++g) {
        const float o = group_sum<T, G, true>(none, s, g)[0];   // the same for every lane of a row
        total = g == b ? o : total;
      }
      st.sums[own][lane] = total;
    }
#pragma unroll
    for (int i = 0; i < kBatchRows; ++i) st.pairs[own][i][lane] = p[i];
    typename X::Codes q[kBatchRows];
#pragma unroll
    for (int i = 0; i < kBatchRows; ++i) codes_of<T>(c[i], q[i]);
    load_x(it + 1);
    load_w(it + kCodesAhead, c, p);
    __syncthreads();
    if (kt0 + 2 * it + half >= kt1) return;
    // bias * sum(x) of up to four groups is one FP32 matrix instruction
    float bias[kBatchRows];
#pragma unroll
    for (int i = 0; i < kBatchRows; ++i) bias[i] = b < kPer ? f16_high(st.pairs[own][i][lane]) : 0.0f;
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      u32x4 s[kSets];
#pragma unroll
      for (int i = 0; i < kSets; ++i) s[i] = st.x[t][i][lane];
      const float ones = st.sums[t][lane];
#pragma unroll
      for (int i = 0; i < kBatchRows; ++i) {
        sum[i][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(bias[i], ones, sum[i][t], 0, 0, 0);
#pragma unroll
        for (int g = 0; g < kPer; ++g) {
          const f32x4 v = group_sum<T, G, false>(q[i], s, g);
          const u32x4 pair = *reinterpret_cast<const u32x4*>(&st.pairs[own][i][16 * g + 4 * b]);
#pragma unroll
          for (int k = 0; k < 4; ++k) sum[i][t][k] = fmaf(f16_low(pair[k]), v[k], sum[i][t][k]);
        }
      }
    }
  };
  for (int it = 0; it < steps; it += kCodesAhead) {
#pragma unroll
    for (int s = 0; s < kCodesAhead; ++s)
      if (it + s < steps) step(it + s, codes[s], pairs[s]);
  }
  __syncthreads();
  f32x4* meet = reinterpret_cast<f32x4*>(&stages[0][0]);
  const auto place = [&](int i, int t) { return ((own * kBatchRows + i) * MT + t) * 64 + lane; };
  if (half) {
#pragma unroll
    for (int i = 0; i < kBatchRows; ++i)
#pragma unroll
      for (int t = 0; t < MT; ++t) meet[place(i, t)] = sum[i][t];
  }
  __syncthreads();
  if (half) return;
#pragma unroll
  for (int i = 0; i < kBatchRows; ++i) {
    const int64_t n = ((nb * kBatchWaves + own) * kBatchRows + i) * 16 + 4 * b;
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      const f32x4 v = sum[i][t] + meet[place(i, t)];
      const int64_t m = row0 + t * 16 + r;
      if (m >= a.m || n >= w.rows) continue;
      if (shares > 1) {
        // rows of whole row tiles: four outputs at once
        *reinterpret_cast<f32x4*>(partial + (share * a.m + m) * w.row_tiles * 16 + n) = v;
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (n + k < w.rows) finish(a, m, n + k, v[k]);
      }
    }
  }
}

// The shares' sums together: four outputs a thread.
__global__ __launch_bounds__(256) void k_w4_join(W4Linear a, W4 w, const float* __restrict__ partial, int shares, int64_t first) {
  const int64_t wide = w.row_tiles * 4, i = (first + blockIdx.x) * 256 + threadIdx.x, m = i / wide, n = i % wide * 4;
  if (m >= a.m || n >= w.rows) return;
  f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
  const f32x4* p = reinterpret_cast<const f32x4*>(partial) + i;
#pragma unroll 4
  for (int s = 0; s < shares; ++s) v += p[s * a.m * wide];
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (n + k < w.rows) finish(a, m, n + k, v[k]);
}

// ---- which of them -----------------------------------------------------------------------------
bool few(int64_t m) { return m <= 16; }

// Shares of the columns: as many workgroups as there are CUs, each with two tiles at least for either half.
int batch_shares(int64_t m, int64_t n, int64_t k, int most_tiles) {
  const int64_t blocks = ceil_div(ceil_div(n, 16), kBatchWaves * kBatchRows) * ceil_div(m, 16 * most_tiles);
  const int64_t tiles = ceil_div(k, kTileCols), want = 256 / blocks, most = tiles / 4;
  const int64_t s = want < most ? want : most;
  return s < 1 ? 1 : (int)s;
}
int most_tiles(int type) { return type == EMB_TYPE_FP32 ? kMostTiles<EMB_TYPE_FP32> : kMostTiles<EMB_TYPE_BF16>; }

template <int T, int G, int MT>
hipError_t batch_as(const W4Linear& a, const W4& w, float* partial, int shares, hipStream_t s) {
  const int64_t blocks = ceil_div(w.row_tiles, kBatchWaves * kBatchRows) * shares * ceil_div(a.m, 16 * MT);
  return in_launches(blocks, kBatchThreads, [&](int64_t first, unsigned n) {
    k_w4_batch<T, G, MT><<<n, kBatchThreads, 0, s>>>(a, w, partial, shares, first);
    return hipGetLastError();
  });
}

template <int T, int G>
hipError_t linear_as(const W4Linear& a, const W4& w, float* partial, hipStream_t s) {
  if (few(a.m) || !w.cols) {
    int waves = 4;   // enough to fill the CUs, of those that have a column tile
    while (waves < kFewWaves && waves < w.col_tiles && waves * w.row_tiles < 256 * kFewWaves) waves *= 2;
    return in_launches(w.row_tiles * ceil_div(a.m, 16), 64 * waves, [&](int64_t first, unsigned n) {
      k_w4_few<T, G><<<n, 64 * waves, 0, s>>>(a, w, first);
      return hipGetLastError();
    });
  }
  const int shares = batch_shares(a.m, w.rows, w.cols, kMostTiles<T>);
  const int64_t tiles = ceil_div(a.m, 16);
  hipError_t e;
  if (tiles <= 2 || kMostTiles<T> == 2)
    e = batch_as<T, G, 2>(a, w, partial, shares, s);
  else if (tiles == 3)
    e = batch_as<T, G, kMostTiles<T> == 2 ? 2 : 3>(a, w, partial, shares, s);
  else
    e = batch_as<T, G, kMostTiles<T>>(a, w, partial, shares, s);
  if (e != hipSuccess || shares == 1) return e;
  return in_launches(ceil_div(a.m * w.row_tiles * 4, 256), 256, [&](int64_t first, unsigned n) {
    k_w4_join<<<n, 256, 0, s>>>(a, w, partial, shares, first);
    return hipGetLastError();
  });
}

template <int T>
hipError_t linear_of(const W4Linear& a, const W4& w, float* partial, hipStream_t s) {
  if (w.group == 32) return linear_as<T, 32>(a, w, partial, s);
  if (w.group == 64) return linear_as<T, 64>(a, w, partial, s);
  return linear_as<T, 128>(a, w, partial, s);
}

}  // namespace

size_t w4_linear_workspace(int type, int64_t m, int64_t n, int64_t k, int group) {
  if (few(m)) return 0;
  const int shares = batch_shares(m, n, k, most_tiles(type));
  return shares > 1 ? (size_t)shares * (size_t)m * (size_t)ceil_div(n, 16) * 16 * 4 : 0;
}

hipError_t launch_w4_linear(const W4Linear& a, int type, const W4& w, void* workspace, hipStream_t s) {
  float* partial = static_cast<float*>(workspace);
  if (type == EMB_TYPE_FP32) return linear_of<EMB_TYPE_FP32>(a, w, partial, s);
  if (type == EMB_TYPE_BF16) return linear_of<EMB_TYPE_BF16>(a, w, partial, s);
  if (type == EMB_TYPE_FP16) return linear_of<EMB_TYPE_FP16>(a, w, partial, s);
  return linear_of<EMB_TYPE_INT8>(a, w, partial, s);
}

}  // namespace embd
