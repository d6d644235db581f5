// MX4 matrices: quantisation by rows and by columns, expansion, and the plain codes.
//
// Rounding to nearest and expansion are bound by memory.  16384 x 12800 BF16 (420 MB): by rows 95 us, by columns
// 100 us, both 122 to 127 us (5.1 to 5.6 TB/s of the bytes that have to move; a copy of 1 GiB reaches 5.0);
// expansion to BF16 114 us (4.7 TB/s).  FP32: 174, 188, 203 and 181 us.  Plain codes to tiles and back 39 and 40 us a
// call, 5.8 and 5.6 TB/s (223 MB, which the last-level cache may hold); 1999 columns, whose rows of codes and scales lie
// at odd addresses, 9.9 us at 16383 rows (3.5 TB/s).
// Stochastic rounding is bound by the VALU: 154, 151 and 214 to 218 us.  Per value 2.3 of its 17 instructions are the
// multiplications of Philox, which issue at a quarter of the rate: two fifths of its time.
#include "dense_device.h"

namespace embd {

namespace {

// The scale byte of a block; with those of the last column tile, zeros for the tiles that its
// group lacks (a product may run over them).
__device__ __forceinline__ void store_scale(uint8_t* out, const Mx4& q, int64_t rt, int64_t kt, int lane, uint32_t s) {
  uint8_t* p = out + q.scale(rt, kt, lane);
  *p = (uint8_t)s;
  if (kt + 1 == q.col_tiles)
    for (int t = (int)(kt % kScaleTiles) + 1; t < kScaleTiles; ++t) *++p = 0;
}

// A workgroup stages 32 rows x 128 columns of x in LDS, read in whole lines, and quantises them along the
// rows, the columns or both: a thread takes 32 values that share a scale, so no step crosses lanes, and
// writes its 16 bytes of codes where 16 threads make 256 contiguous ones.  For both, one half of
// the threads takes the columns (a wave reads a row of the stage at a time) and the other the rows; for one
// the other half only loads (256 x 416: 3.3 us, with 128 threads 3.9; 16384 x 12800: 95 us and 103).
template <int TYPE, bool BY_COLUMNS>
struct Stage {
  static constexpr int kPiece = 16 / Elem<TYPE>::kBytes;
  static constexpr int kRows = kQuantizeRows;
  static constexpr int kThreads = 256;
  static constexpr int kPitch = kTileCols + kPiece;  // 16 more bytes a row: rows start in different banks
  // The scale bytes of four tiles along a quantised axis lie in one dword, and a column's codes of 128 rows in one
  // tile: where there are many workgroups those of 512 rows (by columns) x 512 columns run on one XCD, whose
  // L2 joins what they write.
  static constexpr int kSquareRows = square_rows(BY_COLUMNS);
  static constexpr int kSquare = kSquareRows * kSquareCols;
};
static_assert(kQuantizeRows == kBlock && kQuantizeCols == kTileCols);

template <int TYPE, bool STOCHASTIC, bool BY_ROWS, bool BY_COLUMNS>
__global__ __launch_bounds__(256) void k_quantize(const typename Elem<TYPE>::type* __restrict__ x, Mx4 qr, Mx4 qc,
                                                  int64_t ld, uint8_t* __restrict__ by_rows,
                                                  uint8_t* __restrict__ by_columns, Mx4Random rnd, uint32_t first,
                                                  uint32_t workgroups) {
  using E = typename Elem<TYPE>::type;
  using St = Stage<TYPE, BY_COLUMNS>;
  constexpr int kPiece = St::kPiece, kPitch = St::kPitch, kPieces = kTileCols / kPiece;
  __shared__ __attribute__((aligned(16))) E stage[St::kRows * kPitch];
  const uint32_t wide = (uint32_t)((qr.cols + kTileCols * kSquareCols - 1) / (kTileCols * kSquareCols));
  const uint32_t block = first + blockIdx.x;
  uint32_t square = block / St::kSquare, in = block % St::kSquare;
  if (workgroups >= kSquaresFrom * St::kSquare) {  // workgroups go to the XCDs in turn
    square = block / (8 * St::kSquare) * 8 + block % 8;
    in = block / 8 % St::kSquare;
  }
  // counts of workgroups and tiles are below 2^31: divisions of 32 bits
  const int64_t row0 = ((int64_t)(square / wide) * St::kSquareRows + in / kSquareCols) * St::kRows;
  const int64_t kt0 = (int64_t)(square % wide) * kSquareCols + in % kSquareCols, col0 = kt0 * kTileCols;
  // by columns the rows go on to the end of their tile of 128
  const int64_t row_end = BY_COLUMNS ? qc.col_tiles * kTileCols : qr.row_tiles * kTileRows;
  if (row0 >= row_end || kt0 >= qr.col_tiles) return;
#pragma unroll
  for (int i = 0; i < St::kRows * kPieces / St::kThreads; ++i) {
    const int id = i * St::kThreads + threadIdx.x, r = id / kPieces, c = id % kPieces * kPiece;
    const int64_t row = row0 + r, left = row < qr.rows ? qr.cols - col0 - c : 0;
    Raw<TYPE, kPiece> v;
    load_values(x + (left > 0 ? row * ld + col0 + c : 0), (int)(left < 0 ? 0 : left > kPiece ? kPiece : left), v);
    *reinterpret_cast<uint4*>(&stage[r * kPitch + c]) = make_uint4(v.w[0], v.w[1], v.w[2], v.w[3]);
  }
  __syncthreads();
  Raw<TYPE, kBlock> r;
  uint32_t s;
  if (BY_COLUMNS && threadIdx.x < 128) {
    const int c = threadIdx.x;
    const int64_t col = col0 + c, rt = col / kTileRows, kt = row0 / kTileCols;
    if (rt >= qc.row_tiles) return;
#pragma unroll
    for (int j = 0; j < kBlock; ++j) r.put(j, load_bits<TYPE>(&stage[j * kPitch + c]));
    Mx4Random q = rnd;
    q.tag += 1;
    const uint4 code = quantize_block<TYPE, STOCHASTIC>(r, (uint32_t)(row0 / 8), (uint32_t)col, q, &s);
    const int lane = (int)(row0 % kTileCols / kBlock) * 16 + (int)(col % kTileRows);
    *reinterpret_cast<uint4*>(by_columns + qc.tile(rt, kt) + 16 * lane) = code;
    store_scale(by_columns, qc, rt, kt, lane, s);
  } else if (BY_ROWS && (BY_COLUMNS || threadIdx.x < 128)) {
    const int task = threadIdx.x % 128, rr = task % St::kRows, h = task / St::kRows;
    const int64_t row = row0 + rr, col = col0 + h * kBlock, rt = row / kTileRows;
    if (rt >= qr.row_tiles) return;
#pragma unroll
    for (int i = 0; i < kBlock / kPiece; ++i) {
      const uint4 v = *reinterpret_cast<const uint4*>(&stage[rr * kPitch + h * kBlock + i * kPiece]);
      r.w[4 * i] = v.x, r.w[4 * i + 1] = v.y, r.w[4 * i + 2] = v.z, r.w[4 * i + 3] = v.w;
    }
    const uint4 code = quantize_block<TYPE, STOCHASTIC>(r, (uint32_t)(col / 8), (uint32_t)row, rnd, &s);
    const int lane = h * 16 + (int)(row % kTileRows);
    *reinterpret_cast<uint4*>(by_rows + qr.tile(rt, kt0) + 16 * lane) = code;
    store_scale(by_rows, qr, rt, kt0, lane, s);
  }
}

// Expansion: a thread takes 8 values (one dword of codes), 16 consecutive threads one row of a
// tile, so that a wave writes whole lines.
template <int TYPE>
__global__ __launch_bounds__(256) void k_dequantize(Mx4 q, typename Elem<TYPE>::type* __restrict__ x, int64_t ld,
                                                    uint32_t first) {
  const uint32_t wide = (uint32_t)q.col_tiles, tile = first + blockIdx.x;
  const int64_t rt = tile / wide, kt = tile % wide;
  const int rr = threadIdx.x >> 4, c8 = threadIdx.x & 15, lane = (c8 >> 2) * 16 + rr;
  const int64_t row = rt * kTileRows + rr, col = kt * kTileCols + c8 * 8;
  if (row >= q.rows || col >= q.cols) return;
  const uint32_t c = *reinterpret_cast<const uint32_t*>(q.base + q.tile(rt, kt) + 16 * lane + 4 * (c8 & 3));
  const uint32_t s = q.base[q.scale(rt, kt, lane)];
  Raw<TYPE, 8> r;
#pragma unroll
  for (int j = 0; j < Raw<TYPE, 8>::kWords; ++j) r.w[j] = 0;
  const float f = power_of(s);
  f32x2 v[4];
  v[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, f, 0);
  v[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, f, 1);
  v[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, f, 2);
  v[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, f, 3);
#pragma unroll
  for (int j = 0; j < 8; ++j) r.put(j, to_bits<TYPE>(s == 255u ? __uint_as_float(0x7FC00000u) : v[j / 2][j % 2]));
  typename Elem<TYPE>::type* p = x + row * ld + col;
  const int n = q.cols - col < 8 ? (int)(q.cols - col) : 8;
  if (n == 8) {
#pragma unroll
    for (int i = 0; i < Raw<TYPE, 8>::kWords / 4; ++i) {
      Bytes16 b = {{r.w[4 * i], r.w[4 * i + 1], r.w[4 * i + 2], r.w[4 * i + 3]}};
      reinterpret_cast<Bytes16*>(p)[i] = b;
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (j >= n) continue;
      if constexpr (TYPE == EMB_TYPE_FP32)
        p[j] = __uint_as_float(r.w[j]);
      else
        p[j] = (uint16_t)(j % 2 ? r.w[j / 2] >> 16 : r.w[j / 2]);
    }
  }
}

// Plain codes to tiles and back: a thread takes one block.
__global__ __launch_bounds__(256) void k_pack(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                              Mx4 q, uint8_t* __restrict__ out, uint32_t first) {
  const uint32_t tile = (first + blockIdx.x) * 4 + (threadIdx.x >> 6), wide = (uint32_t)q.col_tiles;
  if (tile >= q.row_tiles * q.col_tiles) return;
  const int lane = threadIdx.x & 63;
  const int64_t rt = tile / wide, kt = tile % wide;
  const int64_t row = rt * kTileRows + (lane & 15), col = kt * kTileCols + (lane >> 4) * kBlock;
  const int64_t left = row < q.rows ? q.cols - col : 0;
  const int n = (int)(left < 0 ? 0 : left > kBlock ? kBlock : left);
  const int64_t pitch = (q.cols + 1) / 2, blocks = (q.cols + kBlock - 1) / kBlock;
  uint32_t w[4] = {0, 0, 0, 0};
  if (n == kBlock) {
    __builtin_memcpy(w, codes + row * pitch + col / 2, 16);
  } else {
#pragma unroll
    for (int i = 0; i < kBlock / 2; ++i) {
      if (2 * i >= n) continue;
      uint32_t b = codes[row * pitch + col / 2 + i];
      if (2 * i + 1 >= n) b &= 15u;
      w[i / 4] |= b << (8 * (i % 4));
    }
  }
  *reinterpret_cast<uint4*>(out + q.tile(rt, kt) + 16 * lane) = make_uint4(w[0], w[1], w[2], w[3]);
  store_scale(out, q, rt, kt, lane, n > 0 ? scales[row * blocks + col / kBlock] : 0u);
}

__global__ __launch_bounds__(256) void k_unpack(Mx4 q, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales,
                                                uint32_t first) {
  const uint32_t tile = (first + blockIdx.x) * 4 + (threadIdx.x >> 6), wide = (uint32_t)q.col_tiles;
  if (tile >= q.row_tiles * q.col_tiles) return;
  const int lane = threadIdx.x & 63;
  const int64_t rt = tile / wide, kt = tile % wide;
  const int64_t row = rt * kTileRows + (lane & 15), col = kt * kTileCols + (lane >> 4) * kBlock;
  const int64_t left = row < q.rows ? q.cols - col : 0;
  if (left <= 0) return;
  const int n = (int)(left > kBlock ? kBlock : left);
  const int64_t pitch = (q.cols + 1) / 2, blocks = (q.cols + kBlock - 1) / kBlock;
  const uint4 v = *reinterpret_cast<const uint4*>(q.base + q.tile(rt, kt) + 16 * lane);
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  if (n == kBlock) {
    __builtin_memcpy(codes + row * pitch + col / 2, w, 16);
  } else {
#pragma unroll
    for (int i = 0; i < kBlock / 2; ++i)
      if (2 * i < n) codes[row * pitch + col / 2 + i] = (uint8_t)(w[i / 4] >> (8 * (i % 4)));
  }
  scales[row * blocks + col / kBlock] = q.base[q.scale(rt, kt, lane)];
}

template <int TYPE, bool STOCHASTIC, bool BY_ROWS, bool BY_COLUMNS>
hipError_t quantize_along(const void* x, int64_t rows, int64_t cols, int64_t ld, void* by_rows, void* by_columns,
                          const Mx4Random& rnd, hipStream_t s) {
  using St = Stage<TYPE, BY_COLUMNS>;
  const int64_t workgroups = quantize_workgroups(rows, cols, BY_COLUMNS);
  return in_launches(workgroups, St::kThreads, [&](int64_t first, unsigned n) {
    k_quantize<TYPE, STOCHASTIC, BY_ROWS, BY_COLUMNS><<<n, St::kThreads, 0, s>>>(
        static_cast<const typename Elem<TYPE>::type*>(x), Mx4(by_rows, rows, cols), Mx4(by_columns, cols, rows), ld,
        static_cast<uint8_t*>(by_rows), static_cast<uint8_t*>(by_columns), rnd, (uint32_t)first, (uint32_t)workgroups);
    return hipGetLastError();
  });
}

template <int TYPE, bool STOCHASTIC>
hipError_t quantize_as(const void* x, int64_t rows, int64_t cols, int64_t ld, void* by_rows, void* by_columns,
                       const Mx4Random& rnd, hipStream_t s) {
  if (!by_columns) return quantize_along<TYPE, STOCHASTIC, true, false>(x, rows, cols, ld, by_rows, by_columns, rnd, s);
  if (!by_rows) return quantize_along<TYPE, STOCHASTIC, false, true>(x, rows, cols, ld, by_rows, by_columns, rnd, s);
  return quantize_along<TYPE, STOCHASTIC, true, true>(x, rows, cols, ld, by_rows, by_columns, rnd, s);
}

}  // namespace

hipError_t launch_quantize(const void* x, int type, int64_t rows, int64_t cols, int64_t ld, void* by_rows,
                           void* by_columns, int rounding, uint64_t seed, uint32_t step, Mx4Stream stream, hipStream_t s) {
  const Mx4Random rnd = {(uint32_t)seed, (uint32_t)(seed >> 32), step, stream};
  const bool sr = rounding == EMB_ROUND_STOCHASTIC;
  switch (type) {
    case EMB_TYPE_FP32:
      return sr ? quantize_as<EMB_TYPE_FP32, true>(x, rows, cols, ld, by_rows, by_columns, rnd, s)
                : quantize_as<EMB_TYPE_FP32, false>(x, rows, cols, ld, by_rows, by_columns, rnd, s);
    case EMB_TYPE_BF16:
      return sr ? quantize_as<EMB_TYPE_BF16, true>(x, rows, cols, ld, by_rows, by_columns, rnd, s)
                : quantize_as<EMB_TYPE_BF16, false>(x, rows, cols, ld, by_rows, by_columns, rnd, s);
    default:
      return sr ? quantize_as<EMB_TYPE_FP16, true>(x, rows, cols, ld, by_rows, by_columns, rnd, s)
                : quantize_as<EMB_TYPE_FP16, false>(x, rows, cols, ld, by_rows, by_columns, rnd, s);
  }
}

hipError_t launch_dequantize(const void* qv, int64_t rows, int64_t cols, void* x, int type, int64_t ld, hipStream_t s) {
  const Mx4 q(qv, rows, cols);
  return in_launches(q.row_tiles * q.col_tiles, 256, [&](int64_t first, unsigned n) {
    const uint32_t f = (uint32_t)first;
    if (type == EMB_TYPE_FP32)
      k_dequantize<EMB_TYPE_FP32><<<n, 256, 0, s>>>(q, static_cast<float*>(x), ld, f);
    else if (type == EMB_TYPE_BF16)
      k_dequantize<EMB_TYPE_BF16><<<n, 256, 0, s>>>(q, static_cast<uint16_t*>(x), ld, f);
    else
      k_dequantize<EMB_TYPE_FP16><<<n, 256, 0, s>>>(q, static_cast<uint16_t*>(x), ld, f);
    return hipGetLastError();
  });
}

hipError_t launch_pack(const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t cols, void* qv,
                       hipStream_t s) {
  const Mx4 q(qv, rows, cols);
  return in_launches(ceil_div(q.row_tiles * q.col_tiles, 4), 256, [&](int64_t first, unsigned n) {
    k_pack<<<n, 256, 0, s>>>(codes, scales, q, static_cast<uint8_t*>(qv), (uint32_t)first);
    return hipGetLastError();
  });
}

hipError_t launch_unpack(const void* qv, int64_t rows, int64_t cols, uint8_t* codes, uint8_t* scales, hipStream_t s) {
  const Mx4 q(qv, rows, cols);
  return in_launches(ceil_div(q.row_tiles * q.col_tiles, 4), 256, [&](int64_t first, unsigned n) {
    k_unpack<<<n, 256, 0, s>>>(q, codes, scales, (uint32_t)first);
    return hipGetLastError();
  });
}

}  // namespace embd
