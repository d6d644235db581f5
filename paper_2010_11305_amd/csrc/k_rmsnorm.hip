// The root-mean-square norm of rows with the residual's addition, its output in 8 bits, and its gradients.
//
// Rows of at most 4096 pieces of 16 bytes (and 16384 columns) stay in the registers of a team of threads, which reads and
// writes every value once; wider ones take a workgroup a row that goes over it as often as it has to, a thread
// always over the same 8 columns at a time, so that what it wrote in one pass it reads in the next.
//
// Memory bounds them.  By the kernel trace, 16384 x 12800 BF16 with a residual (1.68 GB each way): forward 276 us (6.1 TB/s),
// gradients 330 (5.1) and 7.6 to join 512 parts of the gain's.  4096 x 8192 to 8 bits, with a residual, 47.4 us (5.0 TB/s), the codes
// to BF16 16.8 (6.0).  What little there is takes the launch and two or three trips to memory: 2048 x 416 FP32 3.7, 5.5 and
// 2.7 us, one row of 12800 to 8 bits 4.7.  Rows that no registers hold are read two or three times: us a call with a residual in a graph,
// forward and gradients, 8192 x 25600 BF16 409 (4.1 TB/s) and 716 (2.3), 8192 x 16384, in registers, 191 (5.6) and 217 (5.0).  Rows of less
// than a piece take a workgroup each all the same: 2,000,000 x 3 2.7 ms.
// Squares are summed in FP64, which costs nothing there: no row of FP32 overflows or vanishes.  So is the mean that the
// gradients subtract: with its sum in FP32, terms of 2^123 passed the type's end from 32 columns on, and 16384 x 12800 took 8 us
// less of 331, 1000 x 1029 FP16 as long, 20000 x 64, where its shuffles count, 12.1 us instead of 13.6.
#include "dense_device.h"

namespace embd {

namespace {

constexpr int kThreads = 256;
constexpr int kPer = 8;
template <int T>
constexpr int kPiece = 16 / Elem<T>::kBytes;   // values of 16 bytes

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

// N codes of 8-bit rows at any address.
template <int N>
struct __attribute__((packed, aligned(1))) Codes {
  uint32_t w[N / 4];
};
using Codes8 = Codes<kPer>;

// What 127 stands for, over 127: not below the normal numbers, so that its reciprocal is finite.
__device__ __forceinline__ float scale8(uint32_t amax) {
  return fmaxf(__uint_as_float(amax) / 127.0f, 0x1p-126f);
}

// N values to codes.  |v| <= 127.00003 scale, so nothing passes 127.
template <int N>
__device__ __forceinline__ Codes<N> codes_of(const float (&v)[N], float per) {
  Codes<N> c = {};
#pragma unroll
  for (int j = 0; j < N; ++j) c.w[j / 4] |= ((uint32_t)(int)rintf(v[j] * per) & 0xFFu) << (8 * (j % 4));
  return c;
}

template <int N>
__device__ __forceinline__ void store_codes(int8_t* p, int n, const Codes<N>& c) {
  if (n == N) {
    *reinterpret_cast<Codes<N>*>(p) = c;
    return;
  }
#pragma unroll
  for (int j = 0; j < N; ++j)
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

template <int TEAM>
constexpr int kGroup = TEAM < kThreads ? kThreads : TEAM;   // threads of a workgroup of such teams

// Piece k of CH of a thread t: 16 bytes from column c on.  The last piece of a row is moved back to end with it, so that every
// access is of 16 bytes; its first `skip` values are another thread's too, which computes and writes the same.  There are
// more than TEAM CH / 2 pieces unless CH is 1, so the first half of a thread's are whole.  (1000 x 1029 FP16 with a part of a
// piece read value by value: 8.0 us, so 4.8.)
struct Piece {
  int c, skip;
  bool in;
};
template <int T, int TEAM, int CH>
__device__ __forceinline__ Piece piece_of(int64_t cols, int k, int t) {
  const int c = (k * TEAM + t) * kPiece<T>, last = (int)cols - kPiece<T>;
  if (k < CH / 2) return {c, 0, true};
  return {c < last ? c : last, c < last ? 0 : c - last, c < (int)cols};
}

template <int T>
__device__ __forceinline__ Raw<T, kPiece<T>> load_piece(const typename Elem<T>::type* p, const Piece& at) {
  Raw<T, kPiece<T>> r = {};
  if (at.in) {
    const Bytes16 b = *reinterpret_cast<const Bytes16*>(p + at.c);
#pragma unroll
    for (int i = 0; i < 4; ++i) r.w[i] = b.w[i];
  }
  return r;
}
template <int T>
__device__ __forceinline__ void store_piece(typename Elem<T>::type* p, const Piece& at, const Raw<T, kPiece<T>>& r) {
  if (at.in) *reinterpret_cast<Bytes16*>(p + at.c) = Bytes16{{r.w[0], r.w[1], r.w[2], r.w[3]}};
}

// A piece of the gain (which is FP32, or of type T).
template <int T>
__device__ __forceinline__ void gain_piece(const void* gain, bool wide, const Piece& at, float (&g)[kPiece<T>]) {
  constexpr int N = kPiece<T>;
  if (!gain) {
#pragma unroll
    for (int j = 0; j < N; ++j) g[j] = 1.0f;
  } else if (T == EMB_TYPE_FP32 || wide) {
#pragma unroll
    for (int q = 0; q < N; q += 4) {
      const Raw<EMB_TYPE_FP32, 4> r = load_piece<EMB_TYPE_FP32>(static_cast<const float*>(gain) + q, at);
#pragma unroll
      for (int j = 0; j < 4; ++j) g[q + j] = r.get(j);
    }
  } else if constexpr (T != EMB_TYPE_FP32) {
    const Raw<T, N> r = load_piece<T>(static_cast<const uint16_t*>(gain), at);
#pragma unroll
    for (int j = 0; j < N; ++j) g[j] = r.get(j);
  }
}

// A row in the registers of a team, CH pieces a thread.
template <int T, int TEAM, int CH, bool BITS8>
__global__ __launch_bounds__(kGroup<TEAM>) void k_norm_row(NormForward a, bool gain_wide, int64_t first) {
  constexpr int N = kPiece<T>;
  __shared__ double sums[TEAM / 64];
  __shared__ uint32_t tops[TEAM / 64];
  const int t = threadIdx.x % TEAM;
  const int64_t row = (first + blockIdx.x) * (kGroup<TEAM> / TEAM) + threadIdx.x / TEAM;
  if (row >= a.rows) return;   // of a team that is a wave: nothing meets
  Piece at[CH];
  Raw<T, N> h[CH];
  float v[CH][N];   // the gain, then y
#pragma unroll
  for (int k = 0; k < CH; ++k) {
    at[k] = piece_of<T, TEAM, CH>(a.cols, k, t);
    h[k] = load_piece<T>(row_of<T>(a.x, row), at[k]);
  }
  if (a.residual.p) {
    Raw<T, N> r[CH];
#pragma unroll
    for (int k = 0; k < CH; ++k) r[k] = load_piece<T>(row_of<T>(a.residual, row), at[k]);
#pragma unroll
    for (int k = 0; k < CH; ++k)
#pragma unroll
      for (int j = 0; j < N; ++j) h[k].put(j, to_bits<T>(h[k].get(j) + r[k].get(j)));
  }
#pragma unroll
  for (int k = 0; k < CH; ++k) gain_piece<T>(a.gain, gain_wide, at[k], v[k]);
  double squares = 0.0;
#pragma unroll
  for (int k = 0; k < CH; ++k)
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const double x = k < CH / 2 || j >= at[k].skip ? (double)h[k].get(j) : 0.0;
      squares = fma(x, x, squares);
    }
  const float inverse = inverse_of(block_sum<double, TEAM>(squares, sums), a.cols, a.eps);
  // only now, as it may lie over x and pieces overlap
  if (a.sum.p) {
#pragma unroll
    for (int k = 0; k < CH; ++k) store_piece<T>(row_of<T>(a.sum, row), at[k], h[k]);
  }
  if (a.inverse && t == 0) a.inverse[row] = inverse;
#pragma unroll
  for (int k = 0; k < CH; ++k)
#pragma unroll
    for (int j = 0; j < N; ++j) v[k][j] = h[k].get(j) * inverse * v[k][j];
  if constexpr (!BITS8) {
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      Raw<T, N> y = {};
#pragma unroll
      for (int j = 0; j < N; ++j) y.put(j, to_bits<T>(v[k][j]));
      store_piece<T>(row_of<T>(a.y, row), at[k], y);
    }
  } else {
    uint32_t top = 0;
#pragma unroll
    for (int k = 0; k < CH; ++k)
#pragma unroll
      for (int j = 0; j < N; ++j) top = max(top, __float_as_uint(v[k][j]) & 0x7FFFFFFFu);
    top = block_max<TEAM>(top, tops);
    const bool fine = top < 0x7F800000u;
    const float scale = scale8(top), per = fine ? 1.0f / scale : 0.0f;
    if (t == 0) a.scales[row] = fine ? scale : __uint_as_float(0x7FC00000u);
    int8_t* out = static_cast<int8_t*>(const_cast<void*>(a.y.p)) + row * a.y.ld;
#pragma unroll
    for (int k = 0; k < CH; ++k)
      if (at[k].in) *reinterpret_cast<Codes<N>*>(out + at[k].c) = fine ? codes_of(v[k], per) : Codes<N>{};
  }
}

template <int T>
__device__ __forceinline__ void store_gain(const NormBackward& a, bool gain_wide, const Piece& at, const float (&v)[kPiece<T>]) {
  constexpr int N = kPiece<T>;
  if (T == EMB_TYPE_FP32 || gain_wide) {
#pragma unroll
    for (int q = 0; q < N; q += 4) {
      Raw<EMB_TYPE_FP32, 4> r;
#pragma unroll
      for (int j = 0; j < 4; ++j) r.w[j] = __float_as_uint(v[q + j]);
      store_piece<EMB_TYPE_FP32>(static_cast<float*>(a.dgain) + q, at, r);
    }
  } else if constexpr (T != EMB_TYPE_FP32) {
    Raw<T, N> r = {};
#pragma unroll
    for (int j = 0; j < N; ++j) r.put(j, to_bits<T>(v[j]));
    store_piece<T>(static_cast<uint16_t*>(a.dgain), at, r);
  }
}

// Rows first, first + step, .. in the registers of a team.  SUMS: their part of the gain's gradient goes to `sum`.
template <int T, int TEAM, int CH, bool SUMS>
__device__ __forceinline__ void gradient_rows(const NormBackward& a, bool gain_wide, int64_t first, int64_t step, int t, double* sums,
                                              Piece (&at)[CH], float (&sum)[SUMS ? CH : 1][kPiece<T>]) {
  constexpr int N = kPiece<T>;
  float g[CH][N];
#pragma unroll
  for (int k = 0; k < CH; ++k) {
    at[k] = piece_of<T, TEAM, CH>(a.cols, k, t);
    gain_piece<T>(a.gain, gain_wide, at[k], g[k]);
    if constexpr (SUMS)
#pragma unroll
      for (int j = 0; j < N; ++j) sum[k][j] = 0.0f;
  }
  const double cols = (double)a.cols;
  for (int64_t row = first; row < a.rows; row += step) {
    Raw<T, N> d[CH], h[CH], s[CH] = {};
#pragma unroll
    for (int k = 0; k < CH; ++k) d[k] = load_piece<T>(row_of<T>(a.dy, row), at[k]);
#pragma unroll
    for (int k = 0; k < CH; ++k) h[k] = load_piece<T>(row_of<T>(a.h, row), at[k]);
    if (a.dsum.p) {
#pragma unroll
      for (int k = 0; k < CH; ++k) s[k] = load_piece<T>(row_of<T>(a.dsum, row), at[k]);
    }
    const float inverse = a.inverse[row];
    double along = 0.0;
#pragma unroll
    for (int k = 0; k < CH; ++k)
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float u = h[k].get(j) * inverse, dj = d[k].get(j);
        along = fma((double)(k < CH / 2 || j >= at[k].skip ? dj * g[k][j] : 0.0f), (double)u, along);
        if constexpr (SUMS) sum[k][j] = fmaf(dj, u, sum[k][j]);
      }
    const float mean = (float)(block_sum<double, TEAM>(along, sums) / cols);
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      Raw<T, N> out = {};
#pragma unroll
      for (int j = 0; j < N; ++j)
        out.put(j, to_bits<T>((d[k].get(j) * g[k][j] - h[k].get(j) * inverse * mean) * inverse + s[k].get(j)));
      store_piece<T>(row_of<T>(a.dx, row), at[k], out);
    }
  }
}

// The gradients: a workgroup takes every blocks-th row (or group of rows, a team each), keeps its columns' part of the gain's
// gradient in registers and leaves it in `partial`.
template <int T, int TEAM, int CH>
__global__ __launch_bounds__(kGroup<TEAM>) void k_norm_gradients(NormBackward a, bool gain_wide, int64_t first, int64_t blocks) {
  constexpr int N = kPiece<T>, kTeams = kGroup<TEAM> / TEAM;
  __shared__ double sums[TEAM / 64];
  __shared__ float meet[kTeams > 1 ? kTeams - 1 : 1][kTeams > 1 ? CH * N * TEAM : 1];
  const int t = threadIdx.x % TEAM, team = threadIdx.x / TEAM;
  const int64_t block = first + blockIdx.x;
  Piece at[CH];
  float sum[CH][N];
  gradient_rows<T, TEAM, CH, true>(a, gain_wide, block * kTeams + team, blocks * kTeams, t, sums, at, sum);
  if (!a.dgain) return;
  if constexpr (kTeams > 1) {
    if (team) {
#pragma unroll
      for (int k = 0; k < CH; ++k)
#pragma unroll
        for (int j = 0; j < N; ++j) meet[team - 1][(k * N + j) * TEAM + t] = sum[k][j];
    }
    __syncthreads();
    if (team) return;
#pragma unroll
    for (int k = 0; k < CH; ++k)
#pragma unroll
      for (int j = 0; j < N; ++j)
        for (int o = 0; o < kTeams - 1; ++o) sum[k][j] += meet[o][(k * N + j) * TEAM + t];
  }
  float* out = a.partial + block * a.cols;
#pragma unroll
  for (int k = 0; k < CH; ++k)
#pragma unroll
    for (int q = 0; q < N; q += 4) {
      Raw<EMB_TYPE_FP32, 4> r;
#pragma unroll
      for (int j = 0; j < 4; ++j) r.w[j] = __float_as_uint(sum[k][q + j]);
      store_piece<EMB_TYPE_FP32>(out + q, at[k], r);
    }
}

// Both gradients of few rows in one launch, without parts that a second one joins: the first `columns` workgroups each sum
// four pieces of the gain's gradient over all rows, the others take the rows.  dy and h are read twice, the second time
// from a cache.  Measured against k_norm_gradients and k_norm_gain_join, us in a graph: 256 x 416 in FP32 3.1 (5.9),
// 256 x 8192 in BF16 5.0 (11.4), 1000 x 2048 in BF16 6.7 (9.9), 1000 x 1029 in FP16 7.1 (9.9); not taken beyond kOnceRows
// and kOnceBytes: 2048 x 416 in FP32 8.2 (6.8), 4000 x 512 in BF16 12.1 (9.5), 1000 x 2048 in FP32 11.1 (11.2).  A dx that lies
// over dy or h waits for the columns: two launches of the same kernel, so that the gain's gradient has the same bits wherever dx
// lies.  That costs more than both: 256 x 416 5.9, 256 x 8192 11.0, 1000 x 1029 in FP16 13.1, 1000 x 2048 in BF16 14.5.
constexpr int kOncePieces = 4;
template <int T, int TEAM, int CH>
__global__ __launch_bounds__(kGroup<TEAM>) void k_norm_gradients_once(NormBackward a, bool gain_wide, uint32_t columns) {
  constexpr int N = kPiece<T>, kTeams = kGroup<TEAM> / TEAM, kRows = kGroup<TEAM> / kOncePieces, kWaves = kGroup<TEAM> / 64;
  __shared__ double sums[TEAM / 64];
  __shared__ float meet[kWaves][kOncePieces][N];
  if (blockIdx.x >= columns) {
    const int t = threadIdx.x % TEAM, team = threadIdx.x / TEAM;
    Piece at[CH];
    float none[1][N];
    gradient_rows<T, TEAM, CH, false>(a, gain_wide, (int64_t)(blockIdx.x - columns) * kTeams + team, (int64_t)(gridDim.x - columns) * kTeams, t,
                                      sums, at, none);
    return;
  }
  const int p = threadIdx.x % kOncePieces, c = (int)(blockIdx.x * kOncePieces + p) * N, last = (int)a.cols - N;
  const Piece at = {c < last ? c : last, 0, c < (int)a.cols};
  float sum[N] = {};
#pragma unroll 4
  for (int64_t row = threadIdx.x / kOncePieces; row < a.rows; row += kRows) {
    const Raw<T, N> d = load_piece<T>(row_of<T>(a.dy, row), at), h = load_piece<T>(row_of<T>(a.h, row), at);
    const float inverse = a.inverse[row];
#pragma unroll
    for (int j = 0; j < N; ++j) sum[j] = fmaf(d.get(j), h.get(j) * inverse, sum[j]);
  }
#pragma unroll
  for (int j = 0; j < N; ++j) {
#pragma unroll
    for (int m = kOncePieces; m < 64; m *= 2) sum[j] += __shfl_xor(sum[j], m);
    if (threadIdx.x % 64 < kOncePieces) meet[threadIdx.x / 64][p][j] = sum[j];
  }
  __syncthreads();
  if (threadIdx.x >= kOncePieces) return;
#pragma unroll
  for (int j = 0; j < N; ++j)
    for (int w = 1; w < kWaves; ++w) sum[j] += meet[w][p][j];
  store_gain<T>(a, gain_wide, at, sum);
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
      store_codes(out + c, n, fine ? codes_of(v, per) : Codes8{{0, 0}});
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
      if (j < n) along = fma((double)dn[j], (double)u[j], along);
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

// The slabs' parts together: 32 columns a workgroup, 32 threads over the slabs of each.
constexpr int kJoinCols = 32, kJoinThreads = 1024, kJoinWays = kJoinThreads / kJoinCols;
template <int GT>
__global__ __launch_bounds__(kJoinThreads) void k_norm_gain_join(const float* __restrict__ partial, int64_t slabs, int64_t cols,
                                                                 typename Elem<GT>::type* __restrict__ out, int64_t first) {
  __shared__ double sums[kJoinWays / 2][kJoinCols];
  const int col = threadIdx.x % kJoinCols, way = threadIdx.x / kJoinCols;
  const int64_t c = (first + blockIdx.x) * kJoinCols + col;
  double sum = 0.0;
  if (c < cols) {
    const float* p = partial + c;
    int64_t s = way;
    for (; s + 7 * kJoinWays < slabs; s += 8 * kJoinWays) {
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = p[(s + i * kJoinWays) * cols];
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += (double)v[i];
    }
    for (; s < slabs; s += kJoinWays) sum += (double)p[s * cols];
  }
  // a wave holds two ways of its columns; then the first wave adds up the waves
  sum += __shfl_xor(sum, 32);
  if (threadIdx.x % 64 < 32) sums[threadIdx.x / 64][col] = sum;
  __syncthreads();
  if (threadIdx.x >= 64) return;
  sum = 0.0;
#pragma unroll
  for (int w = 0; w < kJoinWays / 4; ++w) sum += sums[way * (kJoinWays / 4) + w][col];
  sum += __shfl_xor(sum, 32);
  if (way || c >= cols) return;
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

int64_t pieces_of(int64_t cols, int type) { return ceil_div(cols, type == EMB_TYPE_FP32 ? 4 : 8); }

// Calls f<TEAM, CH> for a row of so many pieces (more than 2048 of FP32 alone).
template <int T, class F>
hipError_t by_pieces(int64_t pieces, F f) {
  if (pieces <= 64) return f.template operator()<64, 1>();
  if (pieces <= 128) return f.template operator()<64, 2>();
  if (pieces <= 256) return f.template operator()<64, 4>();
  if (pieces <= 512) return f.template operator()<256, 2>();
  if (pieces <= 1024) return f.template operator()<256, 4>();
  if constexpr (T == EMB_TYPE_FP32)
    if (pieces > 2048) return f.template operator()<512, 8>();
  return f.template operator()<512, 4>();
}
// The same for so few rows that each may have a CU to itself (48 x 8192 BF16 to 8 bits: 5.4 us, with 256 threads a row 6.9).
template <int T, class F>
hipError_t by_pieces_of_few(int64_t pieces, F f) {
  if (pieces <= 256) return by_pieces<T>(pieces, f);
  if (pieces <= 512) return f.template operator()<512, 1>();
  if (pieces <= 1024) return f.template operator()<1024, 1>();
  if constexpr (T == EMB_TYPE_FP32)
    if (pieces > 2048) return f.template operator()<1024, 4>();
  return f.template operator()<1024, 2>();
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

template <int T>
hipError_t norm_rows_as(const NormForward& a, bool gain_wide, hipStream_t s) {
  const auto launch = [&]<int TEAM, int CH>() {
    return in_launches(ceil_div(a.rows, kGroup<TEAM> / TEAM), kGroup<TEAM>, [&](int64_t first, unsigned n) {
      if (a.scales)
        k_norm_row<T, TEAM, CH, true><<<n, kGroup<TEAM>, 0, s>>>(a, gain_wide, first);
      else
        k_norm_row<T, TEAM, CH, false><<<n, kGroup<TEAM>, 0, s>>>(a, gain_wide, first);
      return hipGetLastError();
    });
  };
  return a.rows <= 256 ? by_pieces_of_few<T>(pieces_of(a.cols, T), launch) : by_pieces<T>(pieces_of(a.cols, T), launch);
}

hipError_t join(const NormBackward& a, int64_t slabs, int type, hipStream_t s) {
  return in_launches(ceil_div(a.cols, kJoinCols), kJoinThreads, [&](int64_t first, unsigned n) {
#define EMBD_JOIN(GT) \
  k_norm_gain_join<GT><<<n, kJoinThreads, 0, s>>>(a.partial, slabs, a.cols, static_cast<typename Elem<GT>::type*>(a.dgain), first)
    if (type == EMB_TYPE_FP32)
      EMBD_JOIN(EMB_TYPE_FP32);
    else if (type == EMB_TYPE_BF16)
      EMBD_JOIN(EMB_TYPE_BF16);
    else
      EMBD_JOIN(EMB_TYPE_FP16);
#undef EMBD_JOIN
    return hipGetLastError();
  });
}

template <int T, int GT>
hipError_t backward_as(const NormBackward& a, int64_t slabs, hipStream_t s) {
  hipError_t e = hipSuccess;
  if (a.dgain)
    e = in_launches(slabs * ceil_div(a.cols, kThreads), kThreads, [&](int64_t first, unsigned n) {
      k_norm_gain<T><<<n, kThreads, 0, s>>>(a, first);
      return hipGetLastError();
    });
  if (e != hipSuccess) return e;
  return in_launches(a.rows, kThreads, [&](int64_t first, unsigned n) {
    k_norm_dx<T, GT><<<n, kThreads, 0, s>>>(a, first);
    return hipGetLastError();
  });
}

constexpr int64_t kOnceRows = 1024, kOnceBytes = 4 << 20;
static_assert(16 * 16384 * 4 <= kOnceBytes, "rows of one workgroup have no other way to the gain's gradient");
bool once(const NormBackward& a, int type) {
  return a.dgain && a.rows && a.rows <= kOnceRows && a.rows * a.cols * (type == EMB_TYPE_FP32 ? 4 : 2) <= kOnceBytes;
}

template <int T>
hipError_t backward_rows_as(const NormBackward& a, bool gain_wide, int64_t slabs, hipStream_t s) {
  return by_pieces<T>(pieces_of(a.cols, T), [&]<int TEAM, int CH>() {
    if (once(a, T)) {
      const uint32_t columns = (uint32_t)ceil_div(pieces_of(a.cols, T), kOncePieces);
      const uint32_t rows = (uint32_t)ceil_div(a.rows, kGroup<TEAM> / TEAM);
      const bool over = a.dx.p == a.dy.p || a.dx.p == a.h.p;
      if (over) k_norm_gradients_once<T, TEAM, CH><<<columns, kGroup<TEAM>, 0, s>>>(a, gain_wide, columns);
      const uint32_t left = over ? 0 : columns;
      k_norm_gradients_once<T, TEAM, CH><<<left + rows, kGroup<TEAM>, 0, s>>>(a, gain_wide, left);
      return hipGetLastError();
    }
    return in_launches(slabs, kGroup<TEAM>, [&](int64_t first, unsigned n) {
      k_norm_gradients<T, TEAM, CH><<<n, kGroup<TEAM>, 0, s>>>(a, gain_wide, first, slabs);
      return hipGetLastError();
    });
  });
}

}  // namespace

// A row that stays in registers has a whole piece and at most 4096 of them, and 16384 columns.
bool norm_in_registers(int64_t cols, int type) { return cols >= (type == EMB_TYPE_FP32 ? 4 : 8) && cols <= 16384; }

// Workgroups that share the rows, each with a part of the gain's gradient: two to a CU, but no more than have two rows a
// team, and none with more than kNormSlabRows a team.  One, which needs no part, for up to four rows a team: their gain's
// gradient is always of the single launch.
int64_t norm_slabs(int64_t rows, int64_t cols, int type) {
  if (!norm_in_registers(cols, type)) return ceil_div(rows, kNormSlabRows);
  const int64_t teams = pieces_of(cols, type) <= 256 ? 4 : 1;
  if (rows && rows <= 4 * teams) return 1;
  const int64_t most = ceil_div(rows, 2 * teams), least = ceil_div(rows, kNormSlabRows * teams);
  return most < 512 ? most : least > 512 ? least : 512;
}

hipError_t launch_norm(const NormForward& a, int type, bool gain_wide, hipStream_t s) {
  if (norm_in_registers(a.cols, type)) {
    if (type == EMB_TYPE_FP32) return norm_rows_as<EMB_TYPE_FP32>(a, true, s);
    if (type == EMB_TYPE_BF16) return norm_rows_as<EMB_TYPE_BF16>(a, gain_wide, s);
    return norm_rows_as<EMB_TYPE_FP16>(a, gain_wide, s);
  }
  if (type == EMB_TYPE_FP32) return norm_as<EMB_TYPE_FP32, EMB_TYPE_FP32>(a, s);
  if (type == EMB_TYPE_BF16) return gain_wide ? norm_as<EMB_TYPE_BF16, EMB_TYPE_FP32>(a, s) : norm_as<EMB_TYPE_BF16, EMB_TYPE_BF16>(a, s);
  return gain_wide ? norm_as<EMB_TYPE_FP16, EMB_TYPE_FP32>(a, s) : norm_as<EMB_TYPE_FP16, EMB_TYPE_FP16>(a, s);
}

hipError_t launch_norm_backward(const NormBackward& a, int type, bool gain_wide, hipStream_t s) {
  const int64_t slabs = norm_slabs(a.rows, a.cols, type);
  hipError_t e = hipSuccess;
  if (a.rows) {
    if (norm_in_registers(a.cols, type))
      e = type == EMB_TYPE_FP32   ? backward_rows_as<EMB_TYPE_FP32>(a, true, slabs, s)
          : type == EMB_TYPE_BF16 ? backward_rows_as<EMB_TYPE_BF16>(a, gain_wide, slabs, s)
                                  : backward_rows_as<EMB_TYPE_FP16>(a, gain_wide, slabs, s);
    else if (type == EMB_TYPE_FP32)
      e = backward_as<EMB_TYPE_FP32, EMB_TYPE_FP32>(a, slabs, s);
    else if (type == EMB_TYPE_BF16)
      e = gain_wide ? backward_as<EMB_TYPE_BF16, EMB_TYPE_FP32>(a, slabs, s) : backward_as<EMB_TYPE_BF16, EMB_TYPE_BF16>(a, slabs, s);
    else
      e = gain_wide ? backward_as<EMB_TYPE_FP16, EMB_TYPE_FP32>(a, slabs, s) : backward_as<EMB_TYPE_FP16, EMB_TYPE_FP16>(a, slabs, s);
  }
  const bool joined = norm_in_registers(a.cols, type) && once(a, type);
  return e == hipSuccess && a.dgain && !joined ? join(a, slabs, gain_wide ? EMB_TYPE_FP32 : type, s) : e;
}

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
