// Internal declarations of the dense operators (include/emb_dense.h): the layouts of MX4 and W4
// matrices, shared by host and device, and the launchers.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "dense_launch.h"
#include "emb_dense.h"

namespace embd {

constexpr int kBlock = 32;       // values that share a scale
constexpr int kTileRows = 16;    // a tile: the operand of one 16x16x128 matrix instruction,
constexpr int kTileCols = 128;   // lane 16 b + r holding block b of row r
constexpr int kTileBytes = 1024;
constexpr int kScaleTiles = 4;   // column tiles whose scale bytes lie in one dword per lane
constexpr int kScaleBytes = 256;

// An MX4 matrix in its buffer.
struct Mx4 {
  const uint8_t* base;
  int64_t rows, cols;
  int64_t row_tiles, col_tiles, col_groups;
  int64_t scale_offset;

  __host__ __device__ Mx4(const void* b, int64_t r, int64_t c)
      : base(static_cast<const uint8_t*>(b)),
        rows(r),
        cols(c),
        row_tiles((r + kTileRows - 1) / kTileRows),
        col_tiles((c + kTileCols - 1) / kTileCols),
        col_groups((col_tiles + kScaleTiles - 1) / kScaleTiles),
        scale_offset(row_tiles * col_tiles * kTileBytes) {}

  __host__ __device__ int64_t tile(int64_t rt, int64_t kt) const { return (rt * col_tiles + kt) * kTileBytes; }
  // the scale byte of block b of row r in tile (rt, kt), lane = 16 b + r
  __host__ __device__ int64_t scale(int64_t rt, int64_t kt, int lane) const {
    return scale_offset + (rt * col_groups + kt / kScaleTiles) * kScaleBytes + 4 * lane + kt % kScaleTiles;
  }
  __host__ __device__ int64_t bytes() const { return scale_offset + row_tiles * col_groups * kScaleBytes; }
};

constexpr int64_t kMaxDim = (int64_t)1 << 31;  // rows and columns stay below it
constexpr int64_t kMaxDepth = (int64_t)1 << 24;  // columns of a product's operands: offsets inside 8 row tiles fit 31 bits
// no device memory holds a matrix of more bytes; the tile counts of smaller ones fit 31 bits
constexpr double kMaxBytes = (double)((int64_t)1 << 40);

// Last word of the random counter of a matrix quantised by rows; by columns it is the next one.
enum Mx4Stream : uint32_t { kStreamMatrix = 0, kStreamTrainRows = 2 };

hipError_t launch_quantize(const void* x, int type, int64_t rows, int64_t cols, int64_t ld, void* by_rows,
                           void* by_columns, int rounding, uint64_t seed, uint32_t step, Mx4Stream stream, hipStream_t s);
hipError_t launch_dequantize(const void* q, int64_t rows, int64_t cols, void* x, int type, int64_t ld, hipStream_t s);
hipError_t launch_pack(const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t cols, void* q, hipStream_t s);
hipError_t launch_unpack(const void* q, int64_t rows, int64_t cols, uint8_t* codes, uint8_t* scales, hipStream_t s);

hipError_t launch_matmul(const void* a, const void* b, int64_t m, int64_t n, int64_t k, void* c, int type, int64_t ldc,
                         hipStream_t s);
// c1 = a1 b1^T and c2 = a2 b2^T (an empty one is left out), in one launch where both are small
hipError_t launch_two_products(const void* a1, const void* b1, int64_t m1, int64_t n1, int64_t k1, void* c1, int type1,
                               int64_t ldc1, const void* a2, const void* b2, int64_t m2, int64_t n2, int64_t k2, void* c2,
                               int type2, int64_t ldc2, hipStream_t s);
size_t linear_workspace(int64_t m, int64_t n, int64_t k);
hipError_t launch_linear(const void* x, int type, int64_t m, int64_t k, int64_t ldx, const void* w, int64_t n, void* y,
                         int64_t ldy, void* workspace, hipStream_t s);

// ---- AdamW -----------------------------------------------------------------------------------
constexpr int kAdamThreads = 256;
constexpr int kAdamPer = 8;          // elements of a thread
constexpr int kAdamChunk = kAdamThreads * kAdamPer;   // elements of a tensor that one workgroup updates
constexpr int kAdamTensors = 240;    // tensors whose pointers one launch carries (kernel arguments hold 4 KB)

struct AdamTensor {
  int64_t base;    // first element in the state
  int64_t size;
  double decay;    // weight decay
};

struct AdamPart {  // one workgroup's work
  uint32_t tensor;
  uint32_t chunk;
};

struct AdamConst {
  float beta1, beta2, rest1, rest2;  // rest = 1 - beta
  float inv_root;                    // 1 / sqrt(1 - beta2^t)
  float eps;
  float rate;                        // lr / (1 - beta1^t)
  double lr;
  uint32_t k0, k1, t;                // random stream
};

struct AdamDev {
  const AdamTensor* tensors;
  const AdamPart* parts;
  uint8_t* first;
  uint8_t* second;
  uint8_t* first_scale;
  uint8_t* second_scale;
};

struct AdamPointers {
  void* p[kAdamTensors];
  const void* g[kAdamTensors];
};

// Parts [part0, part0 + parts) of tensors [first, first + kAdamTensors).
hipError_t launch_adamw(const AdamDev& d, const AdamPointers& ptr, uint32_t first, int64_t part0, int64_t parts,
                        const AdamConst& c, const float* grad_scale, int param_type, int grad_type, int state_bits,
                        int rounding, hipStream_t s);

// ---- Root-mean-square norm -------------------------------------------------------------------
// A matrix argument: rows of `ld` elements.
struct Rows {
  const void* p;
  int64_t ld;
};

constexpr int64_t kNormSlabRows = 256;   // rows whose part of the gain's gradient is summed in FP32

struct NormForward {
  Rows x, residual, sum, y;   // y: full-precision rows, or codes with `scales`
  int64_t rows, cols;
  const void* gain;
  float* inverse;
  float* scales;
  float eps;
};

struct NormBackward {
  Rows dy, h, dsum, dx;
  int64_t rows, cols;
  const float* inverse;
  const void* gain;
  void* dgain;
  float* partial;   // [slabs][cols]
};

// gain_wide: the gain is FP32 (also where it is NULL), else of `type`.
hipError_t launch_norm(const NormForward& a, int type, bool gain_wide, hipStream_t s);
// Parts of the gain's gradient in the workspace; one of rows in registers goes without.
int64_t norm_slabs(int64_t rows, int64_t cols, int type);
bool norm_in_registers(int64_t cols, int type);
hipError_t launch_norm_backward(const NormBackward& a, int type, bool gain_wide, hipStream_t s);
hipError_t launch_rows8_dequantize(const int8_t* codes, int64_t rows, int64_t cols, int64_t ldc, const float* scales, void* x,
                                   int type, int64_t ldx, hipStream_t s);

// ---- 4-bit weights with group scales -----------------------------------------------------------
// A W4 matrix in its buffer: tiles as an MX4 matrix has them, with other codes, then 16 pairs of FP16 (scale, bias) for
// each row tile and group.
struct W4 {
  const uint8_t* base;
  int64_t rows, cols;
  int group;
  int64_t row_tiles, col_tiles;
  int64_t groups;   // of a row, those of the columns that pad it to whole tiles among them
  int64_t pair_offset;

  __host__ __device__ W4(const void* b, int64_t r, int64_t c, int g)
      : base(static_cast<const uint8_t*>(b)),
        rows(r),
        cols(c),
        group(g),
        row_tiles((r + kTileRows - 1) / kTileRows),
        col_tiles((c + kTileCols - 1) / kTileCols),
        groups(col_tiles * (kTileCols / g)),
        pair_offset(row_tiles * col_tiles * kTileBytes) {}

  __host__ __device__ int64_t tile(int64_t rt, int64_t kt) const { return (rt * col_tiles + kt) * kTileBytes; }
  // the pairs of the 16 rows of tile row rt for a group
  __host__ __device__ int64_t pairs(int64_t rt, int64_t g) const { return pair_offset + (rt * groups + g) * (kTileRows * 4); }
  __host__ __device__ int64_t bytes() const { return pair_offset + row_tiles * groups * (kTileRows * 4); }
};

hipError_t launch_w4_quantize(const void* x, int type, int64_t ld, const W4& q, hipStream_t s);
hipError_t launch_w4_dequantize(const W4& q, void* x, int type, int64_t ld, hipStream_t s);
hipError_t launch_w4_pack(const uint8_t* codes, const uint16_t* scales, const uint16_t* biases, const W4& q, hipStream_t s);
hipError_t launch_w4_unpack(const W4& q, uint8_t* codes, uint16_t* scales, uint16_t* biases, hipStream_t s);

struct W4Linear {
  const void* x;
  const float* scales;   // of 8-bit rows
  int64_t m, ldx;
  const float* bias;
  void* y;
  int64_t ldy;
  int y_type;
  int relu;
};

size_t w4_linear_workspace(int type, int64_t m, int64_t n, int64_t k, int group);
hipError_t launch_w4_linear(const W4Linear& a, int type, const W4& w, void* workspace, hipStream_t s);

// ---- The norm of many gradients ----------------------------------------------------------------
constexpr int kClipThreads = 256;
constexpr int kClipTensors = 480;   // tensors whose pointers one launch carries

struct ClipTensor {
  int64_t size;
  int32_t type;
  uint32_t parts;   // workgroups that share it
};

struct ClipPointers {
  void* g[kClipTensors];
};

struct ClipDev {
  const ClipTensor* tensors;
  const AdamPart* parts;   // chunk: which of a tensor's parts
};

// Squares of parts [part0, part0 + parts) of tensors from `first` on, into partial[part].
hipError_t launch_clip_squares(const ClipDev& d, const ClipPointers& ptr, uint32_t first, int64_t part0, unsigned parts,
                               double* partial, hipStream_t s);
hipError_t launch_clip_join(const double* partial, int64_t parts, double max_norm, float* result, hipStream_t s);
// Joins all parts and scales parts [part0, part0 + some); the launch that holds part 0 writes the result.
hipError_t launch_clip_join_scale(const ClipDev& d, const ClipPointers& ptr, uint32_t first, int64_t part0, unsigned some,
                                  const double* partial, int64_t parts, double max_norm, float* result, hipStream_t s);
hipError_t launch_clip_scale(const ClipDev& d, const ClipPointers& ptr, uint32_t first, int64_t part0, unsigned parts,
                             const float* factor, hipStream_t s);

}  // namespace embd
