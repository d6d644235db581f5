// Internal declarations of the dense operators (include/emb_dense.h): the layout of an MX4
// matrix, shared by host and device, and the launchers.
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

}  // namespace embd
