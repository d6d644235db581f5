/*
 * emb_dense.h -- C ABI of the dense operators above the embedding tables, in the
 * same library (libembcache) and with the same conventions as emb_cache.h:
 * int status codes, caller-owned device memory, `stream` a hipStream_t passed as
 * void*, calls that only enqueue kernels unless they say otherwise.
 *
 * Two groups:
 *   emb_mx4_*    matrices in microscaled 4-bit floating point ("MX4"): quantisation
 *                along either axis, expansion, the product of two of them, and the
 *                linear layer on full-precision rows;
 *   emb_adamw_*  one AdamW step over many tensors, with moments in FP32 or 8 bits.
 *
 * MX4.  A block is 32 consecutive values of a row (the last of a row may be
 * shorter).  With a = max |x| over the block it has one power of two
 *   s = clamp(floor(log2 a) - 2, -127, 127), s = -127 for a = 0,
 * kept as the byte s + 127, and each value is kept as a 4-bit code of x / 2^s: sign,
 * 2 exponent bits, 1 mantissa bit, magnitudes {0, 0.5, 1, 1.5, 2, 3, 4, 6}; beyond 6
 * it saturates.  Rounding is to nearest, ties to the even code, or stochastic: to
 * the next magnitude above with probability (|x|/2^s - below) / (above - below),
 * compared with 16 random bits u: up when u * 2^-16 is less.  They are bits
 * 16 (j mod 2) .. +15 of word j div 2, j = column mod 8, of the Philox4x32-10 block
 * with key `seed` and counter (column div 8, row, step, 0), or (..., 1) for a matrix
 * quantised along its columns, whose rows and columns here are those of the result;
 * (..., 2) and (..., 3) for the rows of emb_mx4_linear_train.  Matrices that meet in a product,
 * or of which one follows from the other, must not draw the same bits: the expectation of the product
 * of their roundings is then not that of their values.  So each of them has a seed or a step of its own; a
 * weight takes another seed than the calls of its layer do.
 * A block that holds a NaN or an infinity has byte 255 and codes 0, and stands for NaN.
 *
 * An MX4 matrix [rows][cols] is one device buffer of emb_mx4_query_bytes, 256-byte
 * aligned, laid out for the matrix instructions (emb_mx4_unpack gives plain codes):
 * tiles of 16 rows x 128 columns, 1024 bytes each, row tiles outermost; in a tile
 * the 16 bytes at 16 (16 b + r) are block b (0..3) of row r, columns in order, the
 * even column in the low half of a byte.  The scale bytes follow, for each row tile
 * and each four column tiles 256 bytes: byte 4 (16 b + r) + t for block b, row r of
 * column tile t.  Codes past the last row or column and scale bytes past the last column
 * tile are 0.
 */
#ifndef EMB_DENSE_H
#define EMB_DENSE_H

#include <stddef.h>
#include <stdint.h>

#include "emb_cache.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of full-precision matrices and vectors. */
#define EMB_TYPE_FP32 0
#define EMB_TYPE_BF16 1
#define EMB_TYPE_FP16 2

/* Bytes of an MX4 matrix (0 when it has no element).  rows, cols: 0 .. 2^31 - 1.  Host only. */
int emb_mx4_query_bytes(int64_t rows, int64_t cols, size_t* bytes);

/* Quantise x [rows][cols] (row stride ld >= cols, in elements; any alignment of
 * the type) into by_rows, an MX4 matrix [rows][cols], and into by_columns, the MX4
 * matrix [cols][rows] of its transpose.  Either may be NULL; with both, which must not overlap, x is
 * read once.  rounding: EMB_ROUND_NEAREST or EMB_ROUND_STOCHASTIC (seed and step are
 * used by the latter).  Enqueue-only. */
int emb_mx4_quantize(const void* x, int32_t type, int64_t rows, int64_t cols, int64_t ld, void* by_rows,
                     void* by_columns, int32_t rounding, uint64_t seed, uint32_t step, void* stream);

/* The values that q [rows][cols] stands for, in x [rows][cols] with row stride ld.
 * Exact in FP32 and BF16, FP16 rounds to nearest even; infinite beyond the type's largest value, which in
 * FP32 and BF16 only scale bytes 253 and 254 reach (packed ones: quantisation ends at 252).
 * Enqueue-only. */
int emb_mx4_dequantize(const void* q, int64_t rows, int64_t cols, void* x, int32_t type, int64_t ld, void* stream);

/* Between an MX4 matrix and plain codes: codes [rows][ceil(cols / 2)], two a byte, the
 * even column in the low half, and scale bytes [rows][ceil(cols / 32)], both on the
 * device and without padding.  With an odd number of columns the last half byte of a
 * row is ignored by pack and 0 from unpack.  Enqueue-only. */
int emb_mx4_pack(const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t cols, void* q, void* stream);
int emb_mx4_unpack(const void* q, int64_t rows, int64_t cols, uint8_t* codes, uint8_t* scales, void* stream);

/* c [m][n] (row stride ldc, in elements) = a b^T for MX4 matrices a [m][k] and
 * b [n][k], k <= 2^24: products and sums in FP32, one rounding to `type` (nearest even); zeros
 * for k = 0.  The order of the sums is a function of m, n and k alone.  Enqueue-only. */
int emb_mx4_matmul(const void* a, const void* b, int64_t m, int64_t n, int64_t k, void* c, int32_t type, int64_t ldc,
                   void* stream);

/* The linear layer: y [m][n] = Q(x) w^T for full-precision rows x [m][k] (row stride
 * ldx), quantised to nearest on the way, and an MX4 weight w [n][k]; y in the type of
 * x, row stride ldy.  Equal to emb_mx4_quantize of x and emb_mx4_matmul up to the order
 * of the FP32 sums.  workspace: emb_mx4_linear_workspace bytes, 256-byte aligned, or NULL
 * when that is 0: then y is written while x is still read, and must share no element with it.
 * Enqueue-only. */
int emb_mx4_linear_workspace(int64_t m, int64_t n, int64_t k, size_t* bytes);
int emb_mx4_linear(const void* x, int32_t type, int64_t m, int64_t k, int64_t ldx, const void* w, int64_t n, void* y,
                   int64_t ldy, void* workspace, size_t workspace_bytes, void* stream);

/* One training pass of the layer, in two calls that only put the ones above together.
 *
 * emb_mx4_linear_train: y [m][n] = Q(x) w^T with w by rows, and `saved`, the MX4 matrix [k][m] of
 * the transpose of x that the backward pass needs (emb_mx4_query_bytes(k, m)); x rounds as
 * `rounding` says (seed and step when stochastic, its draws apart from those of the output gradient under
 * the same seed and step).  y in the type of x.
 *
 * emb_mx4_linear_grad: for an output gradient dy [m][n], rounded as `rounding` says,
 *   dx [m][k] = Q(dy) Q(w^T)^T   in the type of dy, w_columns the MX4 matrix [k][n] of w^T
 *   dw [n][k] = Q(dy^T) saved^T  in dw_type
 * The rounding of the codes is the gradients' only approximation: as usual they are those
 * of the unrounded layer, taken at the rounded values.  The depths of its products are n and m: both at most 2^24.
 *
 * workspace: the bytes that the function's own query reports, 256-byte aligned, or NULL when
 * that is 0.  Enqueue-only. */
int emb_mx4_linear_train_workspace(int64_t m, int64_t n, int64_t k, size_t* bytes);
int emb_mx4_linear_train(const void* x, int32_t type, int64_t m, int64_t k, int64_t ldx, const void* w, int64_t n,
                         void* y, int64_t ldy, void* saved, int32_t rounding, uint64_t seed, uint32_t step,
                         void* workspace, size_t workspace_bytes, void* stream);
int emb_mx4_linear_grad_workspace(int64_t m, int64_t n, int64_t k, size_t* bytes);
int emb_mx4_linear_grad(const void* dy, int32_t type, int64_t m, int64_t n, int64_t ldy, const void* w_columns, int64_t k,
                        const void* saved, void* dx, int64_t ldx, void* dw, int32_t dw_type, int64_t ldw,
                        int32_t rounding, uint64_t seed, uint32_t step, void* workspace, size_t workspace_bytes,
                        void* stream);

/* AdamW over `num_tensors` tensors.  Per element, in FP32 with one rounding per
 * operation, t = steps done including this one:
 *   g = gradient * *grad_scale
 *   m = m * beta1 + g * (1 - beta1);  v = v * beta2 + (g * g) * (1 - beta2)
 *   p = p * (1 - lr * weight_decay)
 *       - (m / (sqrt(v) * (1 / sqrt(1 - beta2^t)) + eps)) * (lr / (1 - beta1^t))
 * (constants computed in FP64, then rounded to FP32).
 *
 * Moments: with state_bits 32, m and v in FP32.  With 8, m and r = sqrt(v) as E4M3
 * elements with one power of two per block of 32 consecutive elements of a tensor, the
 * smallest (at least 2^-127) with which the block's largest magnitude is at most 448,
 * kept as a byte biased by 127; v = r * r when it is read.  An r above 0 is never
 * stored as 0, so that m / (r + eps) stays bounded.  A block with a value that is not
 * finite gets the byte 255 and elements 0, and its moments are NaN from then on.
 *
 * rounding of 8-bit moments and BF16 parameters: to nearest even, or stochastic with
 * 16 random bits each: with i the element's place in the state and w word i mod 4 of the
 * Philox4x32-10 block with key `seed` and counter (low and high half of i div 4, t, 0),
 * the low half of w rounds m (up when its share of 2^16 is below the value's share of
 * the step between two neighbours), the high half r, and their exclusive or the
 * parameter.  The first elements share these blocks with row 0 of an MX4 matrix under the same
 * seed and step: a model's optimizer and its layers have different seeds.  Nearest rounding of slowly moving moments loses their small changes;
 * stochastic rounding keeps them on average.
 *
 *   sizes[t]       elements of tensor t, >= 0
 *   weight_decays  one per tensor, or NULL: weight_decay for all
 *   param_type     EMB_TYPE_FP32 or EMB_TYPE_BF16
 *   grad_type      any element type
 */
typedef struct emb_adamw_config {
  int32_t num_tensors;
  int32_t param_type;
  const int64_t* sizes;
  const double* weight_decays;
  int32_t grad_type;
  int32_t state_bits;
  int32_t rounding;
  int32_t pad;
  double beta1;
  double beta2;
  double eps;
  double weight_decay;
  uint64_t seed;
} emb_adamw_config;

/* The state buffer: `elements` is the sum over the tensors of their size padded to a
 * multiple of 32; tensor t starts at the sum of those before it.  At the byte offsets:
 * the first moments, the second moments (v, or r with 8 bits), and with 8 bits their scale
 * bytes, one for each 32 elements. */
typedef struct emb_adamw_sizes {
  size_t state_bytes;
  int64_t elements;
  size_t first_offset;
  size_t second_offset;
  size_t first_scale_offset;
  size_t second_scale_offset;
} emb_adamw_sizes;

typedef struct emb_adamw* emb_adamw_t;

/* Validate `cfg` and report the state's size and layout.  Host only. */
int emb_adamw_query_sizes(const emb_adamw_config* cfg, emb_adamw_sizes* out);

/* Create a handle over a caller-owned device buffer (256-byte aligned) that must stay
 * allocated until emb_adamw_destroy.  Sets all moments and the step counter to 0.
 * Synchronizes `stream`. */
int emb_adamw_create(const emb_adamw_config* cfg, void* state, size_t state_bytes, void* stream, emb_adamw_t* out);
int emb_adamw_destroy(emb_adamw_t h);

/* One step.  params and grads: host arrays of num_tensors device pointers (read during
 * the call only), each tensor contiguous, at any alignment of its type, no parameter in the memory of
 * another.  A tensor whose gradient is NULL keeps its parameters and moments.  grad_scale: an
 * aligned device FP32 factor of every gradient (what a clipped norm leaves, say), or NULL for 1.  The step counter
 * increases by one; it lives on the host, so a call captured into a HIP graph repeats the
 * constants and draws of the step it was captured in.  Enqueue-only. */
int emb_adamw_step(emb_adamw_t h, void* const* params, const void* const* grads, double lr, const float* grad_scale,
                   void* stream);

/* Steps done (t of the next step minus 1), 0 .. 2^63 - 1. */
int emb_adamw_get_step(emb_adamw_t h, uint64_t* step);
int emb_adamw_set_step(emb_adamw_t h, uint64_t step);

#ifdef __cplusplus
}
#endif

#endif /* EMB_DENSE_H */
