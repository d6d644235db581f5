// The norm of many gradients together, and their scaling.
//
// A workgroup takes one part of one tensor, found in a table laid out with the handle; the pointers travel in the
// kernel arguments.  Sums are kept in FP64: no FP32 gradient's square overflows or vanishes there.
#include "dense_device.h"

namespace embd {

namespace {

constexpr int kPer = 8;

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int m = 32; m; m >>= 1) v += __shfl_xor(v, m);
  return v;
}

template <int T>
__device__ __forceinline__ double squares_of(const void* g, int64_t begin, int64_t end) {
  const auto* p = static_cast<const typename Elem<T>::type*>(g);
  double sum = 0.0;
  for (int64_t i = begin + (int64_t)threadIdx.x * kPer; i < end; i += kClipThreads * kPer) {
    Raw<T, kPer> r;
    load_values(p + i, end - i < kPer ? (int)(end - i) : kPer, r);
#pragma unroll
    for (int j = 0; j < kPer; ++j) sum = fma((double)r.get(j), (double)r.get(j), sum);
  }
  return sum;
}

__global__ __launch_bounds__(kClipThreads) void k_clip_squares(ClipDev d, ClipPointers ptr, uint32_t first, int64_t part0,
                                                               double* __restrict__ partial) {
  __shared__ double sums[kClipThreads / 64];
  const int64_t at = part0 + blockIdx.x;
  const AdamPart part = d.parts[at];
  const ClipTensor t = d.tensors[part.tensor];
  const void* g = ptr.g[part.tensor - first];
  double sum = 0.0;
  if (g) {
    const int64_t begin = part.chunk * d.chunk, end = begin + d.chunk < t.size ? begin + d.chunk : t.size;
    sum = t.type == EMB_TYPE_FP32   ? squares_of<EMB_TYPE_FP32>(g, begin, end)
          : t.type == EMB_TYPE_BF16 ? squares_of<EMB_TYPE_BF16>(g, begin, end)
                                    : squares_of<EMB_TYPE_FP16>(g, begin, end);
  }
  sum = wave_sum(sum);
  if (threadIdx.x % 64 == 0) sums[threadIdx.x / 64] = sum;
  __syncthreads();
  if (threadIdx.x == 0) partial[at] = (sums[0] + sums[1]) + (sums[2] + sums[3]);
}

// The sum of all parts, by a workgroup of THREADS; the order is a function of their number and of THREADS.
template <int THREADS>
__device__ __forceinline__ double join(const double* __restrict__ partial, int64_t parts) {
  __shared__ double sums[THREADS / 64];
  double sum = 0.0;
#pragma unroll 4
  for (int64_t i = threadIdx.x; i < parts; i += THREADS) sum += partial[i];
  sum = wave_sum(sum);
  if (threadIdx.x % 64 == 0) sums[threadIdx.x / 64] = sum;
  __syncthreads();
  sum = 0.0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) sum += sums[w];
  return sum;
}

struct ClipResult {
  float norm, factor;
};
__device__ __forceinline__ ClipResult result_of(double squares, double max_norm) {
  const double norm = sqrt(squares);
  return {(float)norm, max_norm >= norm ? 1.0f : (float)(max_norm / norm)};   // NaN stays NaN, infinity over infinity is no limit
}

__global__ __launch_bounds__(kClipThreads) void k_clip_join(const double* __restrict__ partial, int64_t parts, double max_norm,
                                                            float* __restrict__ result) {
  const ClipResult r = result_of(join<kClipThreads>(partial, parts), max_norm);
  if (threadIdx.x == 0) result[0] = r.norm, result[1] = r.factor;
}

template <int T>
__device__ __forceinline__ void scale_part(void* g, int64_t begin, int64_t end, float f) {
  auto* p = static_cast<typename Elem<T>::type*>(g);
  for (int64_t i = begin + (int64_t)threadIdx.x * kPer; i < end; i += kClipThreads * kPer) {
    const int n = end - i < kPer ? (int)(end - i) : kPer;
    Raw<T, kPer> r;
    load_values(p + i, n, r);
#pragma unroll
    for (int j = 0; j < kPer; ++j) r.put(j, to_bits<T>(r.get(j) * f));
    store_values(p + i, n, r);
  }
}

__device__ __forceinline__ void scale(const ClipDev& d, const ClipPointers& ptr, uint32_t first, int64_t at, float f) {
  if (f == 1.0f) return;
  const AdamPart part = d.parts[at];
  const ClipTensor t = d.tensors[part.tensor];
  void* g = ptr.g[part.tensor - first];
  if (!g) return;
  const int64_t begin = part.chunk * d.chunk, end = begin + d.chunk < t.size ? begin + d.chunk : t.size;
  if (t.type == EMB_TYPE_FP32)
    scale_part<EMB_TYPE_FP32>(g, begin, end, f);
  else if (t.type == EMB_TYPE_BF16)
    scale_part<EMB_TYPE_BF16>(g, begin, end, f);
  else
    scale_part<EMB_TYPE_FP16>(g, begin, end, f);
}

__global__ __launch_bounds__(kClipThreads) void k_clip_scale(ClipDev d, ClipPointers ptr, uint32_t first, int64_t part0,
                                                             const float* __restrict__ factor) {
  scale(d, ptr, first, part0 + blockIdx.x, *factor);
}

// The join and the scaling at once: every workgroup adds up the parts for itself (some 2000 values from the L2, while a
// launch of one workgroup and the gap behind it take 4 us).
__global__ __launch_bounds__(kClipThreads) void k_clip_join_scale(ClipDev d, ClipPointers ptr, uint32_t first, int64_t part0,
                                                                  const double* __restrict__ partial, int64_t parts,
                                                                  double max_norm, float* __restrict__ result) {
  const ClipResult r = result_of(join<kClipThreads>(partial, parts), max_norm);
  const int64_t at = part0 + blockIdx.x;
  if (at == 0 && threadIdx.x == 0) result[0] = r.norm, result[1] = r.factor;
  scale(d, ptr, first, at, r.factor);
}

}  // namespace

hipError_t launch_clip_squares(const ClipDev& d, const ClipPointers& ptr, uint32_t first, int64_t part0, unsigned parts,
                               double* partial, hipStream_t s) {
  k_clip_squares<<<parts, kClipThreads, 0, s>>>(d, ptr, first, part0, partial);
  return hipGetLastError();
}

hipError_t launch_clip_join(const double* partial, int64_t parts, double max_norm, float* result, hipStream_t s) {
  k_clip_join<<<1, kClipThreads, 0, s>>>(partial, parts, max_norm, result);
  return hipGetLastError();
}

hipError_t launch_clip_scale(const ClipDev& d, const ClipPointers& ptr, uint32_t first, int64_t part0, unsigned parts,
                             const float* factor, hipStream_t s) {
  k_clip_scale<<<parts, kClipThreads, 0, s>>>(d, ptr, first, part0, factor);
  return hipGetLastError();
}

hipError_t launch_clip_join_scale(const ClipDev& d, const ClipPointers& ptr, uint32_t first, int64_t part0, unsigned some,
                                  const double* partial, int64_t parts, double max_norm, float* result, hipStream_t s) {
  k_clip_join_scale<<<some, kClipThreads, 0, s>>>(d, ptr, first, part0, partial, parts, max_norm, result);
  return hipGetLastError();
}

}  // namespace embd
