// The norm of many gradients together, and their scaling.
//
// A workgroup takes a part of one tensor, found in a table laid out with the handle; the pointers travel in the kernel
// arguments.  Sums are kept in FP64: no FP32 gradient's square overflows or vanishes there, and its operations are as
// fast as those of FP32.
//
// Memory bounds both kernels where there is much: by the kernel trace, 200M BF16 in 300 tensors, squares 83 us (4.8 TB/s; 120 right
// behind a kernel that wrote them), join and scaling 156 (5.1 TB/s); 350,000 FP32 in 6 tensors 3.5 and 3.9 us, of which a launch
// is most.
#include "dense_device.h"

namespace embd {

namespace {

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int m = 32; m; m >>= 1) v += __shfl_xor(v, m);
  return v;
}

// A workgroup takes every parts-th unit of a tensor, of 16 bytes a thread, so that neighbouring workgroups read neighbouring
// memory, and has four loads under way (200M BF16: 86 us, with one 90).
template <int T>
__device__ __forceinline__ double squares_of(const void* g, const ClipTensor& t, uint32_t part) {
  constexpr int N = 16 / Elem<T>::kBytes, kAtOnce = 4;
  const auto* p = static_cast<const typename Elem<T>::type*>(g);
  const int64_t begin = (int64_t)part * (kClipThreads * N), end = t.size, stride = (int64_t)t.parts * (kClipThreads * N);
  double sum = 0.0;
  int64_t i = begin + threadIdx.x * N;
  for (; i + (kAtOnce - 1) * stride + N <= end; i += kAtOnce * stride) {
    Raw<T, N> r[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const Bytes16 w = *reinterpret_cast<const Bytes16*>(p + i + k * stride);
#pragma unroll
      for (int j = 0; j < 4; ++j) r[k].w[j] = w.w[j];
    }
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k)
#pragma unroll
      for (int j = 0; j < N; ++j) sum = fma((double)r[k].get(j), (double)r[k].get(j), sum);
  }
  for (; i < end; i += stride) {
    Raw<T, N> r;
    load_values(p + i, end - i < N ? (int)(end - i) : N, r);
#pragma unroll
    for (int j = 0; j < N; ++j) sum = fma((double)r.get(j), (double)r.get(j), sum);
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
    sum = t.type == EMB_TYPE_FP32   ? squares_of<EMB_TYPE_FP32>(g, t, part.chunk)
          : t.type == EMB_TYPE_BF16 ? squares_of<EMB_TYPE_BF16>(g, t, part.chunk)
                                    : squares_of<EMB_TYPE_FP16>(g, t, part.chunk);
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
__device__ __forceinline__ void scale_part(void* g, const ClipTensor& t, uint32_t part, float f) {
  constexpr int N = 16 / Elem<T>::kBytes;
  auto* p = static_cast<typename Elem<T>::type*>(g);
  const int64_t stride = (int64_t)t.parts * (kClipThreads * N);
#pragma unroll 2
  for (int64_t i = (int64_t)part * (kClipThreads * N) + threadIdx.x * N; i < t.size; i += stride) {
    const int n = t.size - i < N ? (int)(t.size - i) : N;
    Raw<T, N> r;
    load_values(p + i, n, r);
#pragma unroll
    for (int j = 0; j < N; ++j) r.put(j, to_bits<T>(r.get(j) * f));
    store_values(p + i, n, r);
  }
}

__device__ __forceinline__ void scale(const ClipDev& d, const ClipPointers& ptr, uint32_t first, int64_t at, float f) {
  if (f == 1.0f) return;
  const AdamPart part = d.parts[at];
  const ClipTensor t = d.tensors[part.tensor];
  void* g = ptr.g[part.tensor - first];
  if (!g) return;
  if (t.type == EMB_TYPE_FP32)
    scale_part<EMB_TYPE_FP32>(g, t, part.chunk, f);
  else if (t.type == EMB_TYPE_BF16)
    scale_part<EMB_TYPE_BF16>(g, t, part.chunk, f);
  else
    scale_part<EMB_TYPE_FP16>(g, t, part.chunk, f);
}

__global__ __launch_bounds__(kClipThreads) void k_clip_scale(ClipDev d, ClipPointers ptr, uint32_t first, int64_t part0,
                                                             const float* __restrict__ factor) {
  scale(d, ptr, first, part0 + blockIdx.x, *factor);
}

// The join and the scaling at once: every workgroup adds up all parts for itself, from the L2.  For the tensors of one launch, which
// have 2048 parts and one a tensor at most; every launch more would add them up again, in each of its workgroups.  us in a
// graph, both kernels, against a join of one workgroup and k_clip_scale: 6 tensors of 58,000 4.4 (5.6), 480 of 1000 6.9 (7.6),
// 480 of 8192 15.4 (16.1); of several launches 1000 of 1000 20.6 (19.1), 4000 73 (62), 30,000 of 100 822 (378).
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
