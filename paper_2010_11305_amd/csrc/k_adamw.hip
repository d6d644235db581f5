// One AdamW step over many tensors.
//
// Every element is read and written once; the bound is memory.  100M elements, us (and TB/s of the bytes that have
// to move): FP32 with FP32 gradients 519 (5.4), BF16 gradients 487 (5.3), BF16 parameters 406 (5.4); moments in 8
// bits: FP32 308 (5.2), BF16 193 (5.2).  BF16 with 8-bit moments and stochastic rounding is bound by the VALU
// as well: 239 (4.2), some 95 instructions a value of which Philox, the square root and the division take half.
//
// A workgroup takes one part (up to kAdamChunk elements) of one tensor, found in a table that was laid out with
// the state, so that tensors of any number and size are one launch per kAdamTensors of
// them and no workgroup searches.  2048 elements a part: with 4096 few tensors left CUs idle (350,000 elements:
// 6.6 us against 5.2) and large ones took 3 to 5% longer.  The pointers travel in the kernel arguments: they may
// change from step to step without a copy to the device.  A thread holds 8 consecutive
// elements, so a block of 32 that shares a scale is 4 neighbouring lanes.
#include "dense_device.h"

namespace embd {

namespace {

constexpr int kPer = kAdamPer;
using s16x2 = short __attribute__((ext_vector_type(2)));

// The largest of a value over the 4 lanes of a quad.
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, false));
  return max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, false));
}

// Scale byte of a block of E4M3 elements: the smallest power of two with which its largest
// magnitude is at most 448 = 1.75 * 2^8.
__device__ __forceinline__ uint32_t e4m3_scale(uint32_t amax) {
  const int e = (int)(amax >> 23);
  if (e == 255) return 255u;
  const int s = e - 8 + ((amax & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return s < 0 ? 0u : (uint32_t)s;
}

// 8 moments of a lane to 8 E4M3 elements and the scale byte of the quad's block.  rest: 2^16 - 1 - u of each
// element's random bits in the upper half (unused when rounding to nearest).  KEEP: what is above 0 becomes
// the smallest element at least.
//
// Stochastic: the conversion adds the top 20 bits r of its random word to the fraction of |x| / 2^s between two
// neighbours, cut to 20 bits, and takes the upper one on a carry.  With r = 2^20 - 1 - 16 u that is a fraction
// above u / 2^16, exactly, if the fraction has no bits beyond 20: |x| / 2^s, a multiple of 2^-29 where E4M3 is
// normal, is made one below by rounding it up, which moves no fraction across a multiple of 2^-16.
template <bool STOCHASTIC, bool KEEP>
__device__ __forceinline__ uint2 e4m3_pack(const float (&x)[kPer], const uint32_t (&rest)[kPer], uint32_t* scale) {
  uint32_t a = 0;
#pragma unroll
  for (int j = 0; j < kPer; ++j) a = max(a, __float_as_uint(x[j]) & (KEEP ? ~0u : 0x7FFFFFFFu));  // a root has no sign,
  const uint32_t s = e4m3_scale(quad_max(a) & 0x7FFFFFFFu);                                // unless it is NaN
  *scale = s;
  if (s == 255u) return make_uint2(0, 0);
  uint32_t w[2];
  if constexpr (STOCHASTIC) {
    const int up = 156 - (int)s;
    uint32_t c[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      float z = ceilf(ldexpf(fabsf(x[j]), up));
      // KEEP: 0 stays 0, what is above 0 (1 at least here) becomes 2^20 at least
      z = KEEP ? __builtin_amdgcn_fmed3f(z, 0x1p20f, z * 0x1p20f) : copysignf(z, x[j]);
      c[j] = (uint32_t)__builtin_amdgcn_cvt_scalef32_sr_fp8_f32(0, z, rest[j] | 0xFFFFu, 0x1p29f, 0);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)  // the low byte of each
      w[i] = __builtin_amdgcn_perm(c[4 * i + 1], c[4 * i], 0x0C0C0400u) |
             __builtin_amdgcn_perm(c[4 * i + 3], c[4 * i + 2], 0x0C0C0400u) << 16;
  } else {
    const float f = power_of(s), least = ldexpf(1.0f, (int)s - 136);
    float q[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) q[j] = KEEP ? (x[j] > 0.0f ? fmaxf(x[j], least) : 0.0f) : x[j];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      s16x2 v = {0, 0};
      v = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(v, q[4 * i], q[4 * i + 1], f, false);
      v = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(v, q[4 * i + 2], q[4 * i + 3], f, true);
      w[i] = __builtin_bit_cast(uint32_t, v);
    }
  }
  return make_uint2(w[0], w[1]);
}

__device__ __forceinline__ void e4m3_unpack(uint2 w, uint32_t scale, float (&x)[kPer]) {
  const float f = power_of(scale);
  const uint32_t ws[2] = {w.x, w.y};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const f32x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(ws[i], f, false);
    const f32x2 hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(ws[i], f, true);
    x[4 * i] = lo[0], x[4 * i + 1] = lo[1], x[4 * i + 2] = hi[0], x[4 * i + 3] = hi[1];
  }
  if (scale == 255u) {
#pragma unroll
    for (int j = 0; j < kPer; ++j) x[j] = __uint_as_float(0x7FC00000u);
  }
}

template <int PT, int GT, int BITS, bool STOCHASTIC>
__global__ __launch_bounds__(kAdamThreads) void k_adamw(AdamDev d, AdamPointers ptr, uint32_t first, int64_t part0, AdamConst c,
                                               const float* __restrict__ grad_scale) {
  const AdamPart part = d.parts[part0 + blockIdx.x];
  const uint32_t slot = part.tensor - first;
  using P = typename Elem<PT>::type;
  using G = typename Elem<GT>::type;
  P* p = static_cast<P*>(ptr.p[slot]);
  const G* g = static_cast<const G*>(ptr.g[slot]);
  if (!g) return;
  const AdamTensor t = d.tensors[part.tensor];
  const float keep = (float)(1.0 - c.lr * t.decay);
  const float gs = grad_scale ? *grad_scale : 1.0f;
  const int64_t i = (int64_t)part.chunk * kAdamChunk + threadIdx.x * kPer;
  // a block of 32 that the tensor reaches into is worked on by its whole quad
  if (i >= (t.size + kBlock - 1) / kBlock * kBlock) return;
  const int n = t.size - i >= kPer ? kPer : t.size > i ? (int)(t.size - i) : 0;
  Raw<PT, kPer> rp;
  Raw<GT, kPer> rg;
  load_values(p + (n ? i : 0), n, rp);
  load_values(g + (n ? i : 0), n, rg);
  const int64_t at = t.base + i;
  float m[kPer], v[kPer];
  if constexpr (BITS == 32) {
    const float4* sm = reinterpret_cast<const float4*>(d.first) + at / 4;
    const float4* sv = reinterpret_cast<const float4*>(d.second) + at / 4;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float4 a = sm[h], b = sv[h];
      m[4 * h] = a.x, m[4 * h + 1] = a.y, m[4 * h + 2] = a.z, m[4 * h + 3] = a.w;
      v[4 * h] = b.x, v[4 * h + 1] = b.y, v[4 * h + 2] = b.z, v[4 * h + 3] = b.w;
    }
  } else {
    const uint2 a = *reinterpret_cast<const uint2*>(d.first + at), b = *reinterpret_cast<const uint2*>(d.second + at);
    e4m3_unpack(a, d.first_scale[at / kBlock], m);
    e4m3_unpack(b, d.second_scale[at / kBlock], v);
#pragma unroll
    for (int j = 0; j < kPer; ++j) v[j] = v[j] * v[j];
  }
  uint32_t word[kPer] = {};
  if constexpr (STOCHASTIC) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint64_t n4 = (uint64_t)(at / 4 + h);
      const uint4 w = philox(make_uint4((uint32_t)n4, (uint32_t)(n4 >> 32), c.t, 0), c.k0, c.k1);
      word[4 * h] = w.x, word[4 * h + 1] = w.y, word[4 * h + 2] = w.z, word[4 * h + 3] = w.w;
    }
  }
  float root[kPer];
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const float gj = rg.get(j) * gs;
    m[j] = m[j] * c.beta1 + gj * c.rest1;
    v[j] = v[j] * c.beta2 + (gj * gj) * c.rest2;
    root[j] = sqrtf(v[j]);
    const float away = m[j] / (root[j] * c.inv_root + c.eps);
    const float x = rp.get(j) * keep - away * c.rate;
    if constexpr (PT == EMB_TYPE_FP32) {
      rp.w[j] = __float_as_uint(x);
    } else if constexpr (STOCHASTIC) {
      const uint32_t b = __float_as_uint(x), u = (word[j] ^ word[j] >> 16) & 0xFFFFu;
      rp.put(j, x != x ? 0x7FC0u : (b + u) >> 16);  // an infinity has no low bits to carry from
    } else {
      rp.put(j, bf16_bits(x));
    }
  }
  if (n < kPer) {
#pragma unroll
    for (int j = 0; j < kPer; ++j)
      if (j >= n) m[j] = 0.0f, v[j] = 0.0f, root[j] = 0.0f;
  }
  if (n == kPer) {
#pragma unroll
    for (int h = 0; h < Raw<PT, kPer>::kWords / 4; ++h) {
      const Bytes16 b = {{rp.w[4 * h], rp.w[4 * h + 1], rp.w[4 * h + 2], rp.w[4 * h + 3]}};
      reinterpret_cast<Bytes16*>(p + i)[h] = b;
    }
  } else {
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      if (j >= n) continue;
      if constexpr (PT == EMB_TYPE_FP32)
        p[i + j] = __uint_as_float(rp.w[j]);
      else
        p[i + j] = (uint16_t)(j % 2 ? rp.w[j / 2] >> 16 : rp.w[j / 2]);
    }
  }
  if constexpr (BITS == 32) {
    float4* sm = reinterpret_cast<float4*>(d.first) + at / 4;
    float4* sv = reinterpret_cast<float4*>(d.second) + at / 4;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      sm[h] = make_float4(m[4 * h], m[4 * h + 1], m[4 * h + 2], m[4 * h + 3]);
      sv[h] = make_float4(v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]);
    }
  } else {
    uint32_t um[kPer], ur[kPer], s1, s2;
#pragma unroll
    for (int j = 0; j < kPer; ++j) um[j] = ~word[j] << 16, ur[j] = ~word[j];
    const uint2 a = e4m3_pack<STOCHASTIC, false>(m, um, &s1);
    const uint2 b = e4m3_pack<STOCHASTIC, true>(root, ur, &s2);
    *reinterpret_cast<uint2*>(d.first + at) = a;
    *reinterpret_cast<uint2*>(d.second + at) = b;
    if (threadIdx.x % 4 == 0) {
      d.first_scale[at / kBlock] = (uint8_t)s1;
      d.second_scale[at / kBlock] = (uint8_t)s2;
    }
  }
}

template <int PT, int GT>
hipError_t adamw_as(const AdamDev& d, const AdamPointers& ptr, uint32_t first, int64_t part0, int64_t parts,
                    const AdamConst& c, const float* gs, int bits, int rounding, hipStream_t s) {
  const unsigned grid = (unsigned)parts;
  const bool random = rounding == EMB_ROUND_STOCHASTIC && (bits == 8 || PT != EMB_TYPE_FP32);
  if (bits == 32) {
    if constexpr (PT != EMB_TYPE_FP32) {
      if (random) {
        k_adamw<PT, GT, 32, true><<<grid, kAdamThreads, 0, s>>>(d, ptr, first, part0, c, gs);
        return hipGetLastError();
      }
    }
    k_adamw<PT, GT, 32, false><<<grid, kAdamThreads, 0, s>>>(d, ptr, first, part0, c, gs);
  } else if (random) {
    k_adamw<PT, GT, 8, true><<<grid, kAdamThreads, 0, s>>>(d, ptr, first, part0, c, gs);
  } else {
    k_adamw<PT, GT, 8, false><<<grid, kAdamThreads, 0, s>>>(d, ptr, first, part0, c, gs);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_adamw(const AdamDev& d, const AdamPointers& ptr, uint32_t first, int64_t part0, int64_t parts,
                        const AdamConst& c, const float* grad_scale, int param_type, int grad_type, int state_bits,
                        int rounding, hipStream_t s) {
#define EMBD_GRAD(PT)                                                                                         \
  switch (grad_type) {                                                                                        \
    case EMB_TYPE_FP32:                                                                                       \
      return adamw_as<PT, EMB_TYPE_FP32>(d, ptr, first, part0, parts, c, grad_scale, state_bits, rounding, s); \
    case EMB_TYPE_BF16:                                                                                       \
      return adamw_as<PT, EMB_TYPE_BF16>(d, ptr, first, part0, parts, c, grad_scale, state_bits, rounding, s); \
    default:                                                                                                  \
      return adamw_as<PT, EMB_TYPE_FP16>(d, ptr, first, part0, parts, c, grad_scale, state_bits, rounding, s); \
  }
  if (param_type == EMB_TYPE_FP32) EMBD_GRAD(EMB_TYPE_FP32)
  EMBD_GRAD(EMB_TYPE_BF16)
#undef EMBD_GRAD
}

}  // namespace embd
