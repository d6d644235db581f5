// Products of MX4 matrices on the scaled matrix instruction v_mfma_scale_f32_16x16x128_f8f6f4: a lane's
// operand is one block, 32 codes in four registers, and its scale one byte of a register, which the layout of
// an MX4 matrix holds lane by lane.  Codes and scales go from memory to the instruction as they lie.
//
// k_product: tiles of C of 256, 128 or 64 rows and columns, the operands staged in LDS.  16384 x 8192 x 12800: 642 to
// 780 us from card to card, 5.4 to 4.4 PFLOP/s.  Two things bound it.  Power: on normal values the clock is 1.6 GHz, on
// zeros 2.2 (575 us), with the same 1.25 to 1.27M cycles.  And the cycles, of which the matrix pipes are busy for 65%:
// a step of 128 columns takes 1375 to 1415 (by the time's slope over K, whatever the values) and its instructions
// issue for 1024; start and end of a 256 x 256 tile take some 18000 more.  Of a wave's time 59% issues, 23% waits for
// its turn to issue and 18% at waits and barriers; LDS reads are active for 20% and stall nothing (0.1%).  The 32x32x64
// instruction needs 6% fewer cycles and takes 2% longer.
// k_skinny: few rows against a weight that is read once.  1 row, 4096 x 12800: 5.3 us for 27.9 MB, much of it
// from the last-level cache; 1 row, 32000 x 4096: 14.9 us, 4.7 TB/s.
#include <type_traits>

#include "dense_device.h"

namespace embd {

namespace {

using v8i = int __attribute__((ext_vector_type(8)));
using v4i = int __attribute__((ext_vector_type(4)));
using f32x4 = float __attribute__((ext_vector_type(4)));

// acc += b a over 128 columns with scale byte S of sb and sa.  IN_PLACE: the instruction is written
// out with the accumulator tied to its registers.  With 256 of them the register allocator
// otherwise moves accumulators about between the steps (752 moves for 256 products).  The
// values it reads come from LDS long before; whoever reads acc waits with mma_done.
template <int S, bool IN_PLACE>
__device__ __forceinline__ void mma(f32x4& acc, const v4i& b, const v4i& a, uint32_t sb, uint32_t sa) {
  if constexpr (IN_PLACE) {
#define EMBD_MMA(SEL)                                                                                       \
  asm("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 " SEL " cbsz:4 blgp:4"                       \
      : "+a"(acc)                                                                                           \
      : "v"(b), "v"(a), "v"(sb), "v"(sa))
    if constexpr (S == 0) EMBD_MMA("op_sel:[0,0,0] op_sel_hi:[0,0,0]");
    if constexpr (S == 1) EMBD_MMA("op_sel:[1,1,0] op_sel_hi:[0,0,0]");
    if constexpr (S == 2) EMBD_MMA("op_sel:[0,0,0] op_sel_hi:[1,1,0]");
    if constexpr (S == 3) EMBD_MMA("op_sel:[1,1,0] op_sel_hi:[1,1,0]");
#undef EMBD_MMA
  } else {
    const v8i b8 = {b[0], b[1], b[2], b[3]}, a8 = {a[0], a[1], a[2], a[3]};
    acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b8, a8, acc, 4, 4, S, (int)sb, S, (int)sa);
  }
}

// Wait states between the last matrix instruction and the first read of its result (at most 18); nothing is
// moved across.
__device__ __forceinline__ void mma_done() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_nop 15\n\ts_nop 3" : : : "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// An accumulator on its way out, kept where it is until here: the compiler would copy all 256 registers at once for two
// ways of storing them, and spill (FP32, 4096x4096x8192: 80 us, without 65).
template <int FM>
__device__ __forceinline__ f32x4 fetched(f32x4 v) {
  if constexpr (FM == 8) asm volatile("" : "+a"(v));
  return v;
}

// The rows of C are the columns of an instruction's result (b is its first operand), so that a
// lane holds four consecutive columns of a row of C.

// Columns [col, col + 4) of one row of C.
template <int TYPE>
__device__ __forceinline__ void store4(typename Elem<TYPE>::type* row, int64_t col, int64_t n, const f32x4& v) {
  if (col + 4 <= n) {
    if constexpr (TYPE == EMB_TYPE_FP32) {
      Bytes16 b;
#pragma unroll
      for (int i = 0; i < 4; ++i) b.w[i] = __float_as_uint(v[i]);
      *reinterpret_cast<Bytes16*>(row + col) = b;
    } else {
      Bytes8 b;
#pragma unroll
      for (int i = 0; i < 2; ++i) b.w[i] = to_bits<TYPE>(v[2 * i]) | to_bits<TYPE>(v[2 * i + 1]) << 16;
      *reinterpret_cast<Bytes8*>(row + col) = b;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (col + i >= n) continue;
      if constexpr (TYPE == EMB_TYPE_FP32)
        row[col + i] = v[i];
      else
        row[col + i] = (uint16_t)to_bits<TYPE>(v[i]);
    }
  }
}

// ---- tiles staged through LDS ---------------------------------------------------------------
using Srd = int __attribute__((ext_vector_type(4)));

// A buffer descriptor over the bytes from p on.  Callers keep every offset inside the matrix
// themselves: the scalar part of an offset takes no part in the hardware's range check.
__device__ __forceinline__ Srd make_srd(const uint8_t* p) {
  const uint64_t a = reinterpret_cast<uint64_t>(p);
  Srd r = {__builtin_amdgcn_readfirstlane((int)(uint32_t)a),
           __builtin_amdgcn_readfirstlane((int)((uint32_t)(a >> 32) & 0xFFFFu)), -1, 0x00020000};
  return r;
}

__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p;
}

// 16 bytes a lane from memory into LDS at lds + 16 lane, without registers between.  The
// compiler does not count it: stage_ready waits for it.
__device__ __forceinline__ void load_to_lds(uint32_t lds, uint32_t lane_offset, const Srd& srd, uint32_t offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
               :
               : "s"(lds), "v"(lane_offset), "s"(srd), "s"(offset)
               : "memory", "m0");
}

// All but the last IN_FLIGHT of the wave's loads to LDS have arrived, and its reads of LDS are
// done; then the workgroup meets: every wave sees the stage, and the one read before may
// be overwritten.
template <int IN_FLIGHT>
__device__ __forceinline__ void stage_ready() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "i"(IN_FLIGHT) : "memory");
}

constexpr int kStages = 4;  // one per tile column of a scale group: the loop's body is four steps

// Tiles of 256 x 256 leave one workgroup to a CU (accumulators fill half its registers, four stages its LDS), so
// nothing would run beside the end of a tile and the start of the next: there a workgroup stays and takes
// tile after tile, and the last steps of one load the first stages of the next.
template <int FM>
constexpr bool kStays = FM == 8;
constexpr int kResident = 256;   // workgroups that stay: one to a CU

template <int FM>
using Stages = v4i[kStages][4 * FM][64];     // codes, row tiles of both operands
template <int FM>
using StageScales = uint32_t[2][4 * FM][64];

// Workgroup `block` of `blocks`, of 2 x 2 waves, computes (32 FM) x (32 FM) of C, a wave FM x FM tiles of 16 x 16.
template <int TYPE, int FM>
__device__ __forceinline__ void product(Stages<FM>& stage, StageScales<FM>& scales, v4i* leave, const Mx4& a, const Mx4& b,
                                        typename Elem<TYPE>::type* __restrict__ c, int64_t ldc, uint32_t block, uint32_t blocks) {
  constexpr int kSide = 2 * FM;                       // row tiles of an operand in a stage
  constexpr int kTiles = 2 * kSide;
  constexpr int kLoads = kTiles / 4;                  // a wave's share of them, all of one operand
  constexpr int kScaleLoads = FM >= 4 ? FM / 4 : 1;   // 4 row tiles each
  // Results leave 16 rows x 256 bytes (or a wave's whole width) at a time, through 4 KB of LDS for each wave: beside
  // the stages where the next tile's are in them, else over them.
  constexpr int kBytes = Elem<TYPE>::kBytes;
  constexpr int kOutCols = FM * 16 * kBytes <= 256 ? FM * 16 : 256 / kBytes;
  constexpr int kLanes = kOutCols * kBytes / 16, kRows = 64 / kLanes;   // lanes a row, rows an access
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave >> 1, wn = wave & 1;

  // Workgroups go to the XCDs in turn.  Each XCD takes a run of consecutive tiles, in bands of 8 tile rows, so that what
  // its L2 holds is used by the workgroups that run there together.
  // Their number is below 2^31.
  const uint32_t mt_all = (uint32_t)((a.row_tiles + kSide - 1) / kSide), nt_all = (uint32_t)((b.row_tiles + kSide - 1) / kSide);
  const uint32_t total = mt_all * nt_all, xcd = block % 8;
  const uint32_t run0 = xcd * (total / 8) + (xcd < total % 8 ? xcd : total % 8);
  const uint32_t run = total / 8 + (xcd < total % 8 ? 1 : 0);
  const uint32_t stride = (blocks + 7) / 8;
  const auto place = [&](uint32_t nth, int64_t* rt_a, int64_t* rt_b) {
    const uint32_t id = run0 + nth, band = id / (8 * nt_all), in_band = id % (8 * nt_all);
    const uint32_t band_rows = mt_all - band * 8 < 8 ? mt_all - band * 8 : 8;
    *rt_a = (int64_t)(band * 8 + in_band % band_rows) * kSide;
    *rt_b = (int64_t)(in_band / band_rows) * kSide;
  };

  const int KT = (int)a.col_tiles, KG = (int)a.col_groups;
  const bool of_a = wave < 2;
  const Mx4& mine = of_a ? a : b;
  // What this wave loads: row tiles past the last one are read from it, their products are not stored.
  Srd codes, scale_srd;
  uint32_t code_at[kLoads], scale_at[kScaleLoads];   // a scale load is of 4 row tiles, 16 lanes each
  const auto aim = [&](int64_t rt_a, int64_t rt_b) {
    const auto row_tile = [&](int64_t rt) { return rt < mine.row_tiles ? rt : mine.row_tiles - 1; };
    const int64_t rt0 = row_tile((of_a ? rt_a : rt_b) + (wave & 1) * kLoads);
    codes = make_srd(mine.base + mine.tile(rt0, 0));
#pragma unroll
    for (int i = 0; i < kLoads; ++i) code_at[i] = (uint32_t)(row_tile(rt0 + i) - rt0) * (uint32_t)KT * kTileBytes + lane * 16;
    const int64_t rs0 = row_tile((of_a ? rt_a : rt_b) + (FM >= 4 ? (wave & 1) * FM : 0));
    scale_srd = make_srd(mine.base + mine.scale_offset + rs0 * KG * kScaleBytes);
#pragma unroll
    for (int i = 0; i < kScaleLoads; ++i)
      scale_at[i] = (uint32_t)(row_tile(rs0 + 4 * i + (lane >> 4)) - rs0) * (uint32_t)KG * kScaleBytes + (lane & 15) * 16;
  };
  const uint32_t stage_at = lds_address(&stage[0][wave * kLoads][0]);
  const uint32_t scales_at = lds_address(&scales[0][(of_a ? 0 : kSide) + (FM >= 4 ? (wave & 1) * FM : 0)][0]);

  // Column tiles past the last one are loaded from it again, so that the number of loads in flight
  // stays the same; the steps of the last group that run over them have scale bytes 0 on both
  // sides, 2^-254 of whatever finite codes are there, which FP32 sums do not see.
  const auto load_part = [&](int s, int kt, int i) {
    const int k = kt < KT ? kt : KT - 1;
    load_to_lds(stage_at + s * (kTiles * 1024) + i * 1024, code_at[i], codes, k * kTileBytes);
  };
  const auto load_scales = [&](int parity, int kg) {
    const int k = kg < KG ? kg : KG - 1;
#pragma unroll
    for (int i = 0; i < kScaleLoads; ++i)
      load_to_lds(scales_at + parity * (kTiles * 256) + i * 1024, scale_at[i], scale_srd, k * kScaleBytes);
  };

  uint32_t nth = block / 8;
  int64_t rt_a, rt_b;
  place(nth, &rt_a, &rt_b);
  aim(rt_a, rt_b);
  f32x4 acc[FM][FM] = {};
  v4i fa[2][FM], fb[2][FM];
  uint32_t sa[FM], sb[FM], sna[FM], snb[FM];
  load_scales(0, 0);
#pragma unroll
  for (int s = 0; s < kStages; ++s)
#pragma unroll
    for (int i = 0; i < kLoads; ++i) load_part(s, s, i);
  stage_ready<3 * kLoads>();
#pragma unroll
  for (int i = 0; i < FM; ++i) {
    fa[0][i] = stage[0][wm * FM + i][lane], sa[i] = scales[0][wm * FM + i][lane];
    fb[0][i] = stage[0][kSide + wn * FM + i][lane], sb[i] = scales[0][kSide + wn * FM + i][lane];
  }

  // Step s of a group: wait for the stage of the step behind it, let column tile `ahead` + s be loaded over
  // this step's stage (in registers since the step before), read the next stage while this one's products
  // run.  The loads and reads are spread over the products, one between two of them: left
  // alone, the compiler puts the reads behind them all, and the next step waits for LDS.
  int parity = 0;   // of the group's scales
  const auto step = [&](auto S, int ahead) {
    constexpr int s = decltype(S)::value, cur = s & 1, nxt = cur ^ 1;
    // in flight behind the next stage: two later ones, and between them the scales of a step 0
    stage_ready<2 * kLoads + (s == 1 || s == 2 ? kScaleLoads : 0)>();
    if constexpr (s == 0) load_scales(parity ^ 1, ahead / 4);
#pragma unroll
    for (int i = 0; i < FM; ++i) {
#pragma unroll
      for (int j = 0; j < FM; ++j) {
        mma<s, FM == 8>(acc[i][j], fb[cur][j], fa[cur][i], sb[j], sa[i]);
        __builtin_amdgcn_sched_barrier(0);
        if (j == FM / 4 - (FM == 2 ? 0 : 1)) fa[nxt][i] = stage[(s + 1) % kStages][wm * FM + i][lane];
        if (j == FM / 2 - 1) fb[nxt][i] = stage[(s + 1) % kStages][kSide + wn * FM + i][lane];
        if (j == 3 * FM / 4 - 1 && i < kLoads) load_part(s, ahead + s, i);
        if (s == 3 && j == FM - 1) {
          sna[i] = scales[parity ^ 1][wm * FM + i][lane];
          snb[i] = scales[parity ^ 1][kSide + wn * FM + i][lane];
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    if constexpr (s == 3) {
#pragma unroll
      for (int i = 0; i < FM; ++i) sa[i] = sna[i], sb[i] = snb[i];
    }
  };
  for (;;) {
    const int64_t row0 = (rt_a + wm * FM) * kTileRows, col0 = (rt_b + wn * FM) * kTileRows;
    nth += stride;
    const bool more = kStays<FM> && nth < run;
    for (int kt = 0; kt < KT; kt += kStages) {
      int ahead = kt + kStages;
      if (more && ahead >= KT) {  // the last group loads the first of the next tile
        place(nth, &rt_a, &rt_b);
        aim(rt_a, rt_b);
        ahead = 0;
      }
      step(std::integral_constant<int, 0>{}, ahead);
      step(std::integral_constant<int, 1>{}, ahead);
      step(std::integral_constant<int, 2>{}, ahead);
      step(std::integral_constant<int, 3>{}, ahead);
      parity ^= 1;
      if (FM == 8 && kt + kStages >= KT) mma_done();
    }
    if (!kStays<FM>) stage_ready<0>();  // the stages are free

    // A wave's part of C, where it lies inside: whole lines out of LDS (16-byte pieces of a row exchanged by the row's
    // number, so that no bank is hit twice).  Elsewhere element by element.
    int l = lane;
    asm volatile("" : "+v"(l));  // or the addresses below would be computed ahead of all tiles, and kept
    if (row0 + FM * 16 <= a.rows && col0 + FM * 16 <= b.rows) {
      uint8_t* own = kStays<FM> ? reinterpret_cast<uint8_t*>(leave + wave * 256)
                                : reinterpret_cast<uint8_t*>(&stage[0][0][0]) + wave * 4096;
      typename Elem<TYPE>::type* out = c + (row0 + l / kLanes) * ldc + col0 + l % kLanes * (16 / kBytes);
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j0 = 0; j0 < FM; j0 += kOutCols / 16) {
#pragma unroll
          for (int j = 0; j < kOutCols / 16; ++j) {
            const int at = (j * 16 + (l >> 4) * 4) * kBytes;
            uint8_t* p = own + (l & 15) * (kOutCols * kBytes) + ((at / 16 ^ l) % kLanes) * 16 + at % 16;
            const f32x4 v = fetched<FM>(acc[i][j0 + j]);
            if constexpr (TYPE == EMB_TYPE_FP32)
              *reinterpret_cast<f32x4*>(p) = v;
            else
              *reinterpret_cast<uint2*>(p) = make_uint2(to_bits<TYPE>(v[0]) | to_bits<TYPE>(v[1]) << 16,
                                                        to_bits<TYPE>(v[2]) | to_bits<TYPE>(v[3]) << 16);
          }
          asm volatile("" : : : "memory");
          __builtin_amdgcn_wave_barrier();
#pragma unroll
          for (int r0 = 0; r0 < 16; r0 += kRows) {
            const int r = r0 + l / kLanes;
            const v4i v = *reinterpret_cast<const v4i*>(own + r * (kOutCols * kBytes) + ((l ^ r) % kLanes) * 16);
            const Bytes16 w = {{(uint32_t)v[0], (uint32_t)v[1], (uint32_t)v[2], (uint32_t)v[3]}};
            *reinterpret_cast<Bytes16*>(out + (i * 16 + r0) * ldc + j0 * 16) = w;
          }
          asm volatile("" : : : "memory");
          __builtin_amdgcn_wave_barrier();
          __builtin_amdgcn_sched_barrier(0);  // accumulators are fetched as they leave
        }
    } else {
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FM; ++j) {
          const int64_t row = row0 + i * kTileRows + (l & 15);
          const int64_t col = col0 + j * kTileRows + (l >> 4) * 4;
          if (row < a.rows && col < b.rows) store4<TYPE>(c + row * ldc, col, b.rows, fetched<FM>(acc[i][j]));
        }
    }
    if (!more) break;
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FM; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  if (kStays<FM>) stage_ready<0>();  // no load to LDS outlives the workgroup
}

template <int TYPE, int FM>
__global__ __launch_bounds__(256, FM == 8 ? 1 : 2) void k_product(Mx4 a, Mx4 b,
                                                                 typename Elem<TYPE>::type* __restrict__ c, int64_t ldc) {
  __shared__ Stages<FM> stage;
  __shared__ StageScales<FM> scales;
  __shared__ v4i leave[kStays<FM> ? 4 * 256 : 1];
  product<TYPE, FM>(stage, scales, leave, a, b, c, ldc, blockIdx.x, gridDim.x);
}

// Two products in one launch: the first `blocks1` workgroups compute c1, the others c2.
template <int TYPE1, int TYPE2>
__global__ __launch_bounds__(256, 2) void k_two_products(Mx4 a1, Mx4 b1, typename Elem<TYPE1>::type* __restrict__ c1,
                                                         int64_t ldc1, uint32_t blocks1, Mx4 a2, Mx4 b2,
                                                         typename Elem<TYPE2>::type* __restrict__ c2, int64_t ldc2) {
  __shared__ Stages<2> stage;
  __shared__ StageScales<2> scales;
  if (blockIdx.x < blocks1)
    product<TYPE1, 2>(stage, scales, nullptr, a1, b1, c1, ldc1, blockIdx.x, blocks1);
  else
    product<TYPE2, 2>(stage, scales, nullptr, a2, b2, c2, ldc2, blockIdx.x - blocks1, gridDim.x - blocks1);
}

// ---- few rows ---------------------------------------------------------------------------------
// One operand (x) has few rows: a workgroup takes 16 MT of them (blockIdx.y) and 16 of the other (w), and its
// waves share the columns: a wave takes one group of four column tiles at a time straight into
// registers (4 KB, with the next one already on its way) and the waves' sums meet in LDS, in
// the order of the waves.  XT >= 0: x is a full-precision matrix that every workgroup
// quantises into LDS first, 32 values a thread, while the first group of w arrives.
constexpr int kSkinnyWaves = 16;
constexpr int kFusedValues = 65536;   // of x, most

struct FullRows {
  const void* x;
  int64_t ld;
};

template <int XT, int TYPE, int MT, bool SWAP>
__global__ __launch_bounds__(64 * kSkinnyWaves) void k_skinny(Mx4 w, Mx4 x, FullRows full,
                                                              typename Elem<TYPE>::type* __restrict__ c, int64_t ldc,
                                                              int64_t first) {
  constexpr bool kFused = XT >= 0;
  __shared__ f32x4 sums[kSkinnyWaves][MT][64];
  __shared__ uint4 codes[kFused ? kFusedValues / kBlock : 1];
  __shared__ uint32_t code_scales[kFused ? kFusedValues / kBlock / 4 : 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int64_t rt = first + blockIdx.x;
  const int KT = (int)w.col_tiles, KG = (int)w.col_groups;
  const int64_t x_tile0 = (int64_t)blockIdx.y * MT;
  const int m = (int)(x.rows - x_tile0 * kTileRows < MT * kTileRows ? x.rows - x_tile0 * kTileRows : MT * kTileRows);

  v4i next[4];
  uint32_t next_scale;
  const auto fetch = [&](int kg) {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int kt = kg * 4 + t < KT ? kg * 4 + t : KT - 1;   // past the end: scale byte 0
      next[t] = *reinterpret_cast<const v4i*>(w.base + w.tile(rt, kt) + 16 * lane);
    }
    next_scale = *reinterpret_cast<const uint32_t*>(w.base + w.scale_offset + (rt * KG + kg) * kScaleBytes + 4 * lane);
  };
  if (wave < KG) fetch(wave);

  if constexpr (kFused) {
    // block b of row r of column tile kt at (4 kt + b) m + r; its scale byte in byte kt % 4 of a dword
    const auto* px = static_cast<const typename Elem<XT>::type*>(full.x);
    for (int id = threadIdx.x; id < KG * 16 * m; id += blockDim.x) {
      const int r = id % m, block = id / m;
      const int64_t left = x.cols - (int64_t)block * kBlock;
      Raw<XT, kBlock> v;
      load_values(px + (left > 0 ? r * full.ld + (int64_t)block * kBlock : 0), (int)(left < 0 ? 0 : left > kBlock ? kBlock : left), v);
      uint32_t s;
      codes[id] = quantize_block<XT, false>(v, 0, 0, Mx4Random{}, &s);
      const int kt = block / 4, b = block % 4;
      reinterpret_cast<uint8_t*>(code_scales)[4 * ((kt / 4 * 4 + b) * m + r) + kt % 4] = (uint8_t)s;
    }
    __syncthreads();
  }

  f32x4 acc[MT] = {};
  for (int kg = wave; kg < KG; kg += waves) {
    v4i cur[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) cur[t] = next[t];
    const uint32_t scale = next_scale;
    if (kg + waves < KG) fetch(kg + waves);
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int row = i * 16 + (lane & 15), b = lane >> 4;
      if (i * 16 >= m) break;
      v4i xf[4];
      uint32_t xs;
      if constexpr (kFused) {
        const bool in = row < m;
        xs = in ? code_scales[(kg * 4 + b) * m + row] : 0u;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          xf[t] = v4i{0, 0, 0, 0};
          if (in) xf[t] = __builtin_bit_cast(v4i, codes[((kg * 4 + t) * 4 + b) * m + row]);
        }
      } else {
        xs = *reinterpret_cast<const uint32_t*>(x.base + x.scale_offset + ((x_tile0 + i) * KG + kg) * kScaleBytes + 4 * lane);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const int kt = kg * 4 + t < KT ? kg * 4 + t : KT - 1;
          xf[t] = *reinterpret_cast<const v4i*>(x.base + x.tile(x_tile0 + i, kt) + 16 * lane);
        }
      }
      mma<0, false>(acc[i], cur[0], xf[0], scale, xs);
      mma<1, false>(acc[i], cur[1], xf[1], scale, xs);
      mma<2, false>(acc[i], cur[2], xf[2], scale, xs);
      mma<3, false>(acc[i], cur[3], xf[3], scale, xs);
    }
  }
#pragma unroll
  for (int i = 0; i < MT; ++i) sums[wave][i][lane] = acc[i];
  __syncthreads();
  for (int i = wave; i < MT; i += waves) {
    if (i * 16 + (lane & 15) >= m) continue;
    const int64_t row = (x_tile0 + i) * kTileRows + (lane & 15), col = rt * kTileRows + (lane >> 4) * 4;
    f32x4 v = sums[0][i][lane];
    for (int k = 1; k < waves; ++k) v = v + sums[k][i][lane];
    if constexpr (SWAP) {  // the rows of w are those of C
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (col + q >= w.rows) continue;
        if constexpr (TYPE == EMB_TYPE_FP32)
          c[(col + q) * ldc + row] = v[q];
        else
          c[(col + q) * ldc + row] = (uint16_t)to_bits<TYPE>(v[q]);
      }
    } else if (col < w.rows) {
      store4<TYPE>(c + row * ldc, col, w.rows, v);
    }
  }
}

// Row tiles of a workgroup's x in k_skinny.
int skinny_tiles(int64_t x_tiles) { return x_tiles <= 1 ? 1 : x_tiles <= 2 ? 2 : 4; }

template <int XT, int TYPE, bool SWAP>
hipError_t skinny(const Mx4& w, const Mx4& x, const FullRows& full, typename Elem<TYPE>::type* c, int64_t ldc,
                  hipStream_t s) {
  // as many rounds of groups as 16 waves need, and no more waves than these rounds do
  const int64_t rounds = (w.col_groups + kSkinnyWaves - 1) / kSkinnyWaves;
  const int64_t need = (w.col_groups + rounds - 1) / rounds;
  const unsigned threads = 64u * (unsigned)(XT >= 0 && need < 4 ? 4 : need);
  const int mt = skinny_tiles(x.row_tiles);
  return in_launches(w.row_tiles, (int)threads, [&](int64_t first, unsigned n) {
    const dim3 grid(n, (unsigned)ceil_div(x.row_tiles, mt));
    if (mt == 1)
      k_skinny<XT, TYPE, 1, SWAP><<<grid, threads, 0, s>>>(w, x, full, c, ldc, first);
    else if (mt == 2)
      k_skinny<XT, TYPE, 2, SWAP><<<grid, threads, 0, s>>>(w, x, full, c, ldc, first);
    else
      k_skinny<XT, TYPE, 4, SWAP><<<grid, threads, 0, s>>>(w, x, full, c, ldc, first);
    return hipGetLastError();
  });
}

// C = 0 (a product over no columns).
template <int TYPE>
__global__ __launch_bounds__(256) void k_zero(int64_t m, int64_t n, typename Elem<TYPE>::type* __restrict__ c, int64_t ldc) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < m * n; i += (int64_t)gridDim.x * 256) c[i / n * ldc + i % n] = 0;
}

// ---- the way of a product ------------------------------------------------------------------------
int64_t tiles_of(const Mx4& a, const Mx4& b, int f) { return product_tiles(a.row_tiles, b.row_tiles, f); }

// k_skinny reads its w once for each 64 rows of x and its x once for each 16 rows of w, all of it from L2 at best: it
// wins while its workgroups are about as many as the CUs can hold at once, whatever the columns, and for up
// to 16 rows always.  us, k_skinny against the best of k_product: 300x300x12800 8.6 / 16.1 (95 workgroups of 4
// tiles), 512x512x4096 5.6 / 7.3 (256), 96x3000x6000 9.7 / 10.3 (376), 32x8192x12800 15.6 / 18.0 (512 of 2 tiles);
// 200x2000x12800 21.2 / 17.3 (500), 64x8192x12800 21.1 / 18.3 (512), 1024x1024x12800 31.3 / 18.3 (1024).
bool use_skinny(const Mx4& a, const Mx4& b) {
  const int64_t x = a.row_tiles < b.row_tiles ? a.row_tiles : b.row_tiles;
  const int64_t w = a.row_tiles < b.row_tiles ? b.row_tiles : a.row_tiles;
  const int mt = skinny_tiles(x);
  return x <= 1 || w * ((x + mt - 1) / mt) * (1 + mt) <= 1920;
}

template <int TYPE>
hipError_t matmul_as(const void* a, const void* b, int64_t m, int64_t n, int64_t k, void* cv, int64_t ldc, hipStream_t s) {
  auto* c = static_cast<typename Elem<TYPE>::type*>(cv);
  if (!k) {
    const int64_t blocks = (m * n + 255) / 256;
    k_zero<TYPE><<<(unsigned)(blocks < 65536 ? blocks : 65536), 256, 0, s>>>(m, n, c, ldc);
    return hipGetLastError();
  }
  const Mx4 qa(a, m, k), qb(b, n, k);
  if (use_skinny(qa, qb))
    return qb.row_tiles < qa.row_tiles ? skinny<-1, TYPE, true>(qa, qb, FullRows{}, c, ldc, s)
                                       : skinny<-1, TYPE, false>(qb, qa, FullRows{}, c, ldc, s);
  const int f = product_side(qa.row_tiles, qb.row_tiles);
  const int64_t tiles = tiles_of(qa, qb, f);
  const unsigned grid = (unsigned)(f == 8 && tiles > kResident ? kResident : tiles);
  if (f == 8)
    k_product<TYPE, 8><<<grid, 256, 0, s>>>(qa, qb, c, ldc);
  else if (f == 4)
    k_product<TYPE, 4><<<grid, 256, 0, s>>>(qa, qb, c, ldc);
  else
    k_product<TYPE, 2><<<grid, 256, 0, s>>>(qa, qb, c, ldc);
  return hipGetLastError();
}

// Two products in one launch of 64 x 64 tiles: a launch saved, and the one fills the CUs that the other leaves.  It
// loses where tiles of 256 or many waves along a long axis are worth more.  us of a layer's gradients (quantisation
// included, replayed from a graph), together / one by one: 256x512x416 7.2 / 11.9, 2048x512x416 10.0 / 11.2 (of a
// call 13.9 / 17.5), 2048x2048x512 15.5 / 18.6, 2048x2048x2048 (2048 tiles) 28.5 / 29.4, 4096x4096x512 (32 steps)
// 38.2 / 40.9; past the lines 4096x2048x2048 45.5 / 42.9, 5000x512x416 (40 steps) 16.8 / 15.6, 16384x64x64 28.1 / 23.2.
constexpr int64_t kTogetherTiles = 2048;  // of both
constexpr int64_t kTogetherSteps = 32;    // column tiles of either
bool together(const Mx4& a1, const Mx4& b1, const Mx4& a2, const Mx4& b2) {
  return tiles_of(a1, b1, 2) + tiles_of(a2, b2, 2) <= kTogetherTiles && a1.col_tiles <= kTogetherSteps &&
         a2.col_tiles <= kTogetherSteps;
}

template <int TYPE1, int TYPE2>
hipError_t two_as(const Mx4& a1, const Mx4& b1, void* c1, int64_t ldc1, const Mx4& a2, const Mx4& b2, void* c2, int64_t ldc2,
                  hipStream_t s) {
  const int64_t t1 = tiles_of(a1, b1, 2), t2 = tiles_of(a2, b2, 2);
  k_two_products<TYPE1, TYPE2><<<(unsigned)(t1 + t2), 256, 0, s>>>(
      a1, b1, static_cast<typename Elem<TYPE1>::type*>(c1), ldc1, (uint32_t)t1, a2, b2,
      static_cast<typename Elem<TYPE2>::type*>(c2), ldc2);
  return hipGetLastError();
}

template <int TYPE1>
hipError_t two_first(const Mx4& a1, const Mx4& b1, void* c1, int64_t ldc1, const Mx4& a2, const Mx4& b2, void* c2, int type2,
                     int64_t ldc2, hipStream_t s) {
  if (type2 == EMB_TYPE_FP32) return two_as<TYPE1, EMB_TYPE_FP32>(a1, b1, c1, ldc1, a2, b2, c2, ldc2, s);
  if (type2 == EMB_TYPE_BF16) return two_as<TYPE1, EMB_TYPE_BF16>(a1, b1, c1, ldc1, a2, b2, c2, ldc2, s);
  return two_as<TYPE1, EMB_TYPE_FP16>(a1, b1, c1, ldc1, a2, b2, c2, ldc2, s);
}

// Rows that every workgroup of k_skinny quantises by itself: few values, and not too many workgroups that do.  It saves
// a launch.  us among other calls, with the quantisation inside / as a launch of its own: 16 rows, 4096 x 4096
// 7.3 / 12.1; 4 rows, 4096 x 12800 9.3 / 11.9; 64 rows, 1000 x 1000 8.3 / 12.1, 8192 x 512 10.7 / 12.1; past the line
// 5 rows, 8192 x 12800 16.8 / 15.1; 64 rows, 16384 x 512 20.2 / 12.3; 16 rows, 16384 x 2048 13.3 / 12.1.
// (Replayed from a graph a launch costs less: 7.7 / 6.4, 10.3 / 10.9, 8.9 / 8.0.)
bool fused(int64_t m, int64_t n, int64_t k) {
  const int64_t values = m * ((k + 511) / 512 * 512);
  return m <= 64 && values <= kFusedValues && values * ((n + kTileRows - 1) / kTileRows) <= (int64_t)1 << 24;
}

}  // namespace

hipError_t launch_matmul(const void* a, const void* b, int64_t m, int64_t n, int64_t k, void* c, int type, int64_t ldc,
                         hipStream_t s) {
  if (type == EMB_TYPE_FP32) return matmul_as<EMB_TYPE_FP32>(a, b, m, n, k, c, ldc, s);
  if (type == EMB_TYPE_BF16) return matmul_as<EMB_TYPE_BF16>(a, b, m, n, k, c, ldc, s);
  return matmul_as<EMB_TYPE_FP16>(a, b, m, n, k, c, ldc, s);
}

hipError_t launch_two_products(const void* a1, const void* b1, int64_t m1, int64_t n1, int64_t k1, void* c1, int type1,
                               int64_t ldc1, const void* a2, const void* b2, int64_t m2, int64_t n2, int64_t k2, void* c2,
                               int type2, int64_t ldc2, hipStream_t s) {
  const Mx4 qa1(a1, m1, k1), qb1(b1, n1, k1), qa2(a2, m2, k2), qb2(b2, n2, k2);
  if (m1 && n1 && k1 && m2 && n2 && k2 && together(qa1, qb1, qa2, qb2)) {
    if (type1 == EMB_TYPE_FP32) return two_first<EMB_TYPE_FP32>(qa1, qb1, c1, ldc1, qa2, qb2, c2, type2, ldc2, s);
    if (type1 == EMB_TYPE_BF16) return two_first<EMB_TYPE_BF16>(qa1, qb1, c1, ldc1, qa2, qb2, c2, type2, ldc2, s);
    return two_first<EMB_TYPE_FP16>(qa1, qb1, c1, ldc1, qa2, qb2, c2, type2, ldc2, s);
  }
  hipError_t e = m1 && n1 ? launch_matmul(a1, b1, m1, n1, k1, c1, type1, ldc1, s) : hipSuccess;
  if (e == hipSuccess && m2 && n2) e = launch_matmul(a2, b2, m2, n2, k2, c2, type2, ldc2, s);
  return e;
}

size_t linear_workspace(int64_t m, int64_t n, int64_t k) {
  return fused(m, n, k) ? 0 : (size_t)Mx4(nullptr, m, k).bytes();
}

hipError_t launch_linear(const void* x, int type, int64_t m, int64_t k, int64_t ldx, const void* w, int64_t n, void* y,
                         int64_t ldy, void* workspace, hipStream_t s) {
  if (k && fused(m, n, k)) {
    const Mx4 qw(w, n, k), qx(nullptr, m, k);
    const FullRows full = {x, ldx};
    if (type == EMB_TYPE_FP32)
      return skinny<EMB_TYPE_FP32, EMB_TYPE_FP32, false>(qw, qx, full, static_cast<float*>(y), ldy, s);
    if (type == EMB_TYPE_BF16)
      return skinny<EMB_TYPE_BF16, EMB_TYPE_BF16, false>(qw, qx, full, static_cast<uint16_t*>(y), ldy, s);
    return skinny<EMB_TYPE_FP16, EMB_TYPE_FP16, false>(qw, qx, full, static_cast<uint16_t*>(y), ldy, s);
  }
  if (k) {
    const hipError_t e = launch_quantize(x, type, m, k, ldx, workspace, nullptr, EMB_ROUND_NEAREST, 0, 0, kStreamMatrix, s);
    if (e != hipSuccess) return e;
  }
  return launch_matmul(workspace, w, m, n, k, y, type, ldy, s);
}

}  // namespace embd
