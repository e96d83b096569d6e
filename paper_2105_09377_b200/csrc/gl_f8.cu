// Operands held in 8 bits (F8): blocks of 128 consecutive values of an item, E4M3 codes and one E8M0 scale per block.
//   * gl_f8_quantize / gl_f8_dequantize: between GL_BF16 / GL_F32 patterns and F8 operands;
//   * gl_cartesian_dot_f8: compute dotProd (cartProd A B) of two F8 operands on the block-scaled tensor-core
//     instructions (tcgen05.mma kind::mxf8f6f4), the scales applied by the hardware;
//   * gl_dense_f8: the same with the left operand quantised by the call.
#include <cuda.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cstring>

#include "gl_f8.cuh"
#include "gl_f8.h"
#include "gl_internal.h"
#include "gl_launch.cuh"
#include "gl_tc.cuh"
#include "gl_tmap.h"

using namespace gl;

namespace {

// ------------------------------------------------------------------------
// Quantisation and its inverse
// ------------------------------------------------------------------------

// A warp takes strips of U consecutive units of a row, R rows one below the other, all requested before the first is used: U * R is
// eight when there are strips enough to fill the machine, and U no larger than a row has units.  Places inside a strip are fixed
// distances, so finding them costs next to nothing.
//
// Bound by HBM: 16384 x 8192 bf16 61 us each way, 6.5 TB/s, fp32 100 us, 6.7 TB/s.  With a division per unit, unpacked arithmetic and
// four units in flight bf16 took 75 us: 170 instructions per unit where 112 are left.  Rows that start anywhere: 8192 x 8191 bf16 42 us
// and 38 back, fp32 55 and 60 (aligned rows of that size 31 and 51); with a branch between the requests 62 and 108 us.
struct F8QuantParams {
  int32_t K, pitch;
  uint32_t kt, rows;
  uint32_t strips;      // strips of U units: row groups * strips of a row
  FastDiv per_row;      // strips of a row
};

template <bool F32, bool VEC, int U, int R>
__global__ void __launch_bounds__(256) quantize_f8(const void* __restrict__ in, uint8_t* __restrict__ codes,
                                                   uint8_t* __restrict__ scale, const F8QuantParams p) {
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31;
  const uint32_t strip = blockIdx.x * 8u + (threadIdx.x >> 5);
  if (strip >= p.strips) return;
  uint32_t group, at;
  p.per_row.divmod(strip, group, at);
  const uint32_t row0 = group * R;
  const int k0 = static_cast<int>(at) * (U * kF8Unit);
  Unit<F32, VEC> held[R * U];
#pragma unroll
  for (int r = 0; r < R; ++r)
    if (row0 + r < p.rows) units_read<F32, VEC, U>(in, LaneAt(row0 + r, p.rows, k0, p.K, lane, F32 ? 4 : 2), held + r * U);
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const uint32_t row = row0 + r;
    if (row >= p.rows) break;
    const LaneAt l(row, p.rows, k0, p.K, lane, F32 ? 4 : 2);
    uint8_t* to = codes + static_cast<int64_t>(row) * p.pitch + k0 + lane * 8;
    uint8_t* scale_to = scale + f8_scale_at(row, at * (2 * U), p.kt);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (k0 + u * kF8Unit >= p.K) break;
      float2 v[4];
      unit_values(held[r * U + u], l, u, v);
      unit_store_f8(v, to, p.pitch - k0 - lane * 8, scale_to, u, lane);
    }
  }
}

// Two codes to two values (exact in fp16).
__device__ __forceinline__ float2 f8_values2(uint32_t two) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<uint16_t>(two)));
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

// Going back, aligned fp32 rows are held as two times four values a lane instead of eight in a row: 16-byte stores next to each
// other.
template <bool F32, bool VEC, int U, int R>
__global__ void __launch_bounds__(256) dequantize_f8(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scale,
                                                     void* __restrict__ out, const F8QuantParams p) {
  constexpr bool kHalves = F32 && VEC;
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31;
  const uint32_t strip = blockIdx.x * 8u + (threadIdx.x >> 5);
  if (strip >= p.strips) return;
  uint32_t group, at;
  p.per_row.divmod(strip, group, at);
  const uint32_t row0 = group * R;
  const int k0 = static_cast<int>(at) * (U * kF8Unit);
  uint32_t word[R * U][2], e[R * U];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const uint32_t row = row0 + r;
    if (row >= p.rows) break;
    const uint8_t* src = codes + static_cast<int64_t>(row) * p.pitch + k0;
    const uint8_t* scale_at = scale + f8_scale_at(row, at * (2 * U), p.kt);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      uint32_t(&w)[2] = word[r * U + u];
      w[0] = w[1] = 0;
      if (k0 + u * kF8Unit >= p.K) break;
      e[r * U + u] = *reinterpret_cast<const uint16_t*>(scale_at + (u >> 1) * 512 + (u & 1) * 2);
      if (kHalves) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
          if (k0 + u * kF8Unit + h * 128 + lane * 4 < p.K)
            w[h] = __ldcs(reinterpret_cast<const uint32_t*>(src + lane * 4 + u * kF8Unit + h * 128));
      } else if (k0 + u * kF8Unit + lane * 8 < p.pitch) {
        const uint2 x = __ldcs(reinterpret_cast<const uint2*>(src + lane * 8 + u * kF8Unit));
        w[0] = x.x;
        w[1] = x.y;
      }
    }
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const uint32_t row = row0 + r;
    if (row >= p.rows) break;
    const LaneAt l(row, p.rows, k0, p.K, lane, F32 ? 4 : 2);
    float* o = static_cast<float*>(out) + static_cast<int64_t>(row) * p.K + k0 + lane * 4;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (k0 + u * kF8Unit >= p.K) break;
      const float s0 = f8_scale(e[r * U + u] & 255u), s1 = f8_scale(e[r * U + u] >> 8), mine = lane < 16 ? s0 : s1;
      float2 v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float s = kHalves ? (i < 2 ? s0 : s1) : mine;
        v[i] = mul2(f8_values2(i & 1 ? word[r * U + u][i >> 1] >> 16 : word[r * U + u][i >> 1] & 0xFFFFu), make_float2(s, s));
      }
      if (kHalves) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
          if (k0 + u * kF8Unit + h * 128 + lane * 4 < p.K)
            __stcs(reinterpret_cast<float4*>(o + u * kF8Unit + h * 128), make_float4(v[2 * h].x, v[2 * h].y, v[2 * h + 1].x, v[2 * h + 1].y));
      } else {
        unit_store<F32, VEC>(v, out, l, u, lane);
      }
    }
  }
}

// Rows of up to 128 values, several side by side: with a unit per row half of a warp's lanes or more would have nothing to do
// (327680 x 128 bf16 42 -> 22 us, x 64 41 -> 13, x 96 41 -> 21, x 8 40 -> 4.0, fp32 x 128 62 -> 33; 2560 x 128 1.6 -> 1.4).
template <bool F32, int U>
__global__ void __launch_bounds__(256) quantize_f8_short(const void* __restrict__ in, uint8_t* __restrict__ codes,
                                                         uint8_t* __restrict__ scale, const ShortRows r) {
  pdl_wait();
  pdl_launch_dependents();
  Unit<F32, true> held[U];
#pragma unroll
  for (int u = 0; u < U; ++u) short_read(in, r, ShortAt(r, U, u), held[u]);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float2 v[4];
    short_values(held[u], v);
    short_store_f8(v, codes, scale, r, ShortAt(r, U, u));
  }
}

// Going back, fp32 rows are held as two times four values a lane, half a row apart: 16-byte stores next to each other (327680 x 128
// 33 us; eight values in a row 46; a unit per row 33, x 64 30 -> 18).  bf16 rows 29 -> 21, x 64 29 -> 12.
template <bool F32, int U>
__global__ void __launch_bounds__(256) dequantize_f8_short(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scale,
                                                           void* __restrict__ out, const ShortRows r) {
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & (r.lanes - 1);
  const int k0 = F32 ? lane * 4 : lane * 8, k1 = F32 ? (r.lanes + lane) * 4 : k0 + 4;
  uint32_t word[U][2], e[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const ShortAt at(r, U, u);
    word[u][0] = word[u][1] = e[u] = 0;
    if (at.row >= r.rows) continue;
    const uint8_t* from = codes + static_cast<int64_t>(at.row) * r.pitch;
    if (F32) {
      if (k0 < r.K) word[u][0] = __ldcs(reinterpret_cast<const uint32_t*>(from + k0));
      if (k1 < r.K) word[u][1] = __ldcs(reinterpret_cast<const uint32_t*>(from + k1));
    } else if (k0 < r.K) {
      const uint2 both = __ldcs(reinterpret_cast<const uint2*>(from + k0));
      word[u][0] = both.x;
      word[u][1] = both.y;
    }
    e[u] = scale[f8_scale_at(at.row, 0, 1)];
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const ShortAt at(r, U, u);
    const float s = f8_scale(e[u]);
    float2 v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t w = word[u][i / 2];
      v[i] = mul2(f8_values2(i & 1 ? w >> 16 : w & 0xFFFFu), make_float2(s, s));
    }
    if (!F32) {
      short_store<false>(v, out, r, at);
    } else if (at.row < r.rows) {
      float* to = static_cast<float*>(out) + static_cast<int64_t>(at.row) * r.K;
      if (k0 < r.K) *reinterpret_cast<float4*>(to + k0) = make_float4(v[0].x, v[0].y, v[1].x, v[1].y);
      if (k1 < r.K) *reinterpret_cast<float4*>(to + k1) = make_float4(v[2].x, v[2].y, v[3].x, v[3].y);
    }
  }
}

// Units of a strip and rows of a warp: eight units in flight, four where rows are unaligned (a unit takes half as many registers
// again, and more).
struct StripPlan { int units, rows; };

F8QuantParams f8_quant_params(const F8View& v, StripPlan* plan) {
  const int64_t units = (v.nb + 1) / 2;
  // several units a warp only when every SM has blocks to hold
  const bool many = v.rows * units >= static_cast<int64_t>(num_sms()) * 4 * 8 * 8;
  plan->units = 1;
  const int most = v.K % 8 ? 4 : 8;
  while (many && plan->units < most && plan->units < units) plan->units *= 2;
  plan->rows = many ? most / plan->units : 1;
  F8QuantParams p;
  p.K = static_cast<int32_t>(v.K);
  p.pitch = static_cast<int32_t>(v.pitch);
  p.kt = static_cast<uint32_t>(v.kt);
  p.rows = static_cast<uint32_t>(v.rows);
  const int64_t per_row = (units + plan->units - 1) / plan->units;
  p.strips = static_cast<uint32_t>((v.rows + plan->rows - 1) / plan->rows * per_row);
  p.per_row.set(per_row);
  return p;
}

typedef void (*QuantizeFn)(const void*, uint8_t*, uint8_t*, F8QuantParams);
typedef void (*DequantizeFn)(const uint8_t*, const uint8_t*, void*, F8QuantParams);

template <bool F32, bool VEC>
QuantizeFn quantize_fn(const StripPlan& s) {
  constexpr int kMost = VEC ? 8 : 4;
  if (s.rows == 1 && s.units == 1) return quantize_f8<F32, VEC, 1, 1>;
  switch (s.units) {
    case 1: return quantize_f8<F32, VEC, 1, kMost>;
    case 2: return quantize_f8<F32, VEC, 2, kMost / 2>;
    case 4: return quantize_f8<F32, VEC, 4, kMost / 4>;
    default: return quantize_f8<F32, VEC, kMost, 1>;
  }
}
template <bool F32, bool VEC>
DequantizeFn dequantize_fn(const StripPlan& s) {
  constexpr int kMost = VEC ? 8 : 4;
  if (s.rows == 1 && s.units == 1) return dequantize_f8<F32, VEC, 1, 1>;
  switch (s.units) {
    case 1: return dequantize_f8<F32, VEC, 1, kMost>;
    case 2: return dequantize_f8<F32, VEC, 2, kMost / 2>;
    case 4: return dequantize_f8<F32, VEC, 4, kMost / 4>;
    default: return dequantize_f8<F32, VEC, kMost, 1>;
  }
}

int launch_quantize(const gl_ap& in, const F8View& v, void* codes, void* scale, cudaStream_t st) {
  const bool f32 = in.dtype == GL_F32, vec = v.K % 8 == 0;
  if (is_short(v)) {
    const ShortRows r = short_rows(v);
    const int groups = short_groups(r, num_sms());
    void (*k)(const void*, uint8_t*, uint8_t*, ShortRows) = groups == 4 ? (f32 ? quantize_f8_short<true, 4> : quantize_f8_short<false, 4>)
                                                                        : (f32 ? quantize_f8_short<true, 1> : quantize_f8_short<false, 1>);
    return launch_pdl(k, dim3(short_blocks(r, groups)), dim3(256), 0, st, 1, static_cast<const void*>(in.data), static_cast<uint8_t*>(codes),
                      static_cast<uint8_t*>(scale), r) == cudaSuccess ? GL_OK : GL_ERR_CUDA;
  }
  StripPlan s;
  const F8QuantParams p = f8_quant_params(v, &s);
  const QuantizeFn k = f32 ? (vec ? quantize_fn<true, true>(s) : quantize_fn<true, false>(s))
                           : (vec ? quantize_fn<false, true>(s) : quantize_fn<false, false>(s));
  return launch_pdl(k, dim3((p.strips + 7) / 8), dim3(256), 0, st, 1, static_cast<const void*>(in.data), static_cast<uint8_t*>(codes),
                    static_cast<uint8_t*>(scale), p) == cudaSuccess ? GL_OK : GL_ERR_CUDA;
}

// ------------------------------------------------------------------------
// Block-scaled product
// ------------------------------------------------------------------------

// out[m,o] = sum over blocks b of 2^(ea[m,b] + eb[o,b] - 254) sum_k a[m,k] b[o,k]: the inner products of E4M3 codes, their
// scaling and the fp32 sum are one instruction, tcgen05.mma kind::mxf8f6f4, which wants a scale for every 32 values; the four
// instructions of a block read the same scale byte.  An instruction cuts each of its 32 products to 2^-25 of the largest term (the
// sum so far is one) and their sum toward zero to fp32 (seen with whole numbers around 2^24): 32 * 2^-25 + 2^-23 = 9 * 2^-23 of the
// magnitudes are lost at worst, K 2^-24.8 after K values.  Of the results' root mean square, against fp32 sums of a library: normal
// values, 1024^3 0.6e-7 and 0.4e-7, 4096^3 2.2e-7 and 0.8e-7, 8192^3 5.0e-7 and 1.3e-7; values of one sign come out low, on the
// average by 1.8e-7, 1.4e-6 and 3.9e-6.
//
// What bounds it at size is operands from L2 to the SMs and, beyond a few milliseconds, the power limit: 256 x 256 tiles on a pair
// of SMs need 64 bytes per cycle and SM.  bf16 results, us: 4096^3 50 to 55 (2.7 to 2.5 PFLOP/s; a last round of 34 of 74 pairs),
// 8192^3 361 (3.04), 16384 x 8192 x 8192 727 (3.02) in a run of milliseconds and 830 to 890 (2.65 to 2.5) for seconds on end.
// The measured bf16 rate of the same card, doubled: 3.2 and 2.8.  fp32 results 4096^3 57 us, 68 among other passes.

// D[tmem] (+)= (A * sfa)[smem] * (B * sfb)[smem]^T, K = 32, one scale per row and instruction.
template <int CTAS>
__device__ __forceinline__ void tc_mma_f8(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t sfa, uint32_t sfb,
                                          uint32_t accumulate) {
  if (CTAS == 2)
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory");
}

// One scale tile (32 rows x 16 bytes of shared memory) into four columns of tensor memory, repeated in the four lane
// quarters.  Copies and MMAs of one thread run in the order of their issue.
template <int CTAS>
__device__ __forceinline__ void tc_copy_scales(uint32_t taddr, uint64_t desc) {
  if (CTAS == 2) asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
  else asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}

// Instruction descriptor, kind::mxf8f6f4: A and B E4M3 (bits 7-9 and 10-12 = 0), both K-major, N >> 3 at bit 17, scales E8M0
// (bit 23), M >> 4 at bit 24; which of the four scale bytes of a row the instruction reads: bits 4-5 (B), 29-30 (A).
__device__ __forceinline__ uint32_t make_idesc_f8(int m, int n, uint32_t byte) {
  return (byte << 4) | (static_cast<uint32_t>(n >> 3) << 17) | (1u << 23) | (static_cast<uint32_t>(m >> 4) << 24) | (byte << 29);
}

// relu that lets a NaN through (fmaxf would turn it into 0)
__device__ __forceinline__ float relu_keep_nan(float v) { return v < 0.f ? 0.f : v; }

constexpr int kTile = 128;           // rows of A per block
constexpr int kKBytes = 128;         // bytes of a row per K block: one block of 128 values, one 128-byte swizzle row
constexpr int kF8Threads = 352;      // warp 0 TMA (A), warp 1 MMA, warps 2-9 epilogue, warp 10 TMA (B)
constexpr int kEpiWarps = 8;         // two per quarter of the rows, taking turns at the columns
constexpr int kFewThreads = 224;     // warp 0 TMA (weights), warp 1 MMA, warps 2-5 sums (2-6 round A), warp 6 TMA (A)

// Tile rows of a band, in 256s.  What a band of pairs reads at a time is its rows of A and a few columns of B: 16 rows by 4 or 5
// columns for 74 pairs.  Walked row by row, the whole of B passes for every two rows of tiles, and what does not come from near
// L2 costs power, which is what bounds a long run: 16384 x 8192 x 8192 sustained 930 us with one row, 870 with four, 855 with
// eight, 840 with sixteen, 865 with 24, 930 with 32, 1030 with 64; 8192^3 468, 436, 425, 412, 433 (24), 466 (32).
constexpr int kBandRows = 16;

// K blocks that one accumulator adds up (65536 values), a multiple of the four of a scale tile; a longer K is cut into such
// stretches, which are added with rounding to nearest.  One accumulator would lose what lies 2^-25 below it, of 2^20 small products
// behind a large one up to 2 %.  us with one accumulator / with stretches, bf16 results: 1 x 2^20 x 8192 1352 / 1350, 64 x 2^20 x 2048
// 415 / 420, 128 x 2^20 x 4096 1004 / 1221, 300 x 2^20 x 512 379 / 409, 4096 x 2^17 x 4096 1580 / 2005 (on 128 x 128 tiles).
constexpr int kStretch = 512;

struct F8Params {
  int64_t M, O;
  int tiles_m, tiles_n;   // tiles_m counts 128 * CTAS rows
  int kblocks;            // K blocks of 128 values
  int last_steps;         // instructions (32 values) in the last K block
  int relu, out_bf16, tma_store;
  int group;              // tiles are walked in bands of `group` tile rows, column by column inside a band
  FastDiv div_band, div_group, div_last;   // tiles of a band; tile rows of a band, of the last band
  // Place of tile u.
  __device__ __forceinline__ void tile_at(int u, uint32_t& tm, uint32_t& tn) const {
    uint32_t band, in_band, row;
    div_band.divmod(static_cast<uint32_t>(u), band, in_band);
    const bool last = static_cast<int>(band + 1) * group > tiles_m;
    (last ? div_last : div_group).divmod(in_band, tn, row);
    tm = band * group + row;
  }
};

template <int BN, int CTAS>
struct F8Cfg {
  static constexpr int kStageA = kTile * kKBytes;
  static constexpr int kStageB = (BN / CTAS) * kKBytes;
  static constexpr int kStage = kStageA + kStageB;
  // A scale tile holds four K blocks: every fourth stage brings one per 128 rows of A and of B.
  static constexpr int kScaleA = 512, kScaleB = (BN / 128) * 512, kScales = kScaleA + kScaleB;
  static constexpr int kEpiBytes = kEpiWarps * 4096;
  static constexpr int kStages = (232448 - kEpiBytes - 1024 - 256) / (kStage + kScales);
  static constexpr int kSmemBytes = kStages * (kStage + kScales) + kEpiBytes + 1024 + 256;
  // Tensor memory (512 columns): two sets of scales in the last kSfCols, two accumulators of BN columns before them.
  // 256-wide accumulators do not fit twice: they share kSfCols columns, which the epilogue empties first.
  static constexpr int kSfCols = 8 + BN / 16;
  static constexpr int kSfBase = 512 - kSfCols;
  static constexpr int kAcc1 = 2 * BN <= kSfBase ? BN : kSfBase - BN;
  static constexpr bool kOverlap = kAcc1 < BN;
};

__device__ __forceinline__ void tc_store_32cols(uint32_t taddr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};"
      ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
        "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]),
        "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]),
        "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(taddr)
      : "memory");
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}

// A stretch's 32 columns `r` added to those before if there are any (`add`), and put where the next stretch finds them.
__device__ __forceinline__ void add_stretch(uint32_t taddr, uint32_t (&r)[32], bool add, bool keep) {
  if (add) {
    uint32_t before[32];
    tc_load_32cols(taddr, before);
#pragma unroll
    for (int j = 0; j < 32; ++j) r[j] = __float_as_uint(__uint_as_float(before[j]) + __uint_as_float(r[j]));
  }
  if (keep) tc_store_32cols(taddr, r);
}

// Up to 32 rows that the epilogue has staged (128 bytes a row, 16-byte pieces exchanged as the 128-byte swizzle does) to rows of O
// results that are no multiples of 16 bytes: row by row, neighbouring lanes on neighbouring columns, sixteen rows read from shared
// memory before the first is stored.  KIND 0: fp32, 1: bf16 in whole pairs (O even), 2: bf16 one by one.
template <int KIND>
__device__ __forceinline__ void store_rows(uint32_t buf, char* to, int64_t O, int rows, int cols, int lane) {
  const int col = KIND ? 2 * lane : lane;
  const bool one = col < cols, two = KIND == 2 && col + 1 < cols;
  const int64_t pitch = O * (KIND ? 2 : 4);
  const uint32_t from = buf + (lane & 3) * 4;
  to += col * (KIND ? 2 : 4);
#pragma unroll
  for (int row0 = 0; row0 < 32; row0 += 16) {
    uint32_t v[16];
#pragma unroll
    for (int i = 0; i < 16; ++i)
      asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v[i]) : "r"(from + (row0 + i) * 128 + (((lane >> 2) ^ (i & 7)) << 4)));
    if (row0 + 16 <= rows) {
#pragma unroll
      for (int i = 0; i < 16; ++i, to += pitch) {
        if (KIND < 2) {
          if (one) *reinterpret_cast<uint32_t*>(to) = v[i];
        } else {
          if (one) *reinterpret_cast<uint16_t*>(to) = static_cast<uint16_t>(v[i]);
          if (two) *reinterpret_cast<uint16_t*>(to + 2) = static_cast<uint16_t>(v[i] >> 16);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i, to += pitch) {
        const bool in = row0 + i < rows;
        if (KIND < 2) {
          if (one && in) *reinterpret_cast<uint32_t*>(to) = v[i];
        } else {
          if (one && in) *reinterpret_cast<uint16_t*>(to) = static_cast<uint16_t>(v[i]);
          if (two && in) *reinterpret_cast<uint16_t*>(to + 2) = static_cast<uint16_t>(v[i] >> 16);
        }
      }
    }
  }
}

// LONG: more K blocks than a stretch.  Accumulators change with every stretch as they do from tile to tile, and the epilogue adds
// them up in columns of their own.
template <int BN, int CTAS, bool LONG>
__global__ void __launch_bounds__(kF8Threads, 1)
dot_f8(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
       const __grid_constant__ CUtensorMap map_sa, const __grid_constant__ CUtensorMap map_sb,
       const __grid_constant__ CUtensorMap map_c, void* __restrict__ out, const F8Params p) {
  using Cfg = F8Cfg<BN, CTAS>;
  static_assert(Cfg::kStages >= 2, "ring too shallow");
  static_assert(!LONG || 3 * BN <= Cfg::kSfBase, "two accumulators and their sum");
  extern __shared__ unsigned char smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t tiles = (raw + 1023u) & ~1023u;   // the 128-byte swizzle wants 1024-byte aligned tiles
  unsigned char* gen_tiles = smem_raw + (tiles - raw);
  const uint32_t epi_base = tiles + Cfg::kStages * Cfg::kStage;
  const uint32_t scales = epi_base + Cfg::kEpiBytes;
  uint64_t* bars = reinterpret_cast<uint64_t*>(gen_tiles + Cfg::kStages * (Cfg::kStage + Cfg::kScales) + Cfg::kEpiBytes);
  const uint32_t bar_full = smem_u32(bars);
  const uint32_t bar_empty = bar_full + 8 * Cfg::kStages;
  const uint32_t bar_tfull = bar_empty + 8 * Cfg::kStages;
  const uint32_t bar_tempty = bar_tfull + 16;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * Cfg::kStages + 4);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = CTAS == 2 ? cluster_ctarank() : 0u;

  if (threadIdx.x == 32) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map_a)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map_b)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map_sa)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map_sb)) : "memory");
    if (p.tma_store) asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map_c)) : "memory");
  }
  if (threadIdx.x == 0) {
    for (int s = 0; s < Cfg::kStages; ++s) { mbar_init(bar_full + 8 * s, 2); mbar_init(bar_empty + 8 * s, 1); }
    for (int a = 0; a < 2; ++a) { mbar_init(bar_tfull + 8 * a, 1); mbar_init(bar_tempty + 8 * a, kEpiWarps * CTAS); }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    if (CTAS == 2) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(tmem_slot)) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(tmem_slot)) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  tc_fence_before();
  if (CTAS == 2) cluster_sync_all();
  else __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  const int num_tiles = p.tiles_m * p.tiles_n;
  const int unit0 = static_cast<int>(blockIdx.x) / CTAS, unit_step = static_cast<int>(gridDim.x) / CTAS;
  pdl_wait();
  pdl_launch_dependents();

  if (warp == 0 || warp == 10) {
    // ---------------- TMA producers: warp 0 stages A and its scales, warp 10 stages B and its scales ----------------
    const bool load_a = warp == 0;
    const bool leader = elect_one();
    uint32_t s = 0, ph = 0;
    bool ok = true;
    for (int u = unit0; u < num_tiles && ok; u += unit_step) {
      uint32_t tm, tn;
      p.tile_at(u, tm, tn);
      const int m0 = (static_cast<int>(tm) * CTAS + static_cast<int>(rank)) * kTile;
      const int n0 = static_cast<int>(tn) * BN + static_cast<int>(rank) * (BN / CTAS);
      for (int kb = 0; kb < p.kblocks; ++kb) {
        if (!mbar_wait(bar_empty + 8 * s, ph ^ 1u, abort_flag)) { ok = false; break; }
        const uint32_t full = CTAS == 2 ? map_to_cta(bar_full + 8 * s, 0) : bar_full + 8 * s;
        const uint32_t stage = tiles + s * Cfg::kStage;
        const uint32_t sc = scales + s * Cfg::kScales;
        const bool with_scales = (kb & 3) == 0;
        if (rank == 0 && leader)
          mbar_expect_tx(bar_full + 8 * s, CTAS * (load_a ? Cfg::kStageA + (with_scales ? Cfg::kScaleA : 0)
                                                          : Cfg::kStageB + (with_scales ? Cfg::kScaleB : 0)));
        if (leader) {
          if (load_a) {
            if (CTAS == 2) tma_load_2d_pair(stage, &map_a, kb * kKBytes, m0, full);
            else tma_load_2d(stage, &map_a, kb * kKBytes, m0, full);
            if (with_scales) {
              if (CTAS == 2) tma_load_3d_pair(sc, &map_sa, 0, kb >> 2, m0 / 128, full);
              else tma_load_3d(sc, &map_sa, 0, kb >> 2, m0 / 128, full);
            }
          } else {
            if (CTAS == 2) tma_load_2d_pair(stage + Cfg::kStageA, &map_b, kb * kKBytes, n0, full);
            else tma_load_2d(stage + Cfg::kStageA, &map_b, kb * kKBytes, n0, full);
            if (with_scales) {   // every block of a pair holds the scales of all BN columns
#pragma unroll
              for (int h = 0; h < BN / 128; ++h) {
                const uint32_t dst = sc + Cfg::kScaleA + h * 512;
                const int rt = static_cast<int>(tn) * (BN / 128) + h;
                if (CTAS == 2) tma_load_3d_pair(dst, &map_sb, 0, kb >> 2, rt, full);
                else tma_load_3d(dst, &map_sb, 0, kb >> 2, rt, full);
              }
            }
          }
        }
        if (++s == Cfg::kStages) { s = 0; ph ^= 1u; }
      }
    }
  } else if (warp == 1) {
    // ---------------- MMA issuer ----------------
    if (rank == 0) {
      const bool leader = elect_one();
      const uint64_t desc_a0 = make_desc(tiles, 16, 1024, 2);
      const uint64_t desc_b0 = make_desc(tiles + Cfg::kStageA, 16, 1024, 2);
      const uint64_t desc_s0 = make_desc(scales, 16, 128, 0);
      uint32_t s = 0, ph = 0, tile_it = 0, sets = 0;
      bool ok = true;
      for (int u = unit0; u < num_tiles && ok; u += unit_step) {
        int kb0 = 0;
        do {
          const uint32_t acc = tile_it & 1u;
          // separate accumulators: the one two tiles back has been read; overlapping ones: the shared columns of the
          // previous tile have been read (its epilogue had then finished with the tile before)
          const uint32_t wait_on = Cfg::kOverlap ? acc ^ 1u : acc;
          const uint32_t round = Cfg::kOverlap ? (tile_it + 1) >> 1 : tile_it >> 1;
          if (!mbar_wait(bar_tempty + 8 * wait_on, (round & 1u) ^ 1u, abort_flag)) { ok = false; break; }
          tc_fence_after();
          const uint32_t d_tmem = tmem_base + (acc ? Cfg::kAcc1 : 0);
          uint32_t sfa = 0, sfb = 0;
          const int kb1 = LONG ? min(kb0 + kStretch, p.kblocks) : p.kblocks;
          for (int kb = kb0; kb < kb1; ++kb) {
            if (!mbar_wait(bar_full + 8 * s, ph, abort_flag)) { ok = false; break; }
            tc_fence_after();
            const uint64_t da0 = desc_a0 + ((s * Cfg::kStage) >> 4);
            const uint64_t db0 = desc_b0 + ((s * Cfg::kStage) >> 4);
            if ((kb & 3) == 0) {   // the scales of four K blocks, into the set that the four before do not use
              sfa = tmem_base + Cfg::kSfBase + (sets & 1u) * 4;
              sfb = tmem_base + Cfg::kSfBase + 8 + (sets & 1u) * (BN / 32);
              ++sets;
              if (leader) {
                const uint64_t ds0 = desc_s0 + ((s * Cfg::kScales) >> 4);
                tc_copy_scales<CTAS>(sfa, ds0);
#pragma unroll
                for (int h = 0; h < BN / 128; ++h) tc_copy_scales<CTAS>(sfb + 4 * h, ds0 + ((Cfg::kScaleA + h * 512) >> 4));
              }
            }
            const uint32_t idesc = make_idesc_f8(kTile * CTAS, BN, kb & 3);
            const int steps = kb + 1 == p.kblocks ? p.last_steps : 4;
#pragma unroll
            for (int k = 0; k < 4; ++k)
              if (k < steps && leader) tc_mma_f8<CTAS>(d_tmem, da0 + 2 * k, db0 + 2 * k, idesc, sfa, sfb, ((kb - kb0) | k) != 0 ? 1u : 0u);
            if (leader) {
              if (CTAS == 2) tc_commit_pair(bar_empty + 8 * s);
              else tc_commit(bar_empty + 8 * s);
            }
            if (++s == Cfg::kStages) { s = 0; ph ^= 1u; }
          }
          if (ok && leader) {
            if (CTAS == 2) tc_commit_pair(bar_tfull + 8 * acc);
            else tc_commit(bar_tfull + 8 * acc);
          }
          ++tile_it;
          kb0 = kb1;
        } while (LONG && ok && kb0 < p.kblocks);
      }
    }
  } else {
    // ---------------- epilogue: TMEM -> registers -> (shared memory -> TMA store | global) ----------------
    const int q = warp & 3, turn = (warp - 2) >> 2;
    const bool leader = elect_one();
    uint32_t tile_it = 0;
    bool ok = true;
    const uint32_t buf = epi_base + (warp - 2) * 4096;
    const int cstep = p.out_bf16 ? 64 : 32;
    const int nchunks = BN / cstep;
    for (int u = unit0; u < num_tiles && ok; u += unit_step) {
      uint32_t tmu, tn;
      p.tile_at(u, tmu, tn);
      const int tm = static_cast<int>(tmu) * CTAS + static_cast<int>(rank);
      int kb0 = 0;
      do {
        const uint32_t acc = tile_it & 1u, aph = (tile_it >> 1) & 1u;
        const bool more = LONG && kb0 + kStretch < p.kblocks;   // stretches of this tile are still to come
        if (!mbar_wait(bar_tfull + 8 * acc, aph, abort_flag)) { ok = false; break; }
        tc_fence_after();
        const uint32_t taddr = tmem_base + (acc ? Cfg::kAcc1 : 0) + (static_cast<uint32_t>(q * 32) << 16);
        const uint32_t tmem_sum = tmem_base + 2 * BN + (static_cast<uint32_t>(q * 32) << 16);
        const int64_t m0 = static_cast<int64_t>(tm) * kTile + q * 32;
#pragma unroll 1
        for (int i = turn; i < nchunks; i += 2) {
          // the columns that two overlapping accumulators share go first: the last ones of the first, the first ones
          // of the second (all in the first chunk: the warps of the second turn give theirs back with their first)
          const int c = (Cfg::kOverlap && acc == 0 ? nchunks - 1 - i : i) * cstep;
          const int64_t n0 = static_cast<int64_t>(tn) * BN + c;
          uint32_t r[32];
          tc_load_32cols(taddr + c, r);
          if (LONG) add_stretch(tmem_sum + c, r, kb0 > 0, more);
          if (p.relu && !more) {
#pragma unroll
            for (int j = 0; j < 32; ++j) r[j] = __float_as_uint(relu_keep_nan(__uint_as_float(r[j])));
          }
          if (p.out_bf16) {
#pragma unroll
            for (int j = 0; j < 16; ++j) r[j] = pack_bf16x2(r[2 * j], r[2 * j + 1]);
            uint32_t r2[32];
            tc_load_32cols(taddr + c + 32, r2);
            if (LONG) add_stretch(tmem_sum + c + 32, r2, kb0 > 0, more);
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              float a = __uint_as_float(r2[2 * j]), b = __uint_as_float(r2[2 * j + 1]);
              if (p.relu) { a = relu_keep_nan(a); b = relu_keep_nan(b); }
              r[16 + j] = pack_bf16x2(__float_as_uint(a), __float_as_uint(b));
            }
          }
          if (Cfg::kOverlap ? i == turn : i + 2 >= nchunks) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
              if (CTAS == 2) mbar_arrive_remote(map_to_cta(bar_tempty + 8 * acc, 0));
              else mbar_arrive(bar_tempty + 8 * acc);
            }
          }
          if (more || n0 >= p.O) continue;   // uniform across the warp
          if (p.tma_store && leader) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
          __syncwarp();
#pragma unroll
          for (int j = 0; j < 8; ++j)
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(buf + lane * 128 + ((j ^ (lane & 7)) << 4)),
                         "r"(r[4 * j]), "r"(r[4 * j + 1]), "r"(r[4 * j + 2]), "r"(r[4 * j + 3])
                         : "memory");
          if (p.tma_store) {
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (leader) {
              if (m0 < p.M)
                asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];" ::"l"(
                                 reinterpret_cast<uint64_t>(&map_c)),
                             "r"(static_cast<int>(n0)), "r"(static_cast<int>(m0)), "r"(buf)
                             : "memory");
              asm volatile("cp.async.bulk.commit_group;" ::: "memory");
            }
          } else {
            __syncwarp();
            const int rows = static_cast<int>(min(static_cast<int64_t>(32), p.M - m0));
            const int cols = static_cast<int>(min(static_cast<int64_t>(cstep), p.O - n0));
            if (!p.out_bf16) store_rows<0>(buf, static_cast<char*>(out) + (m0 * p.O + n0) * 4, p.O, rows, cols, lane);
            else if (p.O & 1) store_rows<2>(buf, static_cast<char*>(out) + (m0 * p.O + n0) * 2, p.O, rows, cols, lane);
            else store_rows<1>(buf, static_cast<char*>(out) + (m0 * p.O + n0) * 2, p.O, rows, cols, lane);
          }
        }
        ++tile_it;
        kb0 += kStretch;
      } while (LONG && kb0 < p.kblocks);
    }
    if (p.tma_store && leader) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
  }

  // teardown: a block that gave up lets its copies in flight land before it leaves
  __syncwarp();
  if (*abort_flag) {
    const uint64_t t0 = global_timer();
    while (global_timer() - t0 < 20000000ull) { }
  }
  tc_fence_before();
  if (CTAS == 2) cluster_sync_all();
  else __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    if (CTAS == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem_base) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem_base) : "memory");
  }
}

// ------------------------------------------------------------------------
// Few rows of A: the weights take the 128-row side
// ------------------------------------------------------------------------
//
// With few rows of A the product is bound by reading B (the weights) once.  Tiles of 128 rows of B, BN rows of A (16 to 128) as the N
// side, and K cut over the S blocks of a cluster so that the loads of all SMs are in flight: the blocks' partial sums meet in
// distributed shared memory, added in rank order.  One tile per block, two blocks per SM.  While the kernel that makes A is
// still running the first weights are on their way into L2.
// Weights that come from HBM: 8192 x 8192 one row 13.3 us (67 MB: 5.1 TB/s, of which filling and emptying the machine takes 3 us),
// 64 rows 15.8, 128 rows 18.7; 28672 x 8192 one row 36.4 us, 6.5 TB/s, the rate of a copy.
//
// A few rows of a dense layer (FUSED): the blocks round A themselves, each its own stretch of K, straight into operand order, while
// the first weights are on their way: one launch.  Five warps take four K blocks of a row at a time; up to two rounds of that cost
// less than a launch of its own.  us fused / not, weights of 8192 x 8192 and 4096 x 14336 not in L2:
//   K x O            1 row          2 rows         4 rows         5 rows         6 rows         8 rows
//   1024 x 1024      3.5 / 4.5      3.5 / 4.4      3.6 / 4.6      3.6 / 4.6      4.3 / 4.6      4.3 / 4.6     (1, 1, 1, 1, 2, 2 rounds)
//   3136 x 1000      4.1 / 5.0      4.1 / 5.0      4.1 / 5.1      4.1 / 5.2      4.8 / 5.2      4.8 / 5.1     (1, 1, 1, 1, 2, 2)
//   4096 x 4096      6.3 / 6.7      6.3 / 6.8      6.6 / 7.0      6.7 / 7.0      7.4 / 7.1      8.2 / 7.2     (1, 1, 2, 2, 3, 4)
//   8192 x 8192     13.7 / 15.4    14.4 / 15.6    15.5 / 15.7    15.7 / 15.7    16.5 / 15.9    17.9 / 15.9    (1, 2, 4, 4, 5, 7)
//   4096 x 14336    13.1 / 14.5    13.7 / 14.5    14.9 / 14.8    15.3 / 14.8    15.9 / 14.8    17.2 / 14.8    (1, 2, 4, 4, 5, 7)
constexpr int kFuseRows = 8;
constexpr int kFuseBlocks = 16;   // K blocks of A that a block has room for
constexpr int kFuseWarps = 5, kFuseRounds = 2;
// K blocks that a block asks for before the kernel in front has ended.  More stand in the way of the rows of A behind them, and of
// weights that are wanted sooner: one row, weights not in L2, 8192 x 8192: none 14.2 us, two 13.6, four 13.5, all sixteen 14.1;
// 8192 x 28672: none to eight 37.5, all 53.8; 128 rows through 8192 x 8192: none 19.6, four 19.0, all 20.3.
constexpr int kPrefetch = 4;
constexpr int kJoinWarps = kFewThreads / 32;
// Eight rows of A a K block, 1024 bytes: the instruction's other eight columns read the block behind and are not used.
constexpr int kXBlock = 8 * kKBytes;

struct F8FewParams {
  int64_t M, O;
  int tiles_o;            // tiles of 128 rows of B; a tile of rows of A goes with every one of them
  const void* x;          // FUSED: rows of A as they came
  int64_t K;
  int x_f32;
  int kblocks, last_steps;
  int split;              // blocks per cluster
  int relu, out_bf16;
};

// The S partial sums of a value in rank order.  A warp takes a column of 128 outputs, four a lane; rank r has the columns r, r + S, ..,
// several of a warp's requested before the first is summed.
template <int S>
__device__ __forceinline__ void join_ranks(uint32_t part, int rank, int warp, int lane, int64_t o0, int64_t m0, int rows, void* __restrict__ out,
                                           const F8FewParams& p) {
  constexpr int kCols = 8 / S < 1 ? 1 : 8 / S;   // columns of a warp in flight
  const int64_t o = o0 + lane * 4;
  for (int c0 = rank + warp * S; c0 < rows; c0 += kCols * kJoinWarps * S) {
    float4 x[kCols][S];
#pragma unroll
    for (int j = 0; j < kCols; ++j)
#pragma unroll
      for (int from = 0; from < S; ++from) {
        const int c = c0 + j * kJoinWarps * S;
        if (c < rows)
          asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                       : "=f"(x[j][from].x), "=f"(x[j][from].y), "=f"(x[j][from].z), "=f"(x[j][from].w)
                       : "r"(map_to_cta(part + c * 512 + lane * 16, from)));
      }
#pragma unroll
    for (int j = 0; j < kCols; ++j) {
      const int c = c0 + j * kJoinWarps * S;
      if (c >= rows) break;
      float v[4] = {x[j][0].x, x[j][0].y, x[j][0].z, x[j][0].w};
#pragma unroll
      for (int from = 1; from < S; ++from) { v[0] += x[j][from].x; v[1] += x[j][from].y; v[2] += x[j][from].z; v[3] += x[j][from].w; }
      if (p.relu) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = relu_keep_nan(v[i]);
      }
      if (p.out_bf16) {
        uint16_t* to = static_cast<uint16_t*>(out) + (m0 + c) * p.O + o;
        const uint32_t lo = pack_bf16x2(__float_as_uint(v[0]), __float_as_uint(v[1])), hi = pack_bf16x2(__float_as_uint(v[2]), __float_as_uint(v[3]));
        if ((p.O & 3) == 0) {
          if (o < p.O) *reinterpret_cast<uint2*>(to) = make_uint2(lo, hi);
        } else {
          if (o < p.O) to[0] = static_cast<uint16_t>(lo);
          if (o + 1 < p.O) to[1] = static_cast<uint16_t>(lo >> 16);
          if (o + 2 < p.O) to[2] = static_cast<uint16_t>(hi);
          if (o + 3 < p.O) to[3] = static_cast<uint16_t>(hi >> 16);
        }
      } else {
        float* to = static_cast<float*>(out) + (m0 + c) * p.O + o;
        if ((p.O & 3) == 0) {
          if (o < p.O) *reinterpret_cast<float4*>(to) = make_float4(v[0], v[1], v[2], v[3]);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (o + i < p.O) to[i] = v[i];
        }
      }
    }
  }
}

template <int BN, bool FUSED>
struct F8FewCfg {
  static constexpr int kStageA = kTile * kKBytes;                  // weights
  static constexpr int kStageB = FUSED ? 0 : BN * kKBytes;
  static constexpr int kStage = kStageA + kStageB;
  static constexpr int kScales = FUSED ? 512 : 1024;               // a scale tile (four K blocks) of each side
  static constexpr int kXTiles = kFuseBlocks / 4 + 1;              // FUSED: scale tiles that a stretch of K blocks touches
  static constexpr int kXBytes = FUSED ? (kFuseBlocks + 1) * kXBlock + kXTiles * 512 : 0;
  static constexpr int kStages = (112 * 1024 - 1024 - 256 - kXBytes) / (kStage + kScales);
  static constexpr int kSmemBytes = kStages * (kStage + kScales) + kXBytes + 1024 + 256;
  static constexpr int kTmemCols = BN + 16 <= 32 ? 32 : BN + 16 <= 64 ? 64 : BN + 16 <= 128 ? 128 : 256;
  static constexpr int kSfBase = kTmemCols - 16;                   // two sets of four columns of each side
  static_assert(kStages >= 2 && kStages * kStage >= BN * 128 * 4, "partial sums fit in the ring");
  static_assert(!FUSED || BN == 16, "the instruction's columns are two groups of eight");
};

// Sixteen values of a row of A from element k on, zeros behind its end.
__device__ __forceinline__ void load_row_values(const F8FewParams& p, int m, int64_t k, float (&x)[16]) {
  const int64_t at = static_cast<int64_t>(m) * p.K + k, left = p.K - k;
  if (left >= 16 && (p.K & 7) == 0) {
    if (p.x_f32) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float4 a = *(reinterpret_cast<const float4*>(static_cast<const float*>(p.x) + at) + i);
        x[4 * i] = a.x; x[4 * i + 1] = a.y; x[4 * i + 2] = a.z; x[4 * i + 3] = a.w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint4 a = *(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.x) + at) + i);
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          x[8 * i + 2 * j] = __uint_as_float(w[j] << 16);
          x[8 * i + 2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
        }
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      x[i] = i < left ? (p.x_f32 ? static_cast<const float*>(p.x)[at + i] : bf16_to_f32(static_cast<const uint16_t*>(p.x)[at + i])) : 0.f;
  }
}

// Eight lanes round a K block of row m, sixteen values each, into the swizzled operand row and the scale tiles.
__device__ __forceinline__ void round_row_block(const float (&x)[16], unsigned char* rows, unsigned char* scale, int m, int lane8, bool live) {
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) top = top_of(top, x[i]);
#pragma unroll
  for (int d = 1; d < 8; d *= 2) top = top_of(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
  if (!live) return;
  const uint32_t e = f8_exponent(__float_as_uint(top) & 0x7FFFFFFFu);
  const float f = f8_inverse(e);
  uint32_t word[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) word[i] = e == 255u ? 0u : f8_codes4(x[4 * i] * f, x[4 * i + 1] * f, x[4 * i + 2] * f, x[4 * i + 3] * f);
  *reinterpret_cast<uint4*>(rows + m * 128 + ((lane8 ^ (m & 7)) << 4)) = make_uint4(word[0], word[1], word[2], word[3]);
  if (lane8 == 0) *scale = static_cast<uint8_t>(e);
}

// LONG: a rank has more K blocks than a stretch; the epilogue's warps add the stretches up in registers, the MMAs wait meanwhile (once
// in 65536 values).
template <int BN, bool FUSED, bool LONG>
__global__ void __launch_bounds__(kFewThreads, LONG && BN == 128 ? 1 : 2)
dot_f8_few(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x,
           const __grid_constant__ CUtensorMap map_sw, const __grid_constant__ CUtensorMap map_sx, void* __restrict__ out,
           const F8FewParams p) {
  using Cfg = F8FewCfg<BN, FUSED>;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t tiles = (raw + 1023u) & ~1023u;
  unsigned char* gen_tiles = smem_raw + (tiles - raw);
  const uint32_t xs = tiles + Cfg::kStages * Cfg::kStage;            // FUSED: A, block by block, then its scale tiles
  unsigned char* gen_x = gen_tiles + Cfg::kStages * Cfg::kStage;
  const uint32_t scales = xs + Cfg::kXBytes;
  uint64_t* bars = reinterpret_cast<uint64_t*>(gen_x + Cfg::kXBytes + Cfg::kStages * Cfg::kScales);
  const uint32_t bar_full = smem_u32(bars), bar_empty = bar_full + 8 * Cfg::kStages, bar_done = bar_empty + 8 * Cfg::kStages,
                 bar_x = bar_done + 8, bar_read = bar_x + 8;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * Cfg::kStages + 3);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = p.split > 1 ? static_cast<int>(cluster_ctarank()) : 0;
  const int unit = static_cast<int>(blockIdx.x) / p.split, xt = unit / p.tiles_o, tile = unit - xt * p.tiles_o;
  const int64_t m0 = static_cast<int64_t>(xt) * BN;
  const int rows = static_cast<int>(min(static_cast<int64_t>(BN), p.M - m0));
  // K blocks of this rank, as even as they go
  const int kb0 = static_cast<int>(static_cast<int64_t>(p.kblocks) * rank / p.split);
  const int kb1 = static_cast<int>(static_cast<int64_t>(p.kblocks) * (rank + 1) / p.split);

  if (warp == 0 && elect_one())
    for (int kb = kb0; kb < min(kb1, kb0 + kPrefetch); ++kb) tma_prefetch_2d(&map_w, kb * kKBytes, tile * kTile);
  if (threadIdx.x == 0) {
    for (int s = 0; s < Cfg::kStages; ++s) { mbar_init(bar_full + 8 * s, FUSED ? 1 : 2); mbar_init(bar_empty + 8 * s, 1); }
    mbar_init(bar_done, 1);
    mbar_init(bar_x, kFuseWarps);   // warps 2 to 6
    mbar_init(bar_read, 4);         // warps 2 to 5
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)),
                 "r"(static_cast<uint32_t>(Cfg::kTmemCols)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  pdl_wait();
  pdl_launch_dependents();

  if (FUSED && warp >= 2) {
    // a warp takes four K blocks of a row at a time, eight lanes each
    const int quads = (kb1 - kb0 + 3) / 4;
    unsigned char* xscale = gen_x + (kFuseBlocks + 1) * kXBlock;
    int m = 0, g = warp - 2;
    while (true) {
      while (g >= quads) { g -= quads; ++m; }
      if (m >= rows) break;
      const int b = g * 4 + (lane >> 3), kb = kb0 + b;
      float x[16];
      load_row_values(p, m, static_cast<int64_t>(kb) * kF8Block + (lane & 7) * 16, x);
      round_row_block(x, gen_x + b * kXBlock, xscale + ((kb >> 2) - (kb0 >> 2)) * 512 + m * 16 + (kb & 3), m, lane & 7, kb < kb1);
      g += kFuseWarps;
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (lane == 0) mbar_arrive(bar_x);
  }
  if (warp == 0 || (warp == 6 && !FUSED)) {
    const bool load_w = warp == 0;
    const bool leader = elect_one();
    uint32_t s = 0, ph = 0;
    for (int kb = kb0; kb < kb1; ++kb) {
      if (!mbar_wait(bar_empty + 8 * s, ph ^ 1u, abort_flag)) break;
      const uint32_t full = bar_full + 8 * s, stage = tiles + s * Cfg::kStage, sc = scales + s * Cfg::kScales;
      const bool with_scales = kb == kb0 || (kb & 3) == 0;
      if (leader) {
        mbar_expect_tx(full, (load_w ? Cfg::kStageA : Cfg::kStageB) + (with_scales ? 512 : 0));
        if (load_w) {
          tma_load_2d(stage, &map_w, kb * kKBytes, tile * kTile, full);
          if (with_scales) tma_load_3d(sc, &map_sw, 0, kb >> 2, tile, full);
        } else {
          tma_load_2d(stage + Cfg::kStageA, &map_x, kb * kKBytes, static_cast<int>(m0), full);
          if (with_scales) tma_load_3d(sc + 512, &map_sx, 0, kb >> 2, static_cast<int>(m0 >> 7), full);
        }
      }
      if (++s == Cfg::kStages) { s = 0; ph ^= 1u; }
    }
  } else if (warp == 1) {
    const bool leader = elect_one();
    const uint64_t desc_w0 = make_desc(tiles, 16, 1024, 2), desc_x0 = make_desc(FUSED ? xs : tiles + Cfg::kStageA, 16, 1024, 2);
    const uint64_t desc_s0 = make_desc(scales, 16, 128, 0);
    const uint64_t desc_sx0 = make_desc(FUSED ? xs + (kFuseBlocks + 1) * kXBlock : scales + 512, 16, 128, 0);
    uint32_t s = 0, ph = 0, sets = 0, sfw = 0;
    bool ok = !FUSED || mbar_wait(bar_x, 0, abort_flag);
    int first = kb0, reads = 0;   // of the stretch; accumulators read so far
    for (int kb = kb0; kb < kb1 && ok; ++kb) {
      if (LONG && kb == first + kStretch) {
        if (leader) tc_commit(bar_done);
        if (!mbar_wait(bar_read, reads++ & 1, abort_flag)) { ok = false; break; }
        tc_fence_after();
        first = kb;
      }
      if (!mbar_wait(bar_full + 8 * s, ph, abort_flag)) { ok = false; break; }
      tc_fence_after();
      const uint64_t off = (s * Cfg::kStage) >> 4, xoff = FUSED ? ((kb - kb0) * kXBlock) >> 4 : off;
      if (kb == kb0 || (kb & 3) == 0) {
        sfw = tmem_base + Cfg::kSfBase + (sets & 1u) * 4;
        ++sets;
        if (leader) {
          tc_copy_scales<1>(sfw, desc_s0 + ((s * Cfg::kScales) >> 4));
          tc_copy_scales<1>(sfw + 8, desc_sx0 + ((FUSED ? ((kb >> 2) - (kb0 >> 2)) * 512 : s * Cfg::kScales) >> 4));
        }
      }
      const uint32_t idesc = make_idesc_f8(kTile, BN, kb & 3);
      const int steps = kb + 1 == p.kblocks ? p.last_steps : 4;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (k < steps && leader)
          tc_mma_f8<1>(tmem_base, desc_w0 + off + 2 * k, desc_x0 + xoff + 2 * k, idesc, sfw, sfw + 8, kb != first || k != 0 ? 1u : 0u);
      if (leader) tc_commit(bar_empty + 8 * s);
      if (++s == Cfg::kStages) { s = 0; ph ^= 1u; }
    }
    if (ok && leader) tc_commit(bar_done);
  }
  float* part = reinterpret_cast<float*>(gen_tiles);   // [BN][128]: every MMA has read the ring when bar_done flips
  if (warp >= 2 && warp < 6) {
    const int q = warp & 3;
    float total[LONG ? BN : 1];
    int reads = 0;
    if (LONG) {   // all stretches but the last
#pragma unroll
      for (int c = 0; c < BN; ++c) total[LONG ? c : 0] = 0.f;
      for (int kb = kb0 + kStretch; kb < kb1; kb += kStretch) {
        if (!mbar_wait(bar_done, reads++ & 1, abort_flag)) break;
        tc_fence_after();
#pragma unroll
        for (int c = 0; c < BN; c += 16) {
          uint32_t r[16];
          tc_load_16cols(tmem_base + (static_cast<uint32_t>(q * 32) << 16) + c, r);
#pragma unroll
          for (int j = 0; j < 16; ++j) total[LONG ? c + j : 0] += __uint_as_float(r[j]);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_read);
      }
    }
    const bool ok = mbar_wait(bar_done, reads & 1, abort_flag);
    tc_fence_after();
    if (LONG && ok) {
#pragma unroll
      for (int c = 0; c < BN; c += 16) {
        if (c >= rows) break;
        uint32_t r[16];
        tc_load_16cols(tmem_base + (static_cast<uint32_t>(q * 32) << 16) + c, r);
#pragma unroll
        for (int j = 0; j < 16; ++j) part[(c + j) * 128 + q * 32 + lane] = total[LONG ? c + j : 0] + __uint_as_float(r[j]);
      }
    } else if (ok) {
#pragma unroll 1
      for (int c = 0; c < BN; c += 16) {
        if (c >= rows) break;
        uint32_t r[16];
        tc_load_16cols(tmem_base + (static_cast<uint32_t>(q * 32) << 16) + c, r);
#pragma unroll
        for (int j = 0; j < 16; ++j) part[(c + j) * 128 + q * 32 + lane] = __uint_as_float(r[j]);
      }
    }
    tc_fence_before();
  }
  __syncwarp();
  if (p.split > 1) cluster_sync_all();
  else __syncthreads();
  const int64_t o0 = static_cast<int64_t>(tile) * kTile;
  switch (p.split) {
    case 1: join_ranks<1>(smem_u32(part), rank, warp, lane, o0, m0, rows, out, p); break;
    case 2: join_ranks<2>(smem_u32(part), rank, warp, lane, o0, m0, rows, out, p); break;
    case 4: join_ranks<4>(smem_u32(part), rank, warp, lane, o0, m0, rows, out, p); break;
    default: join_ranks<8>(smem_u32(part), rank, warp, lane, o0, m0, rows, out, p); break;
  }
  __syncwarp();
  if (*abort_flag) {   // copies in flight land before the block leaves
    const uint64_t t0 = global_timer();
    while (global_timer() - t0 < 20000000ull) { }
  }
  if (p.split > 1) cluster_sync_all();   // the other ranks have read this block's sums
  else __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base),
                 "r"(static_cast<uint32_t>(Cfg::kTmemCols)) : "memory");
  }
}

// ---- host side ----

// Tensor maps are encoded on every call: 0.05 us each, no more than looking one up.
bool encode(CUtensorMap* m, CUtensorMapDataType dt, cuuint32_t rank, const void* base, const cuuint64_t* dims, const cuuint64_t* strides,
            const cuuint32_t* box, CUtensorMapSwizzle swz, CUtensorMapL2promotion l2) {
  const cuuint32_t estr[3] = {1, 1, 1};
  return driver_api().tiled(m, dt, rank, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, swz, l2,
                            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct F8Operand { const void* codes; const void* scale; F8View v; };

bool encode_codes(CUtensorMap* m, const F8Operand& a, int box_rows) {
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(a.v.pitch), static_cast<cuuint64_t>(a.v.rows)};
  const cuuint64_t strides[1] = {static_cast<cuuint64_t>(a.v.pitch)};
  const cuuint32_t box[2] = {kKBytes, static_cast<cuuint32_t>(box_rows)};
  return encode(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, a.codes, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B,
                CU_TENSOR_MAP_L2_PROMOTION_L2_256B);
}

// Scale tiles as (128 words, tiles along K, tiles along the rows), one tile a box.  Tiles past the end read as zeros.
bool encode_scales(CUtensorMap* m, const F8Operand& a) {
  const cuuint64_t dims[3] = {128, static_cast<cuuint64_t>(a.v.kt), static_cast<cuuint64_t>(a.v.rt)};
  const cuuint64_t strides[2] = {512, static_cast<cuuint64_t>(a.v.kt) * 512};
  const cuuint32_t box[3] = {128, 1, 1};
  return encode(m, CU_TENSOR_MAP_DATA_TYPE_UINT32, 3, a.scale, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_NONE,
                CU_TENSOR_MAP_L2_PROMOTION_L2_128B);
}

bool encode_out(CUtensorMap* m, void* base, int64_t M, int64_t O, bool bf16) {
  const cuuint64_t es = bf16 ? 2 : 4;
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(O), static_cast<cuuint64_t>(M)};
  const cuuint64_t strides[1] = {static_cast<cuuint64_t>(O) * es};
  const cuuint32_t box[2] = {bf16 ? 64u : 32u, 32};
  return encode(m, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 2, base, dims, strides, box,
                CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_NONE);
}

// Instructions of 32 values along K: in K blocks of four, the last one as far as it goes.
void k_steps(int64_t K, int* kblocks, int* last_steps) {
  const int64_t steps = (K + 31) / 32;
  *kblocks = static_cast<int>((steps + 3) / 4);
  *last_steps = static_cast<int>(steps - 4 * static_cast<int64_t>(*kblocks - 1));
}

struct TilePlanF8 {
  CUtensorMap ma, mb, msa, msb, mc;
  F8Params p;
  void* out;
  int grid;
};

template <int BN, int CTAS, bool LONG>
int plan_tiles(const F8Operand& a, const F8Operand& b, void* out, uint32_t flags, TilePlanF8* t) {
  using Cfg = F8Cfg<BN, CTAS>;
  static std::atomic<int> resident[64];   // per device, 0: not asked yet (threads may ask at once: the calls are idempotent)
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return GL_ERR_CUDA;
  int at_once = resident[dev].load(std::memory_order_acquire);
  if (!at_once) {
    if (cudaFuncSetAttribute(dot_f8<BN, CTAS, LONG>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg::kSmemBytes) != cudaSuccess)
      return GL_ERR_CUDA;
    at_once = num_sms();
    if (CTAS == 2) {   // SMs pair up within a GPC: a persistent grid must not exceed what is resident at once
      cudaLaunchConfig_t cfg;
      std::memset(&cfg, 0, sizeof(cfg));
      cudaLaunchAttribute at;
      std::memset(&at, 0, sizeof(at));
      at.id = cudaLaunchAttributeClusterDimension;
      at.val.clusterDim.x = CTAS;
      at.val.clusterDim.y = at.val.clusterDim.z = 1;
      cfg.gridDim = dim3(static_cast<unsigned>(num_sms() / 2 * 2));
      cfg.blockDim = dim3(kF8Threads);
      cfg.dynamicSmemBytes = Cfg::kSmemBytes;
      cfg.attrs = &at;
      cfg.numAttrs = 1;
      if (cudaOccupancyMaxActiveClusters(&at_once, dot_f8<BN, CTAS, LONG>, &cfg) != cudaSuccess || at_once < 1) return GL_ERR_CUDA;
      at_once = std::min(at_once, num_sms() / 2);
    }
    resident[dev].store(at_once, std::memory_order_release);
  }
  F8Params& p = t->p;
  p.M = a.v.rows;
  p.O = b.v.rows;
  p.tiles_m = static_cast<int>((p.M + kTile * CTAS - 1) / (kTile * CTAS));
  p.tiles_n = static_cast<int>((p.O + BN - 1) / BN);
  if (static_cast<int64_t>(p.tiles_m) * p.tiles_n > (1 << 30)) return GL_ERR_UNSUPPORTED;
  k_steps(a.v.K, &p.kblocks, &p.last_steps);
  p.relu = (flags & GL_EPILOGUE_RELU) ? 1 : 0;
  p.out_bf16 = (flags & GL_OUT_BF16) ? 1 : 0;
  p.tma_store = p.O % (p.out_bf16 ? 8 : 4) == 0 ? 1 : 0;
  p.group = kBandRows;
  if (p.group > p.tiles_m) p.group = p.tiles_m;
  p.div_band.set(static_cast<int64_t>(p.group) * p.tiles_n);
  p.div_group.set(p.group);
  p.div_last.set(p.tiles_m % p.group ? p.tiles_m % p.group : p.group);
  t->out = out;
  t->grid = CTAS * std::min(at_once, p.tiles_m * p.tiles_n);
  if (!encode_codes(&t->ma, a, kTile) || !encode_codes(&t->mb, b, BN / CTAS) || !encode_scales(&t->msa, a) ||
      !encode_scales(&t->msb, b))
    return GL_ERR_CUDA;
  t->mc = t->ma;   // unused without TMA stores; any valid map
  if (p.tma_store && !encode_out(&t->mc, out, p.M, p.O, p.out_bf16 != 0)) return GL_ERR_CUDA;
  return GL_OK;
}

template <int BN, int CTAS, bool LONG>
int run_tiles(const TilePlanF8& t, cudaStream_t st) {
  return launch_pdl(dot_f8<BN, CTAS, LONG>, dim3(static_cast<unsigned>(t.grid)), dim3(kF8Threads), F8Cfg<BN, CTAS>::kSmemBytes, st, CTAS,
                    t.ma, t.mb, t.msa, t.msb, t.mc, t.out, t.p) == cudaSuccess ? GL_OK : GL_ERR_CUDA;
}

struct FewPlanF8 {
  CUtensorMap mw, mx, msw, msx;
  F8FewParams p;
  void* out;
  int grid;
};

// Blocks that share a tile's K.  Half the machine is filled as long as a rank keeps two K blocks, the rest as long as it keeps four
// (eight for clusters of eight, which the hardware then packs two to an SM beside empty ones), and a second block per SM where it
// keeps sixteen: joining costs 1 to 3 us.  us at half / at this many / at twice as many ranks: 64 x 1024 x 1024 4.7 / 4.4 / 4.8;
// 64 x 2048 x 2048 5.4 / 4.9 / 5.7; 128 x 4096 x 4096 - / 9.8 / 11.9; 1 x 8192 x 8192 14.4 / 13.4 / -; 256 x 4096 x 1024 - / 7.1 / 8.9;
// 512 x 8192 x 2048 16.8 / 15.5 / -.
int few_split(int64_t tiles, int kblocks) {
  int split = 1;
  while (split < 8) {
    const int64_t blocks = tiles * split * 2;
    const int left = kblocks / (split * 2);   // K blocks of a rank
    const int need = 2 * blocks <= num_sms() ? 2 : blocks <= num_sms() ? (split == 4 ? 8 : 4) : blocks <= 2 * num_sms() ? 16 : INT32_MAX;
    if (left < need) break;
    split *= 2;
  }
  return split;
}

// `FUSED`: A is still to be rounded, by the product's own blocks.
template <int BN, bool FUSED, bool LONG>
int plan_few(const F8Operand& a, const F8Operand& b, void* out, uint32_t flags, FewPlanF8* t) {
  static std::atomic<bool> attr_set[64];   // per device (threads may set it at once: the call is idempotent)
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return GL_ERR_CUDA;
  if (!attr_set[dev].load(std::memory_order_acquire)) {
    if (cudaFuncSetAttribute(dot_f8_few<BN, FUSED, LONG>, cudaFuncAttributeMaxDynamicSharedMemorySize, F8FewCfg<BN, FUSED>::kSmemBytes) !=
        cudaSuccess)
      return GL_ERR_CUDA;
    attr_set[dev].store(true, std::memory_order_release);
  }
  F8FewParams& p = t->p;
  p.M = a.v.rows;
  p.O = b.v.rows;
  p.x = nullptr;
  p.K = a.v.K;
  p.x_f32 = 0;
  k_steps(a.v.K, &p.kblocks, &p.last_steps);
  p.relu = (flags & GL_EPILOGUE_RELU) ? 1 : 0;
  p.out_bf16 = (flags & GL_OUT_BF16) ? 1 : 0;
  const int64_t all = b.v.rt * ((a.v.rows + BN - 1) / BN);
  if (all > (1 << 27)) return GL_ERR_UNSUPPORTED;
  const int tiles = static_cast<int>(all);
  p.tiles_o = static_cast<int>(b.v.rt);
  p.split = few_split(tiles, p.kblocks);
  t->out = out;
  t->grid = tiles * p.split;
  if (!encode_codes(&t->mw, b, kTile) || !encode_scales(&t->msw, b)) return GL_ERR_CUDA;
  t->mx = t->mw;   // unused when FUSED; any valid map
  t->msx = t->msw;
  return FUSED || (encode_codes(&t->mx, a, BN) && encode_scales(&t->msx, a)) ? GL_OK : GL_ERR_CUDA;
}

template <int BN, bool FUSED, bool LONG>
int run_few(const FewPlanF8& t, cudaStream_t st) {
  return launch_pdl(dot_f8_few<BN, FUSED, LONG>, dim3(static_cast<unsigned>(t.grid)), dim3(kFewThreads), F8FewCfg<BN, FUSED>::kSmemBytes, st,
                    t.p.split, t.mw, t.mx, t.msw, t.msx, t.out, t.p) == cudaSuccess ? GL_OK : GL_ERR_CUDA;
}

template <int BN, typename Pre>
int product_few(const F8Operand& a, const F8Operand& b, gl_ap* out, uint32_t flags, cudaStream_t st, Pre&& pre) {
  FewPlanF8 t;
  int rc = plan_few<BN, false, false>(a, b, out->data, flags, &t);
  if (rc) return rc;
  const bool long_k = t.p.kblocks > t.p.split * kStretch;   // of the longest rank
  if (long_k) rc = plan_few<BN, false, true>(a, b, out->data, flags, &t);
  if (rc) return rc;
  rc = pre();
  if (rc) return rc;
  return long_k ? run_few<BN, false, true>(t, st) : run_few<BN, false, false>(t, st);
}

// Checks shared by the two products: shapes, result, aliasing rules are the caller's.
int check_product(const gl_ap* out, int a_access, const int64_t* a_shape, int a_compute, const gl_f8* a1, uint32_t flags) {
  if (flags & ~(GL_EPILOGUE_RELU | GL_OUT_BF16)) return GL_ERR_UNSUPPORTED;
  if (a_compute != a1->ndim - a1->access_ndim) return GL_ERR_SHAPE;
  for (int i = 0; i < a_compute; ++i)
    if (a_shape[a_access + i] != a1->shape[a1->access_ndim + i]) return GL_ERR_SHAPE;
  if (a_access + a1->access_ndim > GL_MAX_DIMS) return GL_ERR_NDIM;
  gl_ap want;
  std::memset(&want, 0, sizeof(want));
  want.dtype = (flags & GL_OUT_BF16) ? GL_BF16 : GL_F32;
  for (int i = 0; i < a_access; ++i) want.shape[want.ndim++] = a_shape[i];
  for (int i = 0; i < a1->access_ndim; ++i) want.shape[want.ndim++] = a1->shape[i];
  want.access_ndim = want.ndim;
  const int rc = check_same_meta(want, out);
  if (rc) return rc;
  return check_data(out);
}

// Product of two operands that have been checked; everything that can fail does so before `pre` enqueues anything.
template <typename Pre>
int product(const F8Operand& a, const F8Operand& b, gl_ap* out, uint32_t flags, cudaStream_t st, Pre&& pre) {
  if (!driver_api().ok) return GL_ERR_CUDA;
  if (a.v.rows <= 16) return product_few<16>(a, b, out, flags, st, pre);
  if (a.v.rows <= 32) return product_few<32>(a, b, out, flags, st, pre);
  if (a.v.rows <= 64) return product_few<64>(a, b, out, flags, st, pre);
  // More rows: K is cut over clusters where there are few tiles for its length, and a second block per SM saves a round of up to
  // 128 rows.  us cut / on the tiles below: 128 x 1024 x 1024 5.4 / 5.0; 128 x 2048 x 512 5.7 / 6.7; 512 x 2048 x 2048 7.1 / 7.2;
  // 128 x 4096 x 4096 9.7 / 12.0, 256 rows 11.9 / 12.2, 384 rows 13.7 / 12.5; 128 x 4096 x 14336 16.9 / 14.9; 256 x 8192 x 8192
  // 21.8 / 22.2, 384 rows 33 / 28; 512 x 14336 x 4096 32.2 / 32.9; 128 x 8192 x 28672 45 / 48, 129 rows 75 / 56.
  const int64_t tiles128 = ((a.v.rows + 127) / 128) * b.v.rt;
  if ((2 * tiles128 <= num_sms() && a.v.nb >= 16) || (tiles128 <= num_sms() && a.v.nb >= 64) ||
      (a.v.rows <= 128 && tiles128 > num_sms() && tiles128 <= 2 * num_sms()))
    return product_few<128>(a, b, out, flags, st, pre);
  // 256 x 256 tiles on pairs of SMs move half the bytes per flop of 128 x 128 tiles, but there are a quarter as many.
  TilePlanF8 t;
  const bool long_k = a.v.nb > kStretch;
  const auto tiles = [&](int64_t side) { return ((a.v.rows + side - 1) / side) * ((b.v.rows + side - 1) / side); };
  const auto rounds = [](int64_t n, int64_t at_once) { return (n + at_once - 1) / at_once; };
  const bool pairs = 3 * rounds(tiles(256), num_sms() / 2) <= 2 * rounds(tiles(128), num_sms());
  // (Two 256-wide accumulators leave no room for the sum of a long K's stretches.)
  const auto plan = long_k ? plan_tiles<128, 1, true> : pairs ? plan_tiles<256, 2, false> : plan_tiles<128, 1, false>;
  const auto run = long_k ? run_tiles<128, 1, true> : pairs ? run_tiles<256, 2, false> : run_tiles<128, 1, false>;
  int rc = plan(a, b, out->data, flags, &t);
  if (rc) return rc;
  rc = pre();
  if (rc) return rc;
  return run(t, st);
}

size_t round_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

// The left operand of a dense layer, as the call holds it in its workspace.
gl_f8 rounded_left(const gl_ap* a0) {
  gl_f8 q;
  std::memset(&q, 0, sizeof(q));
  q.ndim = a0->ndim;
  q.access_ndim = a0->access_ndim;
  for (int i = 0; i < a0->ndim; ++i) q.shape[i] = a0->shape[i];
  return q;
}

}  // namespace

namespace gl {
int take_status_f8() {
  unsigned int v = 0;
  if (cudaMemcpyFromSymbol(&v, g_status, sizeof(v)) != cudaSuccess) return GL_ERR_CUDA;
  if (!v) return GL_OK;
  const unsigned int zero = 0;
  if (cudaMemcpyToSymbol(g_status, &zero, sizeof(zero)) != cudaSuccess) return GL_ERR_CUDA;
  return GL_ERR_TIMEOUT;
}
}  // namespace gl

extern "C" {

size_t gl_f8_data_bytes(const gl_f8* a) {
  F8View v;
  return check_f8_meta(a, &v) ? 0 : static_cast<size_t>(v.rows) * v.pitch;
}

size_t gl_f8_scale_bytes(const gl_f8* a) {
  F8View v;
  return check_f8_meta(a, &v) ? 0 : static_cast<size_t>(v.rt) * v.kt * 512;
}

int gl_f8_quantize(const gl_ap* in, gl_f8* out, void* stream) {
  int rc = check_data(in);
  if (rc) return rc;
  F8View v;
  rc = check_f8_data(out, &v);
  if (rc) return rc;
  if (!f8_same_shape(in, out)) return GL_ERR_SHAPE;
  return launch_quantize(*in, v, out->data, out->scale, static_cast<cudaStream_t>(stream));
}

int gl_f8_dequantize(const gl_f8* in, gl_ap* out, void* stream) {
  F8View v;
  int rc = check_f8_data(in, &v);
  if (rc) return rc;
  rc = check_data(out);
  if (rc) return rc;
  if (!f8_same_shape(out, in)) return GL_ERR_SHAPE;
  const bool f32 = out->dtype == GL_F32, vec = v.K % 8 == 0;
  if (is_short(v)) {
    const ShortRows r = short_rows(v);
    const int groups = short_groups(r, num_sms());
    void (*k)(const uint8_t*, const uint8_t*, void*, ShortRows) =
        groups == 4 ? (f32 ? dequantize_f8_short<true, 4> : dequantize_f8_short<false, 4>)
                    : (f32 ? dequantize_f8_short<true, 1> : dequantize_f8_short<false, 1>);
    return launch_pdl(k, dim3(short_blocks(r, groups)), dim3(256), 0, static_cast<cudaStream_t>(stream), 1,
                      static_cast<const uint8_t*>(in->data), static_cast<const uint8_t*>(in->scale), out->data, r) == cudaSuccess
               ? GL_OK : GL_ERR_CUDA;
  }
  StripPlan s;
  const F8QuantParams p = f8_quant_params(v, &s);
  const DequantizeFn k = f32 ? (vec ? dequantize_fn<true, true>(s) : dequantize_fn<true, false>(s))
                             : (vec ? dequantize_fn<false, true>(s) : dequantize_fn<false, false>(s));
  return launch_pdl(k, dim3((p.strips + 7) / 8), dim3(256), 0, static_cast<cudaStream_t>(stream), 1,
                    static_cast<const uint8_t*>(in->data), static_cast<const uint8_t*>(in->scale), out->data, p) == cudaSuccess
             ? GL_OK : GL_ERR_CUDA;
}

int gl_cartesian_dot_f8(const gl_f8* a0, const gl_f8* a1, gl_ap* out, uint32_t flags, void* stream) {
  F8Operand a, b;
  int rc = check_f8_data(a0, &a.v);
  if (rc) return rc;
  rc = check_f8_data(a1, &b.v);
  if (rc) return rc;
  rc = check_product(out, a0->access_ndim, a0->shape, a0->ndim - a0->access_ndim, a1, flags);
  if (rc) return rc;
  a.codes = a0->data;
  a.scale = a0->scale;
  b.codes = a1->data;
  b.scale = a1->scale;
  return product(a, b, out, flags, static_cast<cudaStream_t>(stream), [] { return GL_OK; });
}

size_t gl_dense_f8_workspace(const gl_ap* a0, const gl_f8* a1) {
  F8View v;
  if (check_meta(a0) || check_f8_meta(a1, &v)) return 0;
  const gl_f8 q = rounded_left(a0);
  return round_up(gl_f8_data_bytes(&q), 1024) + gl_f8_scale_bytes(&q);
}

int gl_dense_f8(const gl_ap* a0, const gl_f8* a1, gl_ap* out, uint32_t flags, void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check_data(a0);
  if (rc) return rc;
  F8Operand a, b;
  rc = check_f8_data(a1, &b.v);
  if (rc) return rc;
  rc = check_product(out, a0->access_ndim, a0->shape, a0->ndim - a0->access_ndim, a1, flags);
  if (rc) return rc;
  gl_f8 q = rounded_left(a0);
  rc = check_f8_meta(&q, &a.v);
  if (rc) return rc;
  const size_t need = gl_dense_f8_workspace(a0, a1);
  if (!workspace || workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 1023u)) return GL_ERR_WORKSPACE;
  q.data = workspace;
  q.scale = static_cast<char*>(workspace) + round_up(gl_f8_data_bytes(&q), 1024);
  b.codes = a1->data;
  b.scale = a1->scale;
  a.codes = q.data;
  a.scale = q.scale;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (a.v.rows <= kFuseRows) {
    if (!driver_api().ok) return GL_ERR_CUDA;
    FewPlanF8 t;
    rc = plan_few<16, true, false>(a, b, out->data, flags, &t);
    if (rc) return rc;
    const int blocks = (t.p.kblocks + t.p.split - 1) / t.p.split;
    const int items = static_cast<int>(a.v.rows) * ((blocks + 3) / 4);
    if (blocks <= kFuseBlocks && items <= kFuseWarps * kFuseRounds) {
      t.p.x = a0->data;
      t.p.x_f32 = a0->dtype == GL_F32;
      return run_few<16, true, false>(t, st);
    }
  }
  return product(a, b, out, flags, st, [&] { return launch_quantize(*a0, a.v, q.data, q.scale, st); });
}

}  // extern "C"
