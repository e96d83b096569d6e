// Operands held in 4 bits (MX4): blocks of 32 consecutive values of an item, E2M1 codes and one E8M0 scale per block.
//   * gl_mx4_quantize / gl_mx4_dequantize: between GL_BF16 / GL_F32 patterns and MX4 operands;
//   * gl_cartesian_dot_mx4: compute dotProd (cartProd A B) of two MX4 operands on the block-scaled tensor-core
//     instructions (tcgen05.mma kind::mxf4), the scales applied by the hardware;
//   * gl_dense_mx4: the same with the left operand quantised by the call.
//
// Storage.  Codes: one row per item, two codes a byte (even index in the low half), rows of 16-byte multiples, the
// last block filled with zeros.  Scales: tiles of 128 rows x 4 blocks (512 bytes), row r and block b of a tile at
// byte (r % 32) * 16 + (r / 32) * 4 + b: exactly what one tcgen05.cp (32x128b, replicated to the four lane
// quarters) has to find in shared memory, so that a tile goes global -> shared -> tensor memory untouched.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cstring>

#include "gl_f8.h"
#include "gl_internal.h"
#include "gl_launch.cuh"
#include "gl_mx4.cuh"
#include "gl_tc.cuh"
#include "gl_tmap.h"

using namespace gl;

namespace {

constexpr int kBlock = 32;

struct Mx4View {
  int64_t rows, K;
  int64_t pitch;      // bytes per row of codes
  int64_t kt, rt;     // scale tiles along K (128 values each) and along the rows (128 each)
};

int check_mx4_meta(const gl_mx4* a, Mx4View* v) {
  if (!a) return GL_ERR_NULL;
  if (a->ndim < 0 || a->ndim > GL_MAX_DIMS) return GL_ERR_NDIM;
  if (a->access_ndim < 0 || a->access_ndim > a->ndim) return GL_ERR_NDIM;
  for (int i = 0; i < a->ndim; ++i)
    if (a->shape[i] < 1) return GL_ERR_SHAPE;
  v->rows = prod(a->shape, 0, a->access_ndim);
  v->K = prod(a->shape, a->access_ndim, a->ndim);
  v->pitch = (v->K + kBlock - 1) / kBlock * (kBlock / 2);
  v->kt = (v->K + 127) / 128;
  v->rt = (v->rows + 127) / 128;
  return GL_OK;
}

int check_mx4_data(const gl_mx4* a, Mx4View* v) {
  const int rc = check_mx4_meta(a, v);
  if (rc) return rc;
  if (!a->data || !a->scale) return GL_ERR_NULL;
  if ((reinterpret_cast<uintptr_t>(a->data) | reinterpret_cast<uintptr_t>(a->scale)) & 15u) return GL_ERR_ALIGN;
  // item indices are 32-bit in the kernels
  if (v->rows > INT32_MAX - 256 || v->K > (int64_t{1} << 30)) return GL_ERR_UNSUPPORTED;
  return GL_OK;
}

bool same_shape(const gl_ap* a, const gl_mx4* b) {
  if (a->ndim != b->ndim || a->access_ndim != b->access_ndim) return false;
  for (int i = 0; i < a->ndim; ++i)
    if (a->shape[i] != b->shape[i]) return false;
  return true;
}

// ------------------------------------------------------------------------
// Quantisation and its inverse
// ------------------------------------------------------------------------

// 32 bytes of input per thread when quantising (8 fp32 or 16 bf16 values: four or two neighbouring threads per block, sixteen
// or eight per 4-byte group of scales, the unit in which the scale tiles are addressed: one row, 128 values), eight values
// when going back.  U items per thread, 256 apart, are requested before the first is used.
//
// Bound by HBM: 16384 x 8192 bf16 in 53 us each way, 6.36 TB/s, what a copy reaches.  Getting there took instructions out:
// with an index division per item, unpacked comparisons and eight values a thread it was 127 of them a thread and eight
// values, 114 us and 74 us.  So rows and columns advance by additions, bf16 magnitudes are compared two to a register and
// codes become bf16 by moving bits.
struct QuantParams {
  int64_t K, pitch, kt;
  uint32_t items;        // rows * per_row
  uint32_t per_row;      // kt * 128 / values per item
  uint32_t step_rows, step_cols;   // 256 items further on
  FastDiv div_row;       // by per_row
};

struct ItemAt {
  uint32_t row, col;
  __device__ __forceinline__ void advance(const QuantParams& p) {
    row += p.step_rows;
    col += p.step_cols;
    if (col >= p.per_row) { col -= p.per_row; ++row; }
  }
};

// Byte of the scale tiles that holds block group `quad` (4 blocks) of row r.
__device__ __forceinline__ int64_t scale_quad_at(uint32_t r, uint32_t quad, int64_t kt) {
  return (static_cast<int64_t>(r >> 7) * kt + quad) * 512 + ((r & 31u) * 16 + ((r >> 5) & 3u) * 4);
}

// A thread's values, as they came: eight words of bf16 pairs or of floats.
struct Raw { uint32_t w[8]; };

template <bool F32, bool VEC>
__device__ __forceinline__ void load_raw(const void* __restrict__ in, ItemAt at, int64_t K, Raw& v) {
  constexpr int kVals = F32 ? 8 : 16;
#pragma unroll
  for (int i = 0; i < 8; ++i) v.w[i] = 0;
  const int left = static_cast<int>(K) - static_cast<int>(at.col) * kVals;
  const int64_t first = static_cast<int64_t>(at.row) * K + at.col * static_cast<uint32_t>(kVals);
  if (VEC) {
    // K is a multiple of 8: 16 bytes lie wholly inside the row or wholly behind it
    const uint4* src = reinterpret_cast<const uint4*>(static_cast<const char*>(in) + first * (F32 ? 4 : 2));
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (left > i * (kVals / 2)) {
        const uint4 x = __ldcs(src + i);
        v.w[4 * i] = x.x; v.w[4 * i + 1] = x.y; v.w[4 * i + 2] = x.z; v.w[4 * i + 3] = x.w;
      }
  } else {
#pragma unroll
    for (int i = 0; i < kVals; ++i)
      if (i < left) {
        if (F32) v.w[i & 7] = static_cast<const uint32_t*>(in)[first + i];
        else v.w[i / 2 & 7] |= static_cast<uint32_t>(static_cast<const uint16_t*>(in)[first + i]) << (16 * (i & 1));
      }
  }
}

// Largest magnitude of the values, as fp32 bits (NaN > Inf > finite).
template <bool F32>
__device__ __forceinline__ uint32_t largest(const Raw& v) {
  uint32_t top = 0;
  if constexpr (F32) {
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, v.w[i] & 0x7FFFFFFFu);
    return top;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) top = __vmaxu2(top, v.w[i] & 0x7FFF7FFFu);   // both halves: bf16 magnitudes order like integers
    return max(top << 16, top & 0xFFFF0000u);
  }
}

template <bool F32, bool VEC, int U>
__global__ void __launch_bounds__(256) quantize_mx4(const void* __restrict__ in, uint8_t* __restrict__ codes,
                                                    uint8_t* __restrict__ scale, const QuantParams p) {
  constexpr int kBlockThreads = F32 ? 4 : 2, kQuadThreads = 4 * kBlockThreads, kCodeBytes = F32 ? 4 : 8;
  pdl_wait();
  pdl_launch_dependents();
  const uint32_t first = blockIdx.x * (256u * U) + threadIdx.x;
  Raw v[U];
  ItemAt at0;
  p.div_row.divmod(first, at0.row, at0.col);
  ItemAt at = at0;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (first + u * 256u < p.items) load_raw<F32, VEC>(in, at, p.K, v[u]);
    at.advance(p);
  }
  at = at0;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    // groups of kQuadThreads share a row and `items` is a multiple of that: the shuffles stay inside a group
    if (first + u * 256u >= p.items) break;
    const unsigned group = ((1u << kQuadThreads) - 1u) << (threadIdx.x & 31u & ~(kQuadThreads - 1u));
    uint32_t top = largest<F32>(v[u]);
    top = max(top, __shfl_xor_sync(group, top, 1));
    if (F32) top = max(top, __shfl_xor_sync(group, top, 2));
    const uint32_t e = mx4_exponent(top);
    uint32_t quad = __shfl_down_sync(group, e, kBlockThreads, kQuadThreads) << 8 | e;
    quad |= __shfl_down_sync(group, quad, 2 * kBlockThreads, kQuadThreads) << 16;
    uint8_t* to = codes + static_cast<int64_t>(at.row) * p.pitch + at.col * static_cast<uint32_t>(kCodeBytes);
    const bool inside = at.col * static_cast<uint32_t>(kCodeBytes) < static_cast<uint32_t>(p.pitch);
    float x[8];
    if (F32) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(v[u].w[i]);
      if (inside) *reinterpret_cast<uint32_t*>(to) = mx4_codes8(x, e);
    } else {
      uint32_t word[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[2 * i] = __uint_as_float(v[u].w[4 * k + i] << 16);
          x[2 * i + 1] = __uint_as_float(v[u].w[4 * k + i] & 0xFFFF0000u);
        }
        word[k] = mx4_codes8(x, e);
      }
      if (inside) *reinterpret_cast<uint2*>(to) = make_uint2(word[0], word[1]);   // (the pitch is a multiple of 16)
    }
    if ((threadIdx.x & (kQuadThreads - 1u)) == 0)
      *reinterpret_cast<uint32_t*>(scale + scale_quad_at(at.row, at.col / kQuadThreads, p.kt)) = quad;
    at.advance(p);
  }
}

template <bool F32, bool VEC, int U>
__global__ void __launch_bounds__(256) dequantize_mx4(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scale,
                                                      void* __restrict__ out, const QuantParams p) {
  __shared__ __align__(16) uint16_t staged[VEC ? 8 : 256 * 8];
  pdl_wait();
  pdl_launch_dependents();
  const uint32_t first = blockIdx.x * (256u * U) + threadIdx.x;
  uint32_t word[U], e[U];
  ItemAt at0;
  p.div_row.divmod(first, at0.row, at0.col);
  ItemAt at = at0;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    word[u] = e[u] = 0;
    if (first + u * 256u < p.items && static_cast<int>(at.col) * 8 < static_cast<int>(p.K)) {
      word[u] = *reinterpret_cast<const uint32_t*>(codes + static_cast<int64_t>(at.row) * p.pitch + at.col * 4u);
      e[u] = scale[scale_quad_at(at.row, at.col >> 4, p.kt) + ((at.col >> 2) & 3u)];
    }
    at.advance(p);
  }
  at = at0;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int left = static_cast<int>(p.K) - static_cast<int>(at.col) * 8;
    // bf16 holds every value exactly; fp32 is the same bits with zeros behind
    uint32_t w[4];
    mx4_words_bf16(word[u], e[u], w);
    if (F32 && VEC) {
      // Two neighbours' 64 bytes in two stores that each write whole 32-byte sectors: first both halves of the even
      // lane's values, then of the odd lane's (4096 x 4096: 24 us when each lane stored its own halves).
      const bool odd = threadIdx.x & 1u;
      const uint32_t a = __shfl_xor_sync(0xFFFFFFFFu, odd ? w[0] : w[2], 1), b = __shfl_xor_sync(0xFFFFFFFFu, odd ? w[1] : w[3], 1);
      const uint32_t near[2] = {odd ? a : w[0], odd ? b : w[1]}, far[2] = {odd ? w[2] : a, odd ? w[3] : b};
      const uint32_t col = at.col & ~1u;
      if (first + u * 256u < p.items) {
        uint4* o = reinterpret_cast<uint4*>(static_cast<float*>(out) + static_cast<int64_t>(at.row) * p.K + col * 8u) + odd;
        const int room = static_cast<int>(p.K) - static_cast<int>(col) * 8;
        if (room > 0) __stcs(o, make_uint4(near[0] << 16, near[0] & 0xFFFF0000u, near[1] << 16, near[1] & 0xFFFF0000u));
        if (room > 8) __stcs(o + 2, make_uint4(far[0] << 16, far[0] & 0xFFFF0000u, far[1] << 16, far[1] & 0xFFFF0000u));
      }
    } else if (VEC) {
      if (first + u * 256u < p.items && left > 0)
        __stcs(reinterpret_cast<uint4*>(static_cast<uint16_t*>(out) + static_cast<int64_t>(at.row) * p.K + at.col * 8u),
               make_uint4(w[0], w[1], w[2], w[3]));
    } else {
      // rows without alignment: sixteen lanes hold 128 neighbouring values of a row and store them sixteen at a time
      const uint32_t lane16 = threadIdx.x & 15u;
      __syncwarp();
      *reinterpret_cast<uint4*>(&staged[threadIdx.x * 8u]) = make_uint4(w[0], w[1], w[2], w[3]);
      __syncwarp();
      if (first + u * 256u < p.items) {
        const int col = static_cast<int>(at.col & ~15u) * 8;
        const int64_t to = static_cast<int64_t>(at.row) * p.K + col;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int c = j * 16 + static_cast<int>(lane16);
          const uint16_t half = staged[(threadIdx.x & ~15u) * 8u + c];
          if (col + c < static_cast<int>(p.K)) {
            if (F32) static_cast<uint32_t*>(out)[to + c] = static_cast<uint32_t>(half) << 16;
            else static_cast<uint16_t*>(out)[to + c] = half;
          }
        }
      }
    }
    at.advance(p);
  }
}

// Parameters for items of `vals` values.
int quant_params(const Mx4View& v, int vals, QuantParams* p) {
  const int64_t items = v.rows * v.kt * (128 / vals);
  if (v.rows * v.kt * 16 > INT32_MAX - 4096) return GL_ERR_UNSUPPORTED;   // (one limit whatever the type)
  p->K = v.K;
  p->pitch = v.pitch;
  p->kt = v.kt;
  p->items = static_cast<uint32_t>(items);
  p->per_row = static_cast<uint32_t>(v.kt * (128 / vals));
  p->step_rows = 256u / p->per_row;
  p->step_cols = 256u % p->per_row;
  p->div_row.set(p->per_row);
  return GL_OK;
}

// Several items per thread only when every SM has blocks to hold.
constexpr int kItemsPerThread = 4;
bool many_items(const QuantParams& p) { return p.items >= static_cast<uint32_t>(num_sms()) * 4u * 256u * kItemsPerThread; }
dim3 item_grid(const QuantParams& p) {
  const uint32_t per_block = 256u * (many_items(p) ? kItemsPerThread : 1);
  return dim3((p.items + per_block - 1) / per_block);
}

int launch_quantize(const gl_ap& in, const Mx4View& v, void* codes, void* scale, cudaStream_t st) {
  const bool f32 = in.dtype == GL_F32, vec = v.K % 8 == 0;
  QuantParams p;
  const int rc = quant_params(v, f32 ? 8 : 16, &p);
  if (rc) return rc;
  constexpr int kU = kItemsPerThread;
  void (*k)(const void*, uint8_t*, uint8_t*, QuantParams) =
      many_items(p) ? (f32 ? (vec ? quantize_mx4<true, true, kU> : quantize_mx4<true, false, kU>)
                           : (vec ? quantize_mx4<false, true, kU> : quantize_mx4<false, false, kU>))
                    : (f32 ? (vec ? quantize_mx4<true, true, 1> : quantize_mx4<true, false, 1>)
                           : (vec ? quantize_mx4<false, true, 1> : quantize_mx4<false, false, 1>));
  return launch_pdl(k, item_grid(p), dim3(256), 0, st, 1, static_cast<const void*>(in.data), static_cast<uint8_t*>(codes),
                    static_cast<uint8_t*>(scale), p) == cudaSuccess ? GL_OK : GL_ERR_CUDA;
}

// ------------------------------------------------------------------------
// Block-scaled product
// ------------------------------------------------------------------------

// out[m,o] = sum over blocks b of 2^(ea[m,b] + eb[o,b] - 254) sum_k a[m,k] b[o,k]: the inner products of E2M1 codes, their
// scaling and the fp32 sum are one instruction, tcgen05.mma kind::mxf4, four times the bf16 rate per flop and byte.
//
// What bounds it at size is what bounds the bf16 product: operands from L2 to the SMs.  A 256 x 256 tile on a pair of SMs
// needs 64 bytes per cycle and SM, a 128 x 128 tile on one SM twice that.  16384 x 8192 x 8192 with bf16 results: 532 us
// on single SMs, 360 us on pairs, 6.1 PFLOP/s; 4096^3 28 us (fp32 results 34 us: 67 MB to write).  A 256-wide
// accumulator takes half the tensor memory, so two of them and the scales overlap in 24 columns, which the epilogue empties
// first; the next tile's products wait for that only.

// D[tmem] (+)= (A * sfa)[smem] * (B * sfb)[smem]^T, K = 64, scales of 32 values each (two per row and instruction).
template <int CTAS>
__device__ __forceinline__ void tc_mma_mx4(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t sfa,
                                           uint32_t sfb, uint32_t accumulate) {
  if (CTAS == 2)
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory");
}

// One scale tile (32 rows x 16 bytes of shared memory) into four columns of tensor memory, repeated in the four lane
// quarters.  Copies and MMAs of one thread run in the order of their issue.
template <int CTAS>
__device__ __forceinline__ void tc_copy_scales(uint32_t taddr, uint64_t desc) {
  if (CTAS == 2) asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
  else asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}

// Instruction descriptor, kind::mxf4: A and B E2M1 (bits 7-9 and 10-11 = 1), both K-major, N >> 3 at bit 17, scales
// E8M0 (bit 23), M >> 7 at bit 27; which half of the four scale bytes the instruction reads: bits 4-5 (B), 29-30 (A).
__host__ __device__ constexpr uint32_t make_idesc_mx4(int m, int n, int half) {
  return (static_cast<uint32_t>(half * 2) << 4) | (1u << 7) | (1u << 10) | (static_cast<uint32_t>(n >> 3) << 17) | (1u << 23) |
         (static_cast<uint32_t>(m >> 7) << 27) | (static_cast<uint32_t>(half * 2) << 29);
}

// relu that lets a NaN through (fmaxf would turn it into 0)
__device__ __forceinline__ float relu_keep_nan(float v) { return v < 0.f ? 0.f : v; }

constexpr int kTile = 128;           // rows of A per block
constexpr int kKBytes = 128;         // bytes of a row per K block: 256 values, one 128-byte swizzle row
constexpr int kMxThreads = 224;      // warp 0 TMA (A), warp 1 MMA, warps 2-5 epilogue, warp 6 TMA (B)

struct Mx4Params {
  int64_t M, O;
  int tiles_m, tiles_n;   // tiles_m counts 128 * CTAS rows
  int kblocks;            // K blocks of 256 values
  int last_steps;         // instructions (64 values) in the last K block
  int relu, out_bf16, tma_store;
  FastDiv div_tiles_n;
};

template <int BN, int CTAS>
struct MxCfg {
  static constexpr int kStageA = kTile * kKBytes;
  static constexpr int kStageB = (BN / CTAS) * kKBytes;
  static constexpr int kScaleA = 1024, kScaleB = (BN / 128) * 1024;   // two scale tiles along K per row tile
  static constexpr int kStage = kStageA + kStageB + kScaleA + kScaleB;
  static constexpr int kEpiBytes = 4 * 2 * 4096;
  static constexpr int kStages = (232448 - kEpiBytes - 1024 - 256) / kStage;
  static constexpr int kSmemBytes = kStages * kStage + kEpiBytes + 1024 + 256;
  // Tensor memory (512 columns): scales in the last kSfCols, two accumulators of BN columns before them.  256-wide
  // accumulators do not fit twice: they share kSfCols columns, which the epilogue empties first.
  static constexpr int kSfCols = 8 + BN / 16;
  static constexpr int kSfBase = 512 - kSfCols;
  static constexpr int kAcc1 = 2 * BN <= kSfBase ? BN : kSfBase - BN;
  static constexpr bool kOverlap = kAcc1 < BN;
};

template <int BN, int CTAS>
__global__ void __launch_bounds__(kMxThreads, 1)
dot_mx4(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
        const __grid_constant__ CUtensorMap map_sa, const __grid_constant__ CUtensorMap map_sb,
        const __grid_constant__ CUtensorMap map_c, void* __restrict__ out, const Mx4Params p) {
  using Cfg = MxCfg<BN, CTAS>;
  static_assert(Cfg::kStages >= 2, "ring too shallow");
  extern __shared__ unsigned char smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t tiles = (raw + 1023u) & ~1023u;   // the 128-byte swizzle wants 1024-byte aligned tiles
  unsigned char* gen_tiles = smem_raw + (tiles - raw);
  const uint32_t epi_base = tiles + Cfg::kStages * Cfg::kStage;
  uint64_t* bars = reinterpret_cast<uint64_t*>(gen_tiles + Cfg::kStages * Cfg::kStage + Cfg::kEpiBytes);
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
    for (int a = 0; a < 2; ++a) { mbar_init(bar_tfull + 8 * a, 1); mbar_init(bar_tempty + 8 * a, 4 * CTAS); }
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

  if (warp == 0 || warp == 6) {
    // ---------------- TMA producers: warp 0 stages A and its scales, warp 6 stages B and its scales ----------------
    const bool load_a = warp == 0;
    const bool leader = elect_one();
    uint32_t s = 0, ph = 0;
    bool ok = true;
    for (int u = unit0; u < num_tiles && ok; u += unit_step) {
      uint32_t tm, tn;
      p.div_tiles_n.divmod(static_cast<uint32_t>(u), tm, tn);
      const int m0 = (static_cast<int>(tm) * CTAS + static_cast<int>(rank)) * kTile;
      const int n0 = static_cast<int>(tn) * BN + static_cast<int>(rank) * (BN / CTAS);
      for (int kb = 0; kb < p.kblocks; ++kb) {
        if (!mbar_wait(bar_empty + 8 * s, ph ^ 1u, abort_flag)) { ok = false; break; }
        const uint32_t full = CTAS == 2 ? map_to_cta(bar_full + 8 * s, 0) : bar_full + 8 * s;
        const uint32_t stage = tiles + s * Cfg::kStage;
        const uint32_t sc = stage + Cfg::kStageA + Cfg::kStageB;
        if (rank == 0 && leader)
          mbar_expect_tx(bar_full + 8 * s, CTAS * (load_a ? Cfg::kStageA + Cfg::kScaleA : Cfg::kStageB + Cfg::kScaleB));
        if (leader) {
          if (load_a) {
            if (CTAS == 2) {
              tma_load_2d_pair(stage, &map_a, kb * kKBytes, m0, full);
              tma_load_3d_pair(sc, &map_sa, 0, kb * 2, m0 / 128, full);
            } else {
              tma_load_2d(stage, &map_a, kb * kKBytes, m0, full);
              tma_load_3d(sc, &map_sa, 0, kb * 2, m0 / 128, full);
            }
          } else {
            // every block of a pair holds the scales of all BN columns
            if (CTAS == 2) tma_load_2d_pair(stage + Cfg::kStageA, &map_b, kb * kKBytes, n0, full);
            else tma_load_2d(stage + Cfg::kStageA, &map_b, kb * kKBytes, n0, full);
#pragma unroll
            for (int h = 0; h < BN / 128; ++h) {
              const uint32_t dst = sc + Cfg::kScaleA + h * 1024;
              const int rt = static_cast<int>(tn) * (BN / 128) + h;
              if (CTAS == 2) tma_load_3d_pair(dst, &map_sb, 0, kb * 2, rt, full);
              else tma_load_3d(dst, &map_sb, 0, kb * 2, rt, full);
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
      const uint64_t desc_s0 = make_desc(tiles + Cfg::kStageA + Cfg::kStageB, 16, 128, 0);
      const uint32_t sfa = tmem_base + Cfg::kSfBase, sfb = sfa + 8;
      uint32_t s = 0, ph = 0, tile_it = 0;
      bool ok = true;
      for (int u = unit0; u < num_tiles && ok; u += unit_step, ++tile_it) {
        const uint32_t acc = tile_it & 1u;
        // separate accumulators: the one two tiles back has been read; overlapping ones: the shared columns of the
        // previous tile have been read (its epilogue had then finished with the tile before)
        const uint32_t wait_on = Cfg::kOverlap ? acc ^ 1u : acc;
        const uint32_t round = Cfg::kOverlap ? (tile_it + 1) >> 1 : tile_it >> 1;
        if (!mbar_wait(bar_tempty + 8 * wait_on, (round & 1u) ^ 1u, abort_flag)) { ok = false; break; }
        tc_fence_after();
        const uint32_t d_tmem = tmem_base + (acc ? Cfg::kAcc1 : 0);
        for (int kb = 0; kb < p.kblocks; ++kb) {
          if (!mbar_wait(bar_full + 8 * s, ph, abort_flag)) { ok = false; break; }
          tc_fence_after();
          const uint64_t da0 = desc_a0 + ((s * Cfg::kStage) >> 4);
          const uint64_t db0 = desc_b0 + ((s * Cfg::kStage) >> 4);
          const uint64_t ds0 = desc_s0 + ((s * Cfg::kStage) >> 4);
          const int steps = kb + 1 == p.kblocks ? p.last_steps : 4;
#pragma unroll
          for (int g = 0; g < 2; ++g) {   // 128 values: one scale tile per 128 rows
            if (2 * g < steps) {
              if (leader) {
                tc_copy_scales<CTAS>(sfa + 4 * g, ds0 + ((g * 512) >> 4));
#pragma unroll
                for (int h = 0; h < BN / 128; ++h)
                  tc_copy_scales<CTAS>(sfb + g * (BN / 32) + 4 * h, ds0 + ((Cfg::kScaleA + h * 1024 + g * 512) >> 4));
              }
#pragma unroll
              for (int j = 0; j < 2; ++j) {
                const int k = 2 * g + j;
                if (k < steps && leader)
                  tc_mma_mx4<CTAS>(d_tmem, da0 + 2 * k, db0 + 2 * k, make_idesc_mx4(kTile * CTAS, BN, j), sfa + 4 * g,
                                   sfb + g * (BN / 32), (kb | k) != 0 ? 1u : 0u);
              }
            }
          }
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
      }
    }
  } else {
    // ---------------- epilogue: TMEM -> registers -> (shared memory -> TMA store | global) ----------------
    const int q = warp & 3;
    const bool leader = elect_one();
    uint32_t tile_it = 0, chunk_it = 0;
    bool ok = true;
    const uint32_t stage_buf = epi_base + q * 8192;
    const int cstep = p.out_bf16 ? 64 : 32;
    const int nchunks = BN / cstep;
    for (int u = unit0; u < num_tiles && ok; u += unit_step, ++tile_it) {
      const uint32_t acc = tile_it & 1u, aph = (tile_it >> 1) & 1u;
      uint32_t tmu, tn;
      p.div_tiles_n.divmod(static_cast<uint32_t>(u), tmu, tn);
      const int tm = static_cast<int>(tmu) * CTAS + static_cast<int>(rank);
      if (!mbar_wait(bar_tfull + 8 * acc, aph, abort_flag)) { ok = false; break; }
      tc_fence_after();
      const uint32_t taddr = tmem_base + (acc ? Cfg::kAcc1 : 0) + (static_cast<uint32_t>(q * 32) << 16);
#pragma unroll 1
      for (int i = 0; i < nchunks; ++i) {
        // the columns that two overlapping accumulators share go first: the last ones of the first, the first ones
        // of the second
        const int c = (Cfg::kOverlap && acc == 0 ? nchunks - 1 - i : i) * cstep;
        const int64_t n0 = static_cast<int64_t>(tn) * BN + c;
        uint32_t r[32];
        tc_load_32cols(taddr + c, r);
        if (p.relu) {
#pragma unroll
          for (int j = 0; j < 32; ++j) r[j] = __float_as_uint(relu_keep_nan(__uint_as_float(r[j])));
        }
        if (p.out_bf16) {
#pragma unroll
          for (int j = 0; j < 16; ++j) r[j] = pack_bf16x2(r[2 * j], r[2 * j + 1]);
          uint32_t r2[32];
          tc_load_32cols(taddr + c + 32, r2);
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            float a = __uint_as_float(r2[2 * j]), b = __uint_as_float(r2[2 * j + 1]);
            if (p.relu) { a = relu_keep_nan(a); b = relu_keep_nan(b); }
            r[16 + j] = pack_bf16x2(__float_as_uint(a), __float_as_uint(b));
          }
        }
        if (i == (Cfg::kOverlap ? 0 : nchunks - 1)) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) {
            if (CTAS == 2) mbar_arrive_remote(map_to_cta(bar_tempty + 8 * acc, 0));
            else mbar_arrive(bar_tempty + 8 * acc);
          }
        }
        if (n0 >= p.O) continue;   // uniform across the warp
        const uint32_t buf = stage_buf + (chunk_it & 1u) * 4096;
        ++chunk_it;
        if (p.tma_store && leader) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
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
            if (tm * kTile + q * 32 < p.M)
              asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];" ::"l"(
                               reinterpret_cast<uint64_t>(&map_c)),
                           "r"(static_cast<int>(n0)), "r"(tm * kTile + q * 32), "r"(buf)
                           : "memory");
            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
          }
        } else {
          // rows that are no multiples of 16 bytes: row by row, neighbouring lanes on neighbouring columns (a lane
          // per row instead takes 32 memory segments per store: 25 us against 12 us for 301 x 1111 x 777)
          __syncwarp();
          const int rows = static_cast<int>(min(static_cast<int64_t>(32), p.M - (static_cast<int64_t>(tm) * kTile + q * 32)));
          const int cols = static_cast<int>(min(static_cast<int64_t>(cstep), p.O - n0));
          const int64_t base = (static_cast<int64_t>(tm) * kTile + q * 32) * p.O + n0;
#pragma unroll 8
          for (int i = 0; i < rows; ++i) {
            uint32_t v;
            asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(buf + i * 128 + (((lane >> 2) ^ (i & 7)) << 4) + (lane & 3) * 4));
            if (p.out_bf16) {
              uint16_t* to = static_cast<uint16_t*>(out) + base + i * p.O + 2 * lane;
              if ((p.O & 1) == 0) {
                if (2 * lane < cols) *reinterpret_cast<uint32_t*>(to) = v;   // (O even: whole pairs)
              } else {
                if (2 * lane < cols) to[0] = static_cast<uint16_t>(v);
                if (2 * lane + 1 < cols) to[1] = static_cast<uint16_t>(v >> 16);
              }
            } else if (lane < cols) {
              static_cast<float*>(out)[base + i * p.O + lane] = __uint_as_float(v);
            }
          }
        }
      }
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
// With at most 128 rows of A the product is bound by reading B (the weights) once.  Tiles of 128 rows of B, all rows of
// A as the N side (BN = 16 to 128 of them), and K cut over the S blocks of a cluster so that the loads of all SMs are in
// flight: the blocks' partial sums meet in distributed shared memory, added in rank order.  One tile per block, two
// blocks per SM.  While the kernel that rounds A is still running the weights are on their way into L2.
// 8192 x 8192 weights (36 MB) in L2, in a graph: 6.9 us for one row, 8.8 us for 16, 10.3 us for 64; weights that are not in L2,
// one row: 9.2 us, 3.9 TB/s of HBM.  A launch that does nothing is 2 us of it and filling the machine 2 more.

// At most kFuseRows rows (FUSED): the blocks round A themselves, each its own stretch of K, straight into operand order, while
// the first weights are on their way: one launch.  Fused against a launch of its own for the rounding, us:
//   K x O            1 row          4 rows         8 rows         16 rows
//   1024 x 1024      2.9 / 4.1      3.0 / 4.3      3.4 / 4.3      4.4 / 4.5
//   3136 x 1000      3.9 / 4.6      3.9 / 4.7      4.7 / 4.8      6.0 / 5.0
//   4096 x 4096      5.1 / 6.5      5.6 / 6.5      6.7 / 6.8      8.1 / 7.0
//   2048 x 8192      4.6 / 5.7      5.2 / 5.7      6.0 / 5.8      7.5 / 6.0
//   8192 x 8192      6.9 / 8.9      9.1 / 8.7      11.6 / 8.6     16.9 / 8.8
// What every block repeats is rows x K blocks of a rank; up to four rows it is no more than the launch, but for the last line's
// four rows, which lose 5 %.
constexpr int kFuseRows = 4;
constexpr int kFuseBlocks = 12;   // K blocks of A that a block has room for

struct FewParams {
  int M;
  int64_t O;
  const void* x;          // FUSED: rows of A as they came
  int64_t K;
  int x_f32;
  int kblocks, last_steps;
  int split;              // blocks per cluster
  int relu, out_bf16;
};

// Rank r adds up the columns r, r + S, ...: the S partial sums of a value in rank order, those of four columns requested
// before the first is added.
template <int S>
__device__ __forceinline__ void join_ranks(uint32_t mine, int rank, int64_t o, void* __restrict__ out, const FewParams& p) {
  for (int c0 = rank; c0 < p.M; c0 += 4 * S) {
    float x[4][S];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int from = 0; from < S; ++from)   // (columns past M are inside the partial sums' space only up to BN)
        if (c0 + j * S < p.M)
          asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x[j][from]) : "r"(map_to_cta(mine + (c0 + j * S) * 512, from)));
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int c = c0 + j * S;
      if (c >= p.M) break;
      float v = x[j][0];
#pragma unroll
      for (int from = 1; from < S; ++from) v += x[j][from];
      if (p.relu) v = relu_keep_nan(v);
      if (p.out_bf16) static_cast<uint16_t*>(out)[c * p.O + o] = f32_to_bf16(v);
      else static_cast<float*>(out)[c * p.O + o] = v;
    }
  }
}

template <int BN, bool FUSED>
struct FewCfg {
  static constexpr int kStageA = kTile * kKBytes;                  // weights
  static constexpr int kStageB = FUSED ? 0 : BN * kKBytes;
  static constexpr int kStage = kStageA + kStageB + (FUSED ? 1024 : 2048);   // and two scale tiles of each side
  static constexpr int kXBlock = BN * kKBytes + 1024;              // FUSED: a K block of A with its scale tiles
  static constexpr int kXBytes = FUSED ? kFuseBlocks * kXBlock : 0;
  static constexpr int kStages = (112 * 1024 - 1024 - 256 - kXBytes) / kStage;
  static constexpr int kSmemBytes = kStages * kStage + kXBytes + 1024 + 256;
  static constexpr int kTmemCols = BN + 16 <= 32 ? 32 : BN + 16 <= 64 ? 64 : BN + 16 <= 128 ? 128 : 256;
  static constexpr int kSfBase = kTmemCols - 16;
  static_assert(kStages >= 2 && kStages * kStage >= BN * 128 * 4, "partial sums fit in the ring");
};

// One warp rounds K block kb of row m: lane = 8 values, into the swizzled operand row and the scale tiles.
template <int BN>
__device__ __forceinline__ void round_row_block(const FewParams& p, unsigned char* to, int m, int kb, int lane) {
  const int64_t k0 = static_cast<int64_t>(kb) * 256 + lane * 8, left = p.K - k0, at = static_cast<int64_t>(m) * p.K + k0;
  float x[8];
  if (left >= 8 && (p.K & 7) == 0) {
    if (p.x_f32) {
      const float4 a = *reinterpret_cast<const float4*>(static_cast<const float*>(p.x) + at);
      const float4 b = *(reinterpret_cast<const float4*>(static_cast<const float*>(p.x) + at) + 1);
      x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    } else {
      const uint4 a = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.x) + at);
      const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      x[i] = i < left ? (p.x_f32 ? static_cast<const float*>(p.x)[at + i] : bf16_to_f32(static_cast<const uint16_t*>(p.x)[at + i])) : 0.f;
  }
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7FFFFFFFu);
  top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
  top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
  const uint32_t e = mx4_exponent(top);
  *reinterpret_cast<uint32_t*>(to + m * 128 + (((lane >> 2) ^ (m & 7)) << 4) + (lane & 3) * 4) = mx4_codes8(x, e);
  if ((lane & 3) == 0) to[BN * kKBytes + (lane >> 4) * 512 + m * 16 + ((lane >> 2) & 3)] = static_cast<uint8_t>(e);
}

template <int BN, bool FUSED>
__global__ void __launch_bounds__(kMxThreads, 2)
dot_mx4_few(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x,
            const __grid_constant__ CUtensorMap map_sw, const __grid_constant__ CUtensorMap map_sx, void* __restrict__ out,
            const FewParams p) {
  using Cfg = FewCfg<BN, FUSED>;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t tiles = (raw + 1023u) & ~1023u;
  unsigned char* gen_tiles = smem_raw + (tiles - raw);
  const uint32_t xs = tiles + Cfg::kStages * Cfg::kStage;            // FUSED: A, block by block
  uint64_t* bars = reinterpret_cast<uint64_t*>(gen_tiles + Cfg::kStages * Cfg::kStage + Cfg::kXBytes);
  const uint32_t bar_full = smem_u32(bars), bar_empty = bar_full + 8 * Cfg::kStages, bar_done = bar_empty + 8 * Cfg::kStages,
                 bar_x = bar_done + 8;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * Cfg::kStages + 2);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = p.split > 1 ? static_cast<int>(cluster_ctarank()) : 0;
  const int tile = static_cast<int>(blockIdx.x) / p.split;
  // K blocks of this rank, as even as they go
  const int kb0 = static_cast<int>(static_cast<int64_t>(p.kblocks) * rank / p.split);
  const int kb1 = static_cast<int>(static_cast<int64_t>(p.kblocks) * (rank + 1) / p.split);

  if (warp == 0 && elect_one())
    for (int kb = kb0; kb < kb1; ++kb) tma_prefetch_2d(&map_w, kb * kKBytes, tile * kTile);
  if (threadIdx.x == 0) {
    for (int s = 0; s < Cfg::kStages; ++s) { mbar_init(bar_full + 8 * s, FUSED ? 1 : 2); mbar_init(bar_empty + 8 * s, 1); }
    mbar_init(bar_done, 1);
    mbar_init(bar_x, 5);   // warps 2 to 6
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
    const int blocks = kb1 - kb0;   // rows one after the other, their K blocks side by side
    for (int i = warp - 2; i < p.M * blocks; i += 5)
      round_row_block<BN>(p, gen_tiles + Cfg::kStages * Cfg::kStage + (i % blocks) * Cfg::kXBlock, i / blocks, kb0 + i % blocks, lane);
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
      const uint32_t full = bar_full + 8 * s, stage = tiles + s * Cfg::kStage, sc = stage + Cfg::kStageA + Cfg::kStageB;
      if (leader) {
        mbar_expect_tx(full, (load_w ? Cfg::kStageA : Cfg::kStageB) + 1024);
        if (load_w) {
          tma_load_2d(stage, &map_w, kb * kKBytes, tile * kTile, full);
          tma_load_3d(sc, &map_sw, 0, kb * 2, tile, full);
        } else {
          tma_load_2d(stage + Cfg::kStageA, &map_x, kb * kKBytes, 0, full);
          tma_load_3d(sc + 1024, &map_sx, 0, kb * 2, 0, full);
        }
      }
      if (++s == Cfg::kStages) { s = 0; ph ^= 1u; }
    }
  } else if (warp == 1) {
    const bool leader = elect_one();
    const uint64_t desc_w0 = make_desc(tiles, 16, 1024, 2), desc_x0 = make_desc(FUSED ? xs : tiles + Cfg::kStageA, 16, 1024, 2);
    const uint64_t desc_s0 = make_desc(tiles + Cfg::kStageA + Cfg::kStageB, 16, 128, 0);
    const uint64_t desc_sx0 = make_desc(FUSED ? xs + BN * kKBytes : tiles + Cfg::kStageA + Cfg::kStageB + 1024, 16, 128, 0);
    const uint32_t sfw = tmem_base + Cfg::kSfBase, sfx = sfw + 8;
    uint32_t s = 0, ph = 0;
    bool ok = !FUSED || mbar_wait(bar_x, 0, abort_flag);
    for (int kb = kb0; kb < kb1 && ok; ++kb) {
      if (!mbar_wait(bar_full + 8 * s, ph, abort_flag)) { ok = false; break; }
      tc_fence_after();
      const uint64_t off = (s * Cfg::kStage) >> 4, xoff = FUSED ? ((kb - kb0) * Cfg::kXBlock) >> 4 : off;
      const int steps = kb + 1 == p.kblocks ? p.last_steps : 4;
#pragma unroll
      for (int g = 0; g < 2; ++g)
        if (2 * g < steps) {
          if (leader) {
            tc_copy_scales<1>(sfw + 4 * g, desc_s0 + off + ((g * 512) >> 4));
            tc_copy_scales<1>(sfx + 4 * g, desc_sx0 + xoff + ((g * 512) >> 4));
          }
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int k = 2 * g + j;
            if (k < steps && leader)
              tc_mma_mx4<1>(tmem_base, desc_w0 + off + 2 * k, desc_x0 + xoff + 2 * k, make_idesc_mx4(kTile, BN, j), sfw + 4 * g,
                            sfx + 4 * g, kb != kb0 || k != 0 ? 1u : 0u);
          }
        }
      if (leader) tc_commit(bar_empty + 8 * s);
      if (++s == Cfg::kStages) { s = 0; ph ^= 1u; }
    }
    if (ok && leader) tc_commit(bar_done);
  }
  float* part = reinterpret_cast<float*>(gen_tiles);   // [BN][128]: every MMA has read the ring when bar_done flips
  const int q = warp & 3;
  const int64_t o = static_cast<int64_t>(tile) * kTile + q * 32 + lane;
  const bool epilogue = warp >= 2 && warp < 6;
  if (epilogue) {
    const bool ok = mbar_wait(bar_done, 0, abort_flag);
    tc_fence_after();
    if (ok) {
#pragma unroll 1
      for (int c = 0; c < BN; c += 16) {
        if (c >= p.M) break;
        uint32_t r[16];
        tc_load_16cols(tmem_base + (static_cast<uint32_t>(q * 32) << 16) + c, r);
        if (p.split > 1) {
#pragma unroll
          for (int j = 0; j < 16; ++j) part[(c + j) * 128 + q * 32 + lane] = __uint_as_float(r[j]);
        } else if (o < p.O) {
#pragma unroll
          for (int j = 0; j < 16; ++j)
            if (c + j < p.M) {
              const float v = p.relu ? relu_keep_nan(__uint_as_float(r[j])) : __uint_as_float(r[j]);
              if (p.out_bf16) static_cast<uint16_t*>(out)[(c + j) * p.O + o] = f32_to_bf16(v);
              else static_cast<float*>(out)[(c + j) * p.O + o] = v;
            }
        }
      }
    }
    tc_fence_before();
  }
  if (p.split > 1) {
    __syncwarp();
    cluster_sync_all();
    if (epilogue && o < p.O) {
      const uint32_t mine = smem_u32(part) + (q * 32 + lane) * 4;
      switch (p.split) {
        case 2: join_ranks<2>(mine, rank, o, out, p); break;
        case 4: join_ranks<4>(mine, rank, o, out, p); break;
        default: join_ranks<8>(mine, rank, o, out, p); break;
      }
    }
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

struct Mx4Operand { const void* codes; const void* scale; Mx4View v; };

bool encode_codes(CUtensorMap* m, const Mx4Operand& a, int box_rows) {
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(a.v.pitch), static_cast<cuuint64_t>(a.v.rows)};
  const cuuint64_t strides[1] = {static_cast<cuuint64_t>(a.v.pitch)};
  const cuuint32_t box[2] = {kKBytes, static_cast<cuuint32_t>(box_rows)};
  return encode(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, a.codes, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B,
                CU_TENSOR_MAP_L2_PROMOTION_L2_256B);
}

// Scale tiles as (128 words, tiles along K, tiles along the rows); a box is the two tiles of one K block.  Tiles past
// the end read as zeros.
bool encode_scales(CUtensorMap* m, const Mx4Operand& a) {
  const cuuint64_t dims[3] = {128, static_cast<cuuint64_t>(a.v.kt), static_cast<cuuint64_t>(a.v.rt)};
  const cuuint64_t strides[2] = {512, static_cast<cuuint64_t>(a.v.kt) * 512};
  const cuuint32_t box[3] = {128, 2, 1};
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

struct TilePlanMx4 {
  CUtensorMap ma, mb, msa, msb, mc;
  Mx4Params p;
  void* out;
  int grid;
};

template <int BN, int CTAS>
int plan_tiles(const Mx4Operand& a, const Mx4Operand& b, void* out, uint32_t flags, TilePlanMx4* t) {
  using Cfg = MxCfg<BN, CTAS>;
  static std::atomic<int> resident[64];   // per device, 0: not asked yet (threads may ask at once: the calls are idempotent)
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return GL_ERR_CUDA;
  int at_once = resident[dev].load(std::memory_order_acquire);
  if (!at_once) {
    if (cudaFuncSetAttribute(dot_mx4<BN, CTAS>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg::kSmemBytes) != cudaSuccess)
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
      cfg.blockDim = dim3(kMxThreads);
      cfg.dynamicSmemBytes = Cfg::kSmemBytes;
      cfg.attrs = &at;
      cfg.numAttrs = 1;
      if (cudaOccupancyMaxActiveClusters(&at_once, dot_mx4<BN, CTAS>, &cfg) != cudaSuccess || at_once < 1) return GL_ERR_CUDA;
      at_once = std::min(at_once, num_sms() / 2);
    }
    resident[dev].store(at_once, std::memory_order_release);
  }
  Mx4Params& p = t->p;
  p.M = a.v.rows;
  p.O = b.v.rows;
  p.tiles_m = static_cast<int>((p.M + kTile * CTAS - 1) / (kTile * CTAS));
  p.tiles_n = static_cast<int>((p.O + BN - 1) / BN);
  if (static_cast<int64_t>(p.tiles_m) * p.tiles_n > (1 << 30)) return GL_ERR_UNSUPPORTED;
  const int64_t steps = (a.v.K + 63) / 64;
  p.kblocks = static_cast<int>((steps + 3) / 4);
  p.last_steps = static_cast<int>(steps - 4 * static_cast<int64_t>(p.kblocks - 1));
  p.relu = (flags & GL_EPILOGUE_RELU) ? 1 : 0;
  p.out_bf16 = (flags & GL_OUT_BF16) ? 1 : 0;
  p.tma_store = p.O % (p.out_bf16 ? 8 : 4) == 0 ? 1 : 0;
  p.div_tiles_n.set(p.tiles_n);
  t->out = out;
  t->grid = CTAS * std::min(at_once, p.tiles_m * p.tiles_n);
  if (!encode_codes(&t->ma, a, kTile) || !encode_codes(&t->mb, b, BN / CTAS) || !encode_scales(&t->msa, a) ||
      !encode_scales(&t->msb, b))
    return GL_ERR_CUDA;
  t->mc = t->ma;   // unused without TMA stores; any valid map
  if (p.tma_store && !encode_out(&t->mc, out, p.M, p.O, p.out_bf16 != 0)) return GL_ERR_CUDA;
  return GL_OK;
}

template <int BN, int CTAS>
int run_tiles(const TilePlanMx4& t, cudaStream_t st) {
  return launch_pdl(dot_mx4<BN, CTAS>, dim3(static_cast<unsigned>(t.grid)), dim3(kMxThreads), MxCfg<BN, CTAS>::kSmemBytes, st, CTAS,
                    t.ma, t.mb, t.msa, t.msb, t.mc, t.out, t.p) == cudaSuccess ? GL_OK : GL_ERR_CUDA;
}

struct FewPlan {
  CUtensorMap mw, mx, msw, msx;
  FewParams p;
  void* out;
  int grid;
};

// `fused`: A is still to be rounded, by the product's own blocks.
template <int BN, bool FUSED>
int plan_few(const Mx4Operand& a, const Mx4Operand& b, void* out, uint32_t flags, FewPlan* t) {
  static std::atomic<bool> attr_set[64];   // per device (threads may set it at once: the call is idempotent)
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return GL_ERR_CUDA;
  if (!attr_set[dev].load(std::memory_order_acquire)) {
    if (cudaFuncSetAttribute(dot_mx4_few<BN, FUSED>, cudaFuncAttributeMaxDynamicSharedMemorySize, FewCfg<BN, FUSED>::kSmemBytes) != cudaSuccess)
      return GL_ERR_CUDA;
    attr_set[dev].store(true, std::memory_order_release);
  }
  FewParams& p = t->p;
  p.M = static_cast<int>(a.v.rows);
  p.O = b.v.rows;
  const int64_t steps = (a.v.K + 63) / 64;
  p.kblocks = static_cast<int>((steps + 3) / 4);
  p.last_steps = static_cast<int>(steps - 4 * static_cast<int64_t>(p.kblocks - 1));
  p.relu = (flags & GL_EPILOGUE_RELU) ? 1 : 0;
  p.out_bf16 = (flags & GL_OUT_BF16) ? 1 : 0;
  if (b.v.rt > (1 << 27)) return GL_ERR_UNSUPPORTED;
  const int tiles = static_cast<int>(b.v.rt);
  // as many ranks as still leave every one a K block and all blocks resident at once (two per SM)
  p.split = 1;
  while (p.split < 8 && p.split * 2 <= p.kblocks && tiles * p.split * 2 <= 2 * num_sms()) p.split *= 2;
  t->out = out;
  t->grid = tiles * p.split;
  if (!encode_codes(&t->mw, b, kTile) || !encode_scales(&t->msw, b)) return GL_ERR_CUDA;
  t->mx = t->mw;   // unused when FUSED; any valid map
  t->msx = t->msw;
  return FUSED || (encode_codes(&t->mx, a, BN) && encode_scales(&t->msx, a)) ? GL_OK : GL_ERR_CUDA;
}

template <int BN, bool FUSED>
int run_few(const FewPlan& t, cudaStream_t st) {
  return launch_pdl(dot_mx4_few<BN, FUSED>, dim3(static_cast<unsigned>(t.grid)), dim3(kMxThreads), FewCfg<BN, FUSED>::kSmemBytes, st, t.p.split,
                    t.mw, t.mx, t.msw, t.msx, t.out, t.p) == cudaSuccess ? GL_OK : GL_ERR_CUDA;
}

template <int BN, typename Pre>
int product_few(const Mx4Operand& a, const Mx4Operand& b, gl_ap* out, uint32_t flags, cudaStream_t st, Pre&& pre) {
  FewPlan t;
  int rc = plan_few<BN, false>(a, b, out->data, flags, &t);
  if (rc) return rc;
  rc = pre();
  if (rc) return rc;
  return run_few<BN, false>(t, st);
}

// Checks shared by the two products: shapes, result, aliasing rules are the caller's.
int check_product(const gl_ap* out, int a_access, const int64_t* a_shape, int a_compute, const gl_mx4* a1, uint32_t flags) {
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
int product(const Mx4Operand& a, const Mx4Operand& b, gl_ap* out, uint32_t flags, cudaStream_t st, Pre&& pre) {
  if (!driver_api().ok) return GL_ERR_CUDA;
  // Up to 128 rows: the weights as the 128-row side, K cut over clusters (64 x 8192 x 8192: 12.8 us against 20.3 us on
  // the tiles below).
  if (a.v.rows <= 16) return product_few<16>(a, b, out, flags, st, pre);
  if (a.v.rows <= 32) return product_few<32>(a, b, out, flags, st, pre);
  if (a.v.rows <= 64) return product_few<64>(a, b, out, flags, st, pre);
  if (a.v.rows <= 128) return product_few<128>(a, b, out, flags, st, pre);
  // 256 x 256 tiles on pairs of SMs move half the bytes per flop of 128 x 128 tiles, but there are a quarter as many.  A
  // round of them takes one and a half times as long.  bf16 results, single / pairs, us: 1024 x 1024 x 1024 4.5 / 5.9;
  // 256, 512, 768 and 1024 rows through 4096 x 4096 8.1 / 9.4, 8.3 / 9.5, 13.1 / 10.2, 13.3 / 10.4; 129, 256, 384 and 1024 rows
  // through 8192 x 8192 12.9 / 14.1, 13.0 / 14.1, 22.5 / 15.1, 41.8 / 25.2; 8192 x 2048 x 2048 22.2 / 17.2; 4096^3 38.2 / 26.4;
  // fp32 results alike.  The rule takes the shorter one in all of them.
  TilePlanMx4 t;
  const auto tiles = [&](int64_t side) { return ((a.v.rows + side - 1) / side) * ((b.v.rows + side - 1) / side); };
  const auto rounds = [](int64_t n, int64_t at_once) { return (n + at_once - 1) / at_once; };
  const bool pairs = 3 * rounds(tiles(256), num_sms() / 2) <= 2 * rounds(tiles(128), num_sms());
  int rc = pairs ? plan_tiles<256, 2>(a, b, out->data, flags, &t) : plan_tiles<128, 1>(a, b, out->data, flags, &t);
  if (rc) return rc;
  rc = pre();
  if (rc) return rc;
  return pairs ? run_tiles<256, 2>(t, st) : run_tiles<128, 1>(t, st);
}

size_t round_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

}  // namespace

namespace gl {
// The status words of the operators on narrow operands: this file's and gl_f8.cu's.
int take_status_mx4() {
  unsigned int v = 0;
  if (cudaMemcpyFromSymbol(&v, g_status, sizeof(v)) != cudaSuccess) return GL_ERR_CUDA;
  const int eight = take_status_f8();
  if (!v) return eight;
  const unsigned int zero = 0;
  if (cudaMemcpyToSymbol(g_status, &zero, sizeof(zero)) != cudaSuccess) return GL_ERR_CUDA;
  return eight ? eight : GL_ERR_TIMEOUT;
}
}  // namespace gl

extern "C" {

size_t gl_mx4_data_bytes(const gl_mx4* a) {
  Mx4View v;
  return check_mx4_meta(a, &v) ? 0 : static_cast<size_t>(v.rows) * v.pitch;
}

size_t gl_mx4_scale_bytes(const gl_mx4* a) {
  Mx4View v;
  return check_mx4_meta(a, &v) ? 0 : static_cast<size_t>(v.rt) * v.kt * 512;
}

int gl_mx4_quantize(const gl_ap* in, gl_mx4* out, void* stream) {
  int rc = check_data(in);
  if (rc) return rc;
  Mx4View v;
  rc = check_mx4_data(out, &v);
  if (rc) return rc;
  if (!same_shape(in, out)) return GL_ERR_SHAPE;
  return launch_quantize(*in, v, out->data, out->scale, static_cast<cudaStream_t>(stream));
}

int gl_mx4_dequantize(const gl_mx4* in, gl_ap* out, void* stream) {
  Mx4View v;
  int rc = check_mx4_data(in, &v);
  if (rc) return rc;
  rc = check_data(out);
  if (rc) return rc;
  if (!same_shape(out, in)) return GL_ERR_SHAPE;
  QuantParams p;
  rc = quant_params(v, 8, &p);
  if (rc) return rc;
  const bool f32 = out->dtype == GL_F32, vec = v.K % 8 == 0;
  constexpr int kU = kItemsPerThread;
  void (*k)(const uint8_t*, const uint8_t*, void*, QuantParams) =
      many_items(p) ? (f32 ? (vec ? dequantize_mx4<true, true, kU> : dequantize_mx4<true, false, kU>)
                           : (vec ? dequantize_mx4<false, true, kU> : dequantize_mx4<false, false, kU>))
                    : (f32 ? (vec ? dequantize_mx4<true, true, 1> : dequantize_mx4<true, false, 1>)
                           : (vec ? dequantize_mx4<false, true, 1> : dequantize_mx4<false, false, 1>));
  return launch_pdl(k, item_grid(p), dim3(256), 0, static_cast<cudaStream_t>(stream), 1, static_cast<const uint8_t*>(in->data),
                    static_cast<const uint8_t*>(in->scale), out->data, p) == cudaSuccess ? GL_OK : GL_ERR_CUDA;
}

int gl_cartesian_dot_mx4(const gl_mx4* a0, const gl_mx4* a1, gl_ap* out, uint32_t flags, void* stream) {
  Mx4Operand a, b;
  int rc = check_mx4_data(a0, &a.v);
  if (rc) return rc;
  rc = check_mx4_data(a1, &b.v);
  if (rc) return rc;
  rc = check_product(out, a0->access_ndim, a0->shape, a0->ndim - a0->access_ndim, a1, flags);
  if (rc) return rc;
  a.codes = a0->data;
  a.scale = a0->scale;
  b.codes = a1->data;
  b.scale = a1->scale;
  return product(a, b, out, flags, static_cast<cudaStream_t>(stream), [] { return GL_OK; });
}

size_t gl_dense_mx4_workspace(const gl_ap* a0, const gl_mx4* a1) {
  Mx4View v;
  if (check_meta(a0) || check_mx4_meta(a1, &v)) return 0;
  gl_mx4 q;
  std::memset(&q, 0, sizeof(q));
  q.ndim = a0->ndim;
  q.access_ndim = a0->access_ndim;
  for (int i = 0; i < a0->ndim; ++i) q.shape[i] = a0->shape[i];
  return round_up(gl_mx4_data_bytes(&q), 1024) + gl_mx4_scale_bytes(&q);
}

int gl_dense_mx4(const gl_ap* a0, const gl_mx4* a1, gl_ap* out, uint32_t flags, void* workspace, size_t workspace_bytes,
                 void* stream) {
  int rc = check_data(a0);
  if (rc) return rc;
  Mx4Operand a, b;
  rc = check_mx4_data(a1, &b.v);
  if (rc) return rc;
  rc = check_product(out, a0->access_ndim, a0->shape, a0->ndim - a0->access_ndim, a1, flags);
  if (rc) return rc;
  gl_mx4 q;
  std::memset(&q, 0, sizeof(q));
  q.ndim = a0->ndim;
  q.access_ndim = a0->access_ndim;
  for (int i = 0; i < a0->ndim; ++i) q.shape[i] = a0->shape[i];
  const size_t need = gl_dense_mx4_workspace(a0, a1);
  if (need && (!workspace || workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 1023u))) return GL_ERR_WORKSPACE;
  q.data = workspace;
  q.scale = static_cast<char*>(workspace) + round_up(gl_mx4_data_bytes(&q), 1024);
  rc = check_mx4_data(&q, &a.v);
  if (rc) return rc;
  QuantParams qp;
  rc = quant_params(a.v, 8, &qp);
  if (rc) return rc;
  b.codes = a1->data;
  b.scale = a1->scale;
  a.codes = q.data;
  a.scale = q.scale;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (a.v.rows <= kFuseRows) {
    if (!driver_api().ok) return GL_ERR_CUDA;
    FewPlan t;
    rc = plan_few<16, true>(a, b, out->data, flags, &t);
    if (rc) return rc;
    if ((t.p.kblocks + t.p.split - 1) / t.p.split <= kFuseBlocks) {
      t.p.x = a0->data;
      t.p.K = a.v.K;
      t.p.x_f32 = a0->dtype == GL_F32;
      return run_few<16, true>(t, st);
    }
  }
  return product(a, b, out, flags, st, [&] { return launch_quantize(*a0, a.v, q.data, q.scale, st); });
}

}  // extern "C"
