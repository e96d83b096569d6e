// The 8-bit number format, shared by the kernel files: blocks of 128 consecutive values of an item, E4M3 codes (magnitudes up to
// 448) and an E8M0 scale 2^(e - 127) per block; e = 255 stands for NaN.
//
// A warp works on units of 256 values, two blocks, eight values a lane:
//   aligned rows (VEC): lane l holds values 8l .. 8l+7, one or two 16-byte loads, lanes 0-15 the first block;
//   other rows:         lane l holds values 32j + l, j = 0..7, j < 4 the first block, so that loads and stores of neighbouring
//                       lanes still fall next to each other.
// Scales are stored in tiles of 128 rows x 4 blocks (512 bytes), row r and block b of a tile at byte
// (r % 32) * 16 + (r / 32) * 4 + b: what one tcgen05.cp (32x128b, replicated to the four lane quarters) has to find.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>
#include <cstring>

#include "gl_internal.h"

namespace {

constexpr int kF8Block = 128;
constexpr int kF8Unit = 256;   // values of a warp's unit

struct F8View {
  int64_t rows, K;
  int64_t pitch;    // bytes per row of codes
  int64_t nb;       // blocks per row
  int64_t kt, rt;   // scale tiles along K (4 blocks each) and along the rows (128 each)
};

inline int check_f8_meta(const gl_f8* a, F8View* v) {
  if (!a) return GL_ERR_NULL;
  if (a->ndim < 0 || a->ndim > GL_MAX_DIMS) return GL_ERR_NDIM;
  if (a->access_ndim < 0 || a->access_ndim > a->ndim) return GL_ERR_NDIM;
  int64_t side[2] = {1, 1};   // rows, K: each bounded before the next factor
  for (int i = 0; i < a->ndim; ++i) {
    if (a->shape[i] < 1) return GL_ERR_SHAPE;
    int64_t& n = side[i >= a->access_ndim];
    if (a->shape[i] > (int64_t{1} << 40) / n) return GL_ERR_UNSUPPORTED;
    n *= a->shape[i];
  }
  v->rows = side[0];
  v->K = side[1];
  v->pitch = (v->K + 15) / 16 * 16;
  v->nb = (v->K + kF8Block - 1) / kF8Block;
  v->kt = (v->nb + 3) / 4;
  v->rt = (v->rows + 127) / 128;
  // item indices are 32-bit in the kernels, blocks of the whole operand too
  if (v->rows > INT32_MAX - 256 || v->K > (int64_t{1} << 30) || v->rows * (v->nb + 1) > INT32_MAX) return GL_ERR_UNSUPPORTED;
  return GL_OK;
}

inline int check_f8_data(const gl_f8* a, F8View* v) {
  const int rc = check_f8_meta(a, v);
  if (rc) return rc;
  if (!a->data || !a->scale) return GL_ERR_NULL;
  if ((reinterpret_cast<uintptr_t>(a->data) | reinterpret_cast<uintptr_t>(a->scale)) & 15u) return GL_ERR_ALIGN;
  return GL_OK;
}

inline bool f8_same_shape(const gl_ap* a, const gl_f8* b) {
  if (a->ndim != b->ndim || a->access_ndim != b->access_ndim) return false;
  for (int i = 0; i < a->ndim; ++i)
    if (a->shape[i] != b->shape[i]) return false;
  return true;
}

// Scale exponent of a block whose largest magnitude has the bits `top`: the smallest power of two that brings it to 448 = 1.75 *
// 2^8 or below.  Adding the mantissa bits above 1.75 carries into the exponent.  An Inf or a NaN makes the block NaN.
__device__ __forceinline__ uint32_t f8_exponent(uint32_t top) {
  const uint32_t b = (top + 0x1FFFFFu) >> 23;
  return top >= 0x7F800000u ? 255u : (b > 8u ? b - 8u : 0u);
}
// 2^(127 - e), exact; 0 for a NaN block, whose codes are zeros
__device__ __forceinline__ float f8_inverse(uint32_t e) { return e == 255u ? 0.f : __uint_as_float((254u - e) << 23); }
// 2^(e - 127) as fp32 (e = 0 is subnormal), NaN for e = 255
__device__ __forceinline__ float f8_scale(uint32_t e) {
  return e == 255u ? __uint_as_float(0x7FC00000u) : __uint_as_float(max(e << 23, 0x00400000u));
}
// Two values (already divided by the scale) to two codes, `lo` in the low byte, nearest even.
__device__ __forceinline__ uint32_t f8_codes2(float lo, float hi) {
  uint16_t d;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(d) : "f"(hi), "f"(lo));
  return d;
}
__device__ __forceinline__ uint32_t f8_codes4(float a, float b, float c, float d) { return f8_codes2(a, b) | f8_codes2(c, d) << 16; }

// Byte of the scale tiles that holds block b of row r.
__device__ __forceinline__ int64_t f8_scale_at(uint32_t r, uint32_t b, uint32_t kt) {
  return (static_cast<int64_t>(r >> 7) * kt + (b >> 2)) * 512 + ((r & 31u) * 16 + ((r >> 5) & 3u) * 4 + (b & 3u));
}

// Place of a lane's value j inside a unit.
template <bool VEC>
__device__ __forceinline__ int unit_at(int lane, int j) { return VEC ? lane * 8 + j : j * 32 + lane; }

// Eight values of the row that starts at `row` (element `k0` is the unit's first), zeros behind K.
template <bool F32, bool VEC>
__device__ __forceinline__ void unit_load(const void* __restrict__ row, int k0, int K, int lane, uint32_t (&raw)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) raw[j] = 0;
  if (VEC) {   // K is a multiple of 8: a lane's values lie wholly inside the row or wholly behind it
    const int at = k0 + lane * 8;
    if (at < K) {
      const uint4* src = reinterpret_cast<const uint4*>(static_cast<const char*>(row) + static_cast<int64_t>(at) * (F32 ? 4 : 2));
#pragma unroll
      for (int i = 0; i < (F32 ? 2 : 1); ++i) {
        const uint4 x = __ldcs(src + i);
        raw[4 * i] = x.x; raw[4 * i + 1] = x.y; raw[4 * i + 2] = x.z; raw[4 * i + 3] = x.w;
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int at = k0 + j * 32 + lane;
      if (at < K) raw[j] = F32 ? static_cast<const uint32_t*>(row)[at] : static_cast<const uint16_t*>(row)[at];
    }
  }
}
// What unit_load brought, as fp32.
template <bool F32, bool VEC>
__device__ __forceinline__ float unit_value(const uint32_t (&raw)[8], int j) {
  if (F32) return __uint_as_float(raw[j]);
  if (VEC) return __uint_as_float(j & 1 ? raw[j >> 1] & 0xFFFF0000u : raw[j >> 1] << 16);
  return __uint_as_float(raw[j] << 16);
}

// A unit's eight values per lane to codes and scales.  `codes`: the row of codes, `scale`: the scale byte of the unit's first
// block (even, so that both bytes are one aligned store; a second block behind the row's end has room in the tile).
// Every lane of the warp takes part.
template <bool VEC>
__device__ __forceinline__ void unit_store_f8(const float (&v)[8], uint8_t* __restrict__ codes, int k0, int pitch, int lane,
                                              uint8_t* __restrict__ scale) {
  uint32_t top[2] = {0, 0};
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    uint32_t& t = top[!VEC && j >= 4];
    t = max(t, __float_as_uint(v[j]) & 0x7FFFFFFFu);
  }
#pragma unroll
  for (int d = 1; d < (VEC ? 16 : 32); d *= 2) {
    top[0] = max(top[0], __shfl_xor_sync(0xFFFFFFFFu, top[0], d));
    if (!VEC) top[1] = max(top[1], __shfl_xor_sync(0xFFFFFFFFu, top[1], d));
  }
  const uint32_t e0 = f8_exponent(top[0]);
  if (VEC) {
    const float f = f8_inverse(e0);
    const int at = k0 + lane * 8;
    if (at < pitch)   // (the pitch is a multiple of 16; values behind K are zeros)
      *reinterpret_cast<uint2*>(codes + at) =
          make_uint2(e0 == 255u ? 0u : f8_codes4(v[0] * f, v[1] * f, v[2] * f, v[3] * f),
                     e0 == 255u ? 0u : f8_codes4(v[4] * f, v[5] * f, v[6] * f, v[7] * f));
    const uint32_t e1 = __shfl_sync(0xFFFFFFFFu, e0, 16);
    if (lane == 0) *reinterpret_cast<uint16_t*>(scale) = static_cast<uint16_t>(e0 | e1 << 8);
  } else {
    const uint32_t e1 = f8_exponent(top[1]);
    const float f0 = f8_inverse(e0), f1 = f8_inverse(e1);
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
      const bool nan = (j < 4 ? e0 : e1) == 255u;
      const float f = j < 4 ? f0 : f1;
      const uint32_t two = nan ? 0u : f8_codes2(v[j] * f, v[j + 1] * f);
      const int at = k0 + j * 32 + lane;
      if (at < pitch) codes[at] = static_cast<uint8_t>(two);
      if (at + 32 < pitch) codes[at + 32] = static_cast<uint8_t>(two >> 8);
    }
    if (lane == 0) *reinterpret_cast<uint16_t*>(scale) = static_cast<uint16_t>(e0 | e1 << 8);
  }
}

}  // namespace
