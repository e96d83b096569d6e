// The 8-bit number format, shared by the kernel files: blocks of 128 consecutive values of an item, E4M3 codes (magnitudes up to
// 448) and an E8M0 scale 2^(e - 127) per block; e = 255 stands for NaN.
//
// A warp works on units of 256 values, two blocks: lane l holds values 8l .. 8l+7, lanes 0-15 the first block.  Where the rows of a
// pattern are multiples of 16 bytes (VEC) these are 16-byte accesses as they stand.  Other rows start anywhere: the same 16-byte
// accesses are made at the boundaries before, and the values shifted into place, by the same distance in all lanes.  Codes
// always start at a boundary.
// Scales are stored in tiles of 128 rows x 4 blocks (512 bytes), row r and block b of a tile at byte
// (r % 32) * 16 + (r / 32) * 4 + b: what one tcgen05.cp (32x128b, replicated to the four lane quarters) has to find.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>
#include <cstring>

#include "gl_internal.h"
#include "gl_tc.cuh"

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
  // item indices are 32-bit in the kernels, blocks of the whole operand too; 2^28 values of an item are 2^12 stretches of a product,
  // which fp32 adds up to 2^-12
  if (v->rows > INT32_MAX - 256 || v->K > (int64_t{1} << 28) || v->rows * (v->nb + 1) > INT32_MAX) return GL_ERR_UNSUPPORTED;
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

// Two fp32 operations an instruction.
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(reinterpret_cast<uint64_t&>(d)) : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)));
  return d;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(reinterpret_cast<uint64_t&>(d))
      : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)), "l"(reinterpret_cast<uint64_t&>(c)));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(reinterpret_cast<uint64_t&>(d)) : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)));
  return d;
}
__device__ __forceinline__ float2 sub2(float2 a, float2 b) {
  float2 d;
  asm("sub.rn.f32x2 %0, %1, %2;" : "=l"(reinterpret_cast<uint64_t&>(d)) : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)));
  return d;
}
// The larger magnitude; a NaN wins.
__device__ __forceinline__ float top_of(float a, float b) {
  float d;
  asm("{\n\t.reg .f32 x, y;\n\tabs.f32 x, %1;\n\tabs.f32 y, %2;\n\tmax.NaN.f32 %0, x, y;\n\t}" : "=f"(d) : "f"(a), "f"(b));
  return d;
}

// Byte of the scale tiles that holds block b of row r.
__device__ __forceinline__ int64_t f8_scale_at(uint32_t r, uint32_t b, uint32_t kt) {
  return (static_cast<int64_t>(r >> 7) * kt + (b >> 2)) * 512 + ((r & 31u) * 16 + ((r >> 5) & 3u) * 4 + (b & 3u));
}

// ---- units of patterns whose items are `K` values, in memory at `base` (16-byte aligned) ----

// Words i .. of `w` from byte `t` on (t < 16, even; a multiple of 4 for fp32).
template <int N, int OUT>
__device__ __forceinline__ void shift_words(uint32_t (&w)[N], int t, uint32_t (&out)[OUT]) {
#pragma unroll
  for (int i = 0; i + 2 < N; ++i) w[i] = (t & 8) ? w[i + 2] : w[i];
#pragma unroll
  for (int i = 0; i + 3 < N; ++i) w[i] = (t & 4) ? w[i + 1] : w[i];
#pragma unroll
  for (int i = 0; i < OUT; ++i) out[i] = i + 1 < N ? __funnelshift_r(w[i], w[i + 1], (t & 2) * 8) : w[i];
}

// A lane's place in a pattern whose items are `K` values: its values of unit c are the eight from byte at + c * 256 values on.
struct LaneAt {
  int64_t at;     // of the lane's first value in the strip's first unit
  int left;       // values of the row from there on
  int strip;      // values of the row from the strip's beginning on (the same for all lanes)
  bool inside;    // the 16 bytes that hold the row's last value lie wholly inside the pattern (the same for all lanes)
  __device__ __forceinline__ LaneAt(uint32_t row, uint32_t rows, int k0, int K, int lane, int value_bytes)
      : at((static_cast<int64_t>(row) * K + k0 + lane * 8) * value_bytes), left(K - k0 - lane * 8), strip(K - k0),
        inside(((static_cast<int64_t>(row) + 1) * K * value_bytes + 15 & ~int64_t{15}) <= static_cast<int64_t>(rows) * K * value_bytes) {}
};

// What a lane has read of a unit: its eight values, or the 16-byte pieces that hold them.
template <bool F32, bool VEC>
struct Unit {
  static constexpr int kWords = F32 ? 8 : 4, kHeld = kWords + (VEC ? 0 : 4);
  uint32_t w[kHeld];
};

// Requests unit c; nothing behind the row's end is read but what shares a piece with its last value.
template <bool F32, bool VEC>
__device__ __forceinline__ void unit_read(const void* base, const LaneAt& l, int c, Unit<F32, VEC>& u) {
  constexpr int kEs = F32 ? 4 : 2;
  const int left = l.left - c * kF8Unit, t = VEC ? 0 : static_cast<int>(l.at & 15), bytes = t + min(8, left) * kEs;
  const uint4* q = reinterpret_cast<const uint4*>(static_cast<const char*>(base) + l.at - t + c * kF8Unit * kEs);
#pragma unroll
  for (int i = 0; i < Unit<F32, VEC>::kHeld / 4; ++i) {
    uint4 x = make_uint4(0, 0, 0, 0);
    // (aligned rows are multiples of eight values: a lane's lie wholly inside or wholly behind; of the other rows a lane's last
    // piece is the next one's first, which comes from L1)
    if (VEC && left > 0) x = __ldcs(q + i);
    if (!VEC && left > 0 && 16 * i < bytes) x = q[i];
    u.w[4 * i] = x.x; u.w[4 * i + 1] = x.y; u.w[4 * i + 2] = x.z; u.w[4 * i + 3] = x.w;
  }
}

// The same value by value, for the rows whose last piece is not wholly inside the pattern.
template <bool F32, bool VEC>
__device__ __forceinline__ void unit_read_edge(const void* base, const LaneAt& l, int c, Unit<F32, VEC>& u) {
  constexpr int kEs = F32 ? 4 : 2;
  const int left = l.left - c * kF8Unit, t = static_cast<int>(l.at & 15), bytes = left > 0 ? t + min(8, left) * kEs : 0;
  const char* q = static_cast<const char*>(base) + l.at - t + c * kF8Unit * kEs;
#pragma unroll
  for (int i = 0; i < Unit<F32, VEC>::kHeld; ++i) u.w[i] = 0;
#pragma unroll
  for (int i = 0; i < Unit<F32, VEC>::kHeld * 4 / kEs; ++i)
    if (i * kEs >= t && i * kEs < bytes) {
      if (F32) u.w[i] = *reinterpret_cast<const uint32_t*>(q + 4 * i);
      else u.w[i >> 1] |= static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(q + 2 * i)) << (16 * (i & 1));
    }
}

// N units of a strip, all requested before the first is used (no branch lies between the requests).
template <bool F32, bool VEC, int N>
__device__ __forceinline__ void units_read(const void* base, const LaneAt& l, Unit<F32, VEC>* u) {
  if (VEC || l.inside) {
#pragma unroll
    for (int c = 0; c < N; ++c) unit_read(base, l, c, u[c]);
  } else {
#pragma unroll
    for (int c = 0; c < N; ++c) unit_read_edge(base, l, c, u[c]);
  }
}

// A unit's values as fp32, zeros behind the row's end.
template <bool F32, bool VEC>
__device__ __forceinline__ void unit_values(const Unit<F32, VEC>& u, const LaneAt& l, int c, float2 (&v)[4]) {
  constexpr int kWords = Unit<F32, VEC>::kWords;
  uint32_t x[8];
  if constexpr (VEC) {
#pragma unroll
    for (int i = 0; i < kWords; ++i) x[i] = u.w[i];
  } else {
    uint32_t w[kWords + 4], y[kWords];
#pragma unroll
    for (int i = 0; i < kWords + 4; ++i) w[i] = u.w[i];
    shift_words(w, static_cast<int>(l.at & 15), y);
#pragma unroll
    for (int i = 0; i < kWords; ++i) x[i] = y[i];
    if (l.strip - c * kF8Unit < kF8Unit) {   // the row's last, partial unit
      const int left = l.left - c * kF8Unit;
#pragma unroll
      for (int i = 0; i < kWords; ++i) {
        if (F32) x[i] = i < left ? x[i] : 0u;
        else x[i] = 2 * i + 1 < left ? x[i] : 2 * i < left ? x[i] & 0xFFFFu : 0u;
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    v[i] = F32 ? make_float2(__uint_as_float(x[2 * i & 7]), __uint_as_float(x[2 * i + 1 & 7]))
               : make_float2(__uint_as_float(x[i] << 16), __uint_as_float(x[i] & 0xFFFF0000u));
}

// Eight values per lane to unit c.  Every lane of the warp takes part, whether or not it has values.
template <bool F32, bool VEC>
__device__ __forceinline__ void unit_store(const float2 (&v)[4], void* base, const LaneAt& l, int c, int lane) {
  constexpr int kEs = F32 ? 4 : 2;
  char* p = static_cast<char*>(base) + l.at + c * kF8Unit * kEs;
  const int left = l.left - c * kF8Unit;
  uint32_t w[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (F32) { w[2 * i] = __float_as_uint(v[i].x); w[2 * i + 1] = __float_as_uint(v[i].y); }
    else { w[i] = pack_bf16x2(__float_as_uint(v[i].x), __float_as_uint(v[i].y)); w[4 + i] = 0; }
  }
  if (VEC && F32) {
    // two lanes' 64 bytes in two stores that each write whole 32-byte sectors: first the even lane's values, then the odd's
    const bool odd = lane & 1;
    uint32_t got[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) got[i] = __shfl_xor_sync(0xFFFFFFFFu, odd ? w[i] : w[4 + i], 1);
    const int pair = left + (odd ? 8 : 0);   // values from the even lane's first on
    uint4* o = reinterpret_cast<uint4*>(p - (odd ? 16 : 0));
    if (pair > 0) *o = odd ? make_uint4(got[0], got[1], got[2], got[3]) : make_uint4(w[0], w[1], w[2], w[3]);
    if (pair > 8) o[2] = odd ? make_uint4(w[4], w[5], w[6], w[7]) : make_uint4(got[0], got[1], got[2], got[3]);
  } else if (VEC) {
    if (left > 0) *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  } else if (l.strip - c * kF8Unit < kF8Unit) {
    // the row's last, partial unit
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < left) {
        if (F32) *reinterpret_cast<uint32_t*>(p + 4 * j) = w[j];
        else *reinterpret_cast<uint16_t*>(p + 2 * j) = static_cast<uint16_t>(w[j >> 1 & 3] >> (16 * (j & 1)));
      }
  } else if (F32) {
    // Whole 16-byte pieces between the boundaries: the lane before has the first one's beginning.  The unit's own first and last
    // bytes, whose pieces belong to other units too, go one word at a time.
    const int t = static_cast<int>(-l.at & 15), s = t >> 2;   // bytes, words to the first boundary
    uint32_t z[12], q[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) z[i] = __shfl_up_sync(0xFFFFFFFFu, w[4 + i], 1);
#pragma unroll
    for (int i = 0; i < 8; ++i) z[4 + i] = w[i];
    if (s == 0) {
#pragma unroll
      for (int i = 0; i < 2; ++i) reinterpret_cast<uint4*>(p)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
      return;
    }
    shift_words(z, t, q);
    uint4* o = reinterpret_cast<uint4*>(p + t - 16);
    if (lane > 0) o[0] = make_uint4(q[0], q[1], q[2], q[3]);
    o[1] = make_uint4(q[4], q[5], q[6], q[7]);
    uint32_t* words = reinterpret_cast<uint32_t*>(p);
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      if (lane == 0 && i < s) words[i] = w[i];
      if (lane == 31 && 7 - i >= 4 + s) words[7 - i] = w[7 - i];
    }
  } else {
    const int t = static_cast<int>(-l.at & 15);
    uint32_t z[8], q[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) { z[i] = __shfl_up_sync(0xFFFFFFFFu, w[i], 1); z[4 + i] = w[i]; }
    if (t == 0) {
      *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
      return;
    }
    shift_words(z, t, q);
    if (lane > 0) *reinterpret_cast<uint4*>(p + t - 16) = make_uint4(q[0], q[1], q[2], q[3]);
    // values before the first boundary (lane 0) and from it on (lane 31), two at a time where they share a word
    const bool mine = lane == 0 || lane == 31;
    if (t & 2) {
      if (lane == 0) *reinterpret_cast<uint16_t*>(p) = static_cast<uint16_t>(w[0]);
#pragma unroll
      for (int i = 0; i < 3; ++i)
        if (mine && (2 + 4 * i < t) == (lane == 0)) *reinterpret_cast<uint32_t*>(p + 2 + 4 * i) = __funnelshift_r(w[i], w[i + 1], 16);
      if (lane == 31) *reinterpret_cast<uint16_t*>(p + 14) = static_cast<uint16_t>(w[3] >> 16);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (mine && (4 * i < t) == (lane == 0)) *reinterpret_cast<uint32_t*>(p + 4 * i) = w[i];
    }
  }
}

// Unit c's eight values per lane to codes and scales.  `codes`: the lane's first code in the strip's first unit, `room`: bytes of
// the row of codes from there on, `scale`: the scale byte of the strip's first block.  A unit's two scales are one aligned store; a
// second block behind the row's end has room in the tile.  A strip of several units begins with an even one, so that its units
// lie in the scale tiles at fixed distances.  Every lane of the warp takes part.
__device__ __forceinline__ void unit_store_f8(const float2 (&v)[4], uint8_t* codes, int room, uint8_t* scale, int c, int lane) {
  float largest = top_of(top_of(top_of(v[0].x, v[0].y), top_of(v[1].x, v[1].y)), top_of(top_of(v[2].x, v[2].y), top_of(v[3].x, v[3].y)));
#pragma unroll
  for (int d = 1; d < 16; d *= 2) largest = top_of(largest, __shfl_xor_sync(0xFFFFFFFFu, largest, d));
  const uint32_t e = f8_exponent(__float_as_uint(largest) & 0x7FFFFFFFu);
  const float f = f8_inverse(e);
  float2 q[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) q[i] = mul2(v[i], make_float2(f, f));
  if (room > c * kF8Unit)   // (the pitch is a multiple of 16; values behind K are zeros)
    *reinterpret_cast<uint2*>(codes + c * kF8Unit) = make_uint2(e == 255u ? 0u : f8_codes4(q[0].x, q[0].y, q[1].x, q[1].y),
                                                                e == 255u ? 0u : f8_codes4(q[2].x, q[2].y, q[3].x, q[3].y));
  const uint32_t second = __shfl_sync(0xFFFFFFFFu, e, 16);
  if (lane == 0) *reinterpret_cast<uint16_t*>(scale + (c >> 1) * 512 + (c & 1) * 2) = static_cast<uint16_t>(e | second << 8);
}

// ---- rows of up to 128 values, a multiple of eight: several side by side in a warp ----

// A row takes `lanes` lanes, a power of two, of eight values each (those behind the row's end are idle); U groups of 32 / lanes rows a
// warp, one below the other.
struct ShortRows {
  uint32_t rows;
  int32_t K, pitch;
  int32_t lanes, log_lanes;
};

inline ShortRows short_rows(const F8View& v) {
  ShortRows r;
  r.rows = static_cast<uint32_t>(v.rows);
  r.K = static_cast<int32_t>(v.K);
  r.pitch = static_cast<int32_t>(v.pitch);
  r.lanes = 1;
  r.log_lanes = 0;
  while (r.lanes * 8 < r.K) { r.lanes *= 2; ++r.log_lanes; }
  return r;
}
inline bool is_short(const F8View& v) { return v.K <= 128 && v.K % 8 == 0; }
// Four groups a warp when that still fills every SM with 64 warps (one group and four, us: rounding 327680 x 128 bf16 27.7 and 22.1,
// 80000 x 128 8.1 and 7.4, 40000 x 128 4.9 and 5.8, 80000 x 64 4.8 and 5.6, 2560 x 128 1.4 and 1.9).
inline int short_groups(const ShortRows& r, int sms) {
  return static_cast<int64_t>(r.rows) * r.lanes >= static_cast<int64_t>(sms) * 64 * 4 * 32 ? 4 : 1;
}
inline unsigned short_blocks(const ShortRows& r, int groups) {   // of eight warps
  const int64_t per_block = static_cast<int64_t>(8) * groups * (32 / r.lanes);
  return static_cast<unsigned>((r.rows + per_block - 1) / per_block);
}

// Row of this lane in group u, its place in the row, and whether there is such a value.
struct ShortAt {
  uint32_t row;
  int k;
  bool live;
  __device__ __forceinline__ ShortAt(const ShortRows& r, int groups, int u) {
    const int lane = threadIdx.x & 31;
    const uint32_t warp = blockIdx.x * 8u + (threadIdx.x >> 5);
    row = ((warp * groups + u) << (5 - r.log_lanes)) + (lane >> r.log_lanes);
    k = (lane & (r.lanes - 1)) * 8;
    live = row < r.rows && k < r.K;
  }
};

template <bool F32>
__device__ __forceinline__ void short_read(const void* base, const ShortRows& r, const ShortAt& at, Unit<F32, true>& u) {
  const uint4* q = reinterpret_cast<const uint4*>(static_cast<const char*>(base) + (static_cast<int64_t>(at.row) * r.K + at.k) * (F32 ? 4 : 2));
#pragma unroll
  for (int i = 0; i < Unit<F32, true>::kHeld / 4; ++i) {
    uint4 x = make_uint4(0, 0, 0, 0);
    if (at.live) x = __ldcs(q + i);
    u.w[4 * i] = x.x; u.w[4 * i + 1] = x.y; u.w[4 * i + 2] = x.z; u.w[4 * i + 3] = x.w;
  }
}
template <bool F32>
__device__ __forceinline__ void short_values(const Unit<F32, true>& u, float2 (&v)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    v[i] = F32 ? make_float2(__uint_as_float(u.w[(2 * i) % Unit<F32, true>::kHeld]), __uint_as_float(u.w[(2 * i + 1) % Unit<F32, true>::kHeld]))
               : make_float2(__uint_as_float(u.w[i] << 16), __uint_as_float(u.w[i] & 0xFFFF0000u));
}
template <bool F32>
__device__ __forceinline__ void short_store(const float2 (&v)[4], void* base, const ShortRows& r, const ShortAt& at) {
  if (!at.live) return;
  char* p = static_cast<char*>(base) + (static_cast<int64_t>(at.row) * r.K + at.k) * (F32 ? 4 : 2);
  if (F32) {
    reinterpret_cast<float4*>(p)[0] = make_float4(v[0].x, v[0].y, v[1].x, v[1].y);
    reinterpret_cast<float4*>(p)[1] = make_float4(v[2].x, v[2].y, v[3].x, v[3].y);
  } else {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = pack_bf16x2(__float_as_uint(v[i].x), __float_as_uint(v[i].y));
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}
// Codes and scale of rows that are one block (one scale tile along K).  Every lane of the warp takes part.
__device__ __forceinline__ void short_store_f8(const float2 (&v)[4], uint8_t* codes, uint8_t* scale, const ShortRows& r, const ShortAt& at) {
  float largest = top_of(top_of(top_of(v[0].x, v[0].y), top_of(v[1].x, v[1].y)), top_of(top_of(v[2].x, v[2].y), top_of(v[3].x, v[3].y)));
  for (int d = 1; d < r.lanes; d *= 2) largest = top_of(largest, __shfl_xor_sync(0xFFFFFFFFu, largest, d));
  if (!at.live) return;
  const uint32_t e = f8_exponent(__float_as_uint(largest) & 0x7FFFFFFFu);
  const float f = f8_inverse(e);
  float2 q[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) q[i] = mul2(v[i], make_float2(f, f));
  uint2* to = reinterpret_cast<uint2*>(codes + static_cast<int64_t>(at.row) * r.pitch + at.k);
  to[0] = make_uint2(e == 255u ? 0u : f8_codes4(q[0].x, q[0].y, q[1].x, q[1].y), e == 255u ? 0u : f8_codes4(q[2].x, q[2].y, q[3].x, q[3].y));
  if (at.k + 8 == r.K && r.K < r.pitch) to[1] = make_uint2(0u, 0u);   // (the pitch is the next multiple of 16)
  if (at.k == 0) scale[f8_scale_at(at.row, 0, 1)] = static_cast<uint8_t>(e);
}

}  // namespace
