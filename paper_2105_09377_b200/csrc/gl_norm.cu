// compute norm_rms: items divided by their root mean square, optionally with a residual added first, results as GL_BF16,
// GL_F32 or as an F8 operand.
//   h = x + residual;  sum = h in the residual's type;  y = h / sqrt(mean(h^2) + eps) * weight
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <initializer_list>

#include "gl_f8.cuh"
#include "gl_internal.h"
#include "gl_launch.cuh"
#include "gl_tc.cuh"
#include "gl_tmap.h"

using namespace gl;

namespace {

enum { kNone = 0, kBf16 = 1, kF32 = 2 };              // types of the residual and of the weights
enum { kOutBf16 = 0, kOutF32 = 1, kOutF8 = 2 };

struct NormParams {
  const void* x;
  const void* res;
  const void* weight;
  void* sum;
  void* out;             // values, or codes
  uint8_t* scale;        // F8 only
  uint32_t rows;
  int32_t K, pitch;
  uint32_t kt;
  int32_t units;         // units of 256 values per row
  int32_t weight_type;
  FastDiv row_warps;     // warps per row
  int32_t block_rows;    // rows per block
  float eps, inv_k;
};

// Weights of unit c, eight a lane (one row: always at a boundary, the last ones alone).
__device__ __forceinline__ void load_weights(const NormParams& p, int k, int c, float2 (&w)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = make_float2(1.f, 1.f);
  const int at = k + c * kF8Unit, left = p.K - at;
  if (p.weight_type == kNone || left <= 0) return;
  if (left >= 8) {
    if (p.weight_type == kF32) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float4 v = __ldg(reinterpret_cast<const float4*>(static_cast<const float*>(p.weight) + at) + i);
        w[2 * i] = make_float2(v.x, v.y);
        w[2 * i + 1] = make_float2(v.z, v.w);
      }
    } else {
      const uint4 v = __ldg(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.weight) + at));
      const uint32_t raw[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = make_float2(__uint_as_float(raw[i] << 16), __uint_as_float(raw[i] & 0xFFFF0000u));
    }
  } else {
    float x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j)
      x[j] = j >= left ? 0.f
             : p.weight_type == kF32 ? __ldg(static_cast<const float*>(p.weight) + at + j)
                                     : bf16_to_f32(__ldg(static_cast<const uint16_t*>(p.weight) + at + j));
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = make_float2(x[2 * i], x[2 * i + 1]);
  }
}

// A warp's strip of a row: where its operands and results lie.
template <bool XF32, int RES, int OUT>
struct Strip {
  LaneAt x, r, o;
  uint8_t* codes;
  uint8_t* scale;
  int k, room;
  __device__ __forceinline__ Strip(const NormParams& p, uint32_t row, int k0, int lane)
      : x(row, p.rows, k0, p.K, lane, XF32 ? 4 : 2), r(row, p.rows, k0, p.K, lane, RES == kF32 ? 4 : 2),
        o(row, p.rows, k0, p.K, lane, OUT == kOutF32 ? 4 : 2),
        codes(static_cast<uint8_t*>(p.out) + static_cast<int64_t>(row) * p.pitch + k0 + lane * 8),
        scale(p.scale + f8_scale_at(row, static_cast<uint32_t>(k0) / kF8Block, p.kt)), k(k0 + lane * 8), room(p.pitch - k0 - lane * 8) {}
};

// h of unit c from what was read.
template <bool XF32, int RES, bool VEC, typename S>
__device__ __forceinline__ void add_residual(const Unit<XF32, VEC>& x, const Unit<RES == kF32, VEC>& r, const S& at, int c, float2 (&h)[4]) {
  unit_values(x, at.x, c, h);
  if (RES != kNone) {
    float2 v[4];
    unit_values(r, at.r, c, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = add2(h[i], v[i]);
  }
}

template <int OUT, bool VEC, typename S>
__device__ __forceinline__ void store_result(const float2 (&h)[4], float rs, const NormParams& p, const S& at, int c, int lane) {
  float2 y[4];
  load_weights(p, at.k, c, y);
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = mul2(mul2(h[i], make_float2(rs, rs)), y[i]);
  if (OUT == kOutF8) unit_store_f8(y, at.codes, at.room, at.scale, c, lane);
  else unit_store<OUT == kOutF32, VEC>(y, p.out, at.o, c, lane);
}

// Sum over the warps of a row, the block's warps from `first` on, G sums each; `slots` holds all of them, added in their order.  All
// threads of the block call it.
template <int G>
__device__ __forceinline__ float row_sum(float (&s)[G], float* slots, int first, int row_warps) {
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) s[g] += __shfl_xor_sync(0xFFFFFFFFu, s[g], d);
  if (G == 1 && row_warps == 1) return s[0];
  if ((threadIdx.x & 31) == 0) {
#pragma unroll
    for (int g = 0; g < G; ++g) slots[(threadIdx.x >> 5) * G + g] = s[g];
  }
  __syncthreads();
  float sum = 0.f;
  for (int w = 0; w < row_warps * G; ++w) sum += slots[first * G + w];
  return sum;
}

// A row stays in registers between the sum of its squares and its results: strips of C units a warp, `row_warps` warps a row, as
// many rows a block as fit.  Everything is read once.  Bound by HBM where a residual is added: 16384 x 8192 bf16 into F8 143 us, 6.6
// TB/s (940 MB), into bf16 159 us, fp32 throughout 160 us for 8192 x 8192.  Without a residual into bf16 81 us, 6.7 TB/s, into F8 85
// us, 4.7 TB/s (74 without weights): 122 instructions a unit (into bf16 87) on 74 % of the issue slots, and fewer bytes in flight.
// Rows that start anywhere: 8192 x 8191 bf16 122 us (79 aligned), fp32 185 us.  A row alone, 8192: 2.6 us, a launch that does next to
// nothing 2.0.
template <bool XF32, int RES, int OUT, bool VEC, int C>
__global__ void __launch_bounds__(C >= 4 ? 512 : 1024) norm_rms(const NormParams p) {
  __shared__ float slots[32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint32_t block_row, row_warp;
  p.row_warps.divmod(static_cast<uint32_t>(warp), block_row, row_warp);
  const uint32_t row = blockIdx.x * p.block_rows + block_row;
  const int k0 = static_cast<int>(row_warp) * (C * kF8Unit);
  const bool live = row < p.rows;
  const Strip<XF32, RES, OUT> at(p, row, k0, lane);
  pdl_wait();
  Unit<XF32, VEC> x[C];
  Unit<RES == kF32, VEC> r[C];
  if (live) {
    units_read<XF32, VEC, C>(p.x, at.x, x);
    if (RES != kNone) units_read<RES == kF32, VEC, C>(p.res, at.r, r);
  }
  // (bf16 rows without a residual are held as they came, in half the registers, and converted twice)
  constexpr bool kHeldRaw = RES == kNone && !XF32 && VEC;
  // Eight units are summed as two warps' four each: the order of a row's sum, and so its F8 result, is that of its fp32 result.
  constexpr int kSums = C == 8 ? 2 : 1;
  float2 h[kHeldRaw ? 1 : C][4], pair[kSums];
  float s[kSums];
#pragma unroll
  for (int g = 0; g < kSums; ++g) pair[g] = make_float2(0.f, 0.f);
#pragma unroll
  for (int c = 0; c < C; ++c) {
    if (!live || k0 + c * kF8Unit >= p.K) break;
    float2(&v)[4] = h[kHeldRaw ? 0 : c];
    add_residual<XF32, RES, VEC>(x[c], r[c], at, c, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) pair[kSums == 2 ? c / 4 : 0] = fma2(v[i], v[i], pair[kSums == 2 ? c / 4 : 0]);
    if (RES != kNone && p.sum) unit_store<RES == kF32, VEC>(v, p.sum, at.r, c, lane);
  }
  // (The next kernel may start now: at the top its prefetches would stand in the way of this one's operands.  The norm and a product
  // behind it, 1 x 8192 x 8192: 16.6 -> 15.9 us, 128 x 4096 x 4096: 14.0 -> 12.3 us.)
  pdl_launch_dependents();
#pragma unroll
  for (int g = 0; g < kSums; ++g) s[g] = pair[g].x + pair[g].y;
  // (rsqrtf is off by up to 2.1 * 2^-24 and 0.47 * 2^-24 on the average over all mantissas, 1 / sqrtf by 1.5 and 0.50)
  const float rs = rsqrtf(row_sum(s, slots, warp - static_cast<int>(row_warp), static_cast<int>(p.row_warps.d)) * p.inv_k + p.eps);
#pragma unroll
  for (int c = 0; c < C; ++c) {
    if (!live || k0 + c * kF8Unit >= p.K) break;
    if (kHeldRaw) {
#pragma unroll
      for (int i = 0; i < Unit<XF32, VEC>::kHeld; ++i) asm volatile("" : "+r"(x[c].w[i]));   // (not the first conversion's results)
      unit_values(x[c], at.x, c, h[0]);
    }
    store_result<OUT, VEC>(h[kHeldRaw ? 0 : c], rs, p, at, c, lane);
  }
}

// Rows that do not fit in a block's registers: a block per row, read twice (the second time mostly from L2).  Nothing is written
// before a value's second reading, so results may take the operands' place here too.
template <bool XF32, int RES, int OUT, bool VEC>
__global__ void __launch_bounds__(1024) norm_rms_long(const NormParams p) {
  __shared__ float slots[32];
  const int lane = threadIdx.x & 31;
  const uint32_t row = blockIdx.x;
  pdl_wait();
  pdl_launch_dependents();
  // (In 64 bits: a lane adds up 2^15 units of eight squares for the longest rows, 2^18 values, and where these are much alike every
  // addition to an fp32 sum is rounded the same way: rows of one value came out up to 93 * 2^-24 off at 2^23 values and 410 * 2^-24 at
  // 2^25.  4096 x 32768 155 us either way.)
  double total = 0.0;
  Unit<XF32, VEC> x[1];
  Unit<RES == kF32, VEC> r[1];
  float2 h[4];
  for (int unit = threadIdx.x >> 5; unit < p.units; unit += 32) {
    const Strip<XF32, RES, OUT> at(p, row, unit * kF8Unit, lane);
    units_read<XF32, VEC, 1>(p.x, at.x, x);
    if (RES != kNone) units_read<RES == kF32, VEC, 1>(p.res, at.r, r);
    add_residual<XF32, RES, VEC>(x[0], r[0], at, 0, h);
    float2 s = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < 4; ++i) s = fma2(h[i], h[i], s);
    total += static_cast<double>(s.x + s.y);
  }
  float lane_sum[1] = {static_cast<float>(total)};
  const float rs = rsqrtf(row_sum(lane_sum, slots, 0, 32) * p.inv_k + p.eps);
  for (int unit = threadIdx.x >> 5; unit < p.units; unit += 32) {
    const Strip<XF32, RES, OUT> at(p, row, unit * kF8Unit, lane);
    units_read<XF32, VEC, 1>(p.x, at.x, x);
    if (RES != kNone) units_read<RES == kF32, VEC, 1>(p.res, at.r, r);
    add_residual<XF32, RES, VEC>(x[0], r[0], at, 0, h);
    if (RES != kNone && p.sum) unit_store<RES == kF32, VEC>(h, p.sum, at.r, 0, lane);
    store_result<OUT, VEC>(h, rs, p, at, 0, lane);
  }
}

// Rows of up to 128 values (a head's, say), several side by side in a warp, whatever the result's type; a lane's weights are the same
// for all of its rows.  Against a unit per row: 327680 x 128 bf16 53 -> 27 us (6.3 TB/s), with a residual into F8 80 -> 47, x 64 52 ->
// 14 and 79 -> 25, fp32 throughout with a residual 100 and 99; 20000 x 128 into F8 6.0 -> 3.8, 40 x 128 1.5 -> 1.2.
template <bool XF32, int RES, int OUT, int U>
__global__ void __launch_bounds__(256) norm_rms_short(const NormParams p, const ShortRows r) {
  pdl_wait();
  pdl_launch_dependents();
  Unit<XF32, true> x[U];
  Unit<RES == kF32, true> res[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const ShortAt at(r, U, u);
    short_read(p.x, r, at, x[u]);
    if (RES != kNone) short_read(p.res, r, at, res[u]);
  }
  float2 w[4];
  load_weights(p, (threadIdx.x & (r.lanes - 1)) * 8, 0, w);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const ShortAt at(r, U, u);
    float2 h[4], s = make_float2(0.f, 0.f);
    short_values(x[u], h);
    if (RES != kNone) {
      float2 v[4];
      short_values(res[u], v);
#pragma unroll
      for (int i = 0; i < 4; ++i) h[i] = add2(h[i], v[i]);
      if (p.sum) short_store<RES == kF32>(h, p.sum, r, at);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) s = fma2(h[i], h[i], s);
    float sum = s.x + s.y;
    for (int d = 1; d < r.lanes; d *= 2) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
    const float rs = rsqrtf(sum * p.inv_k + p.eps);
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = mul2(mul2(h[i], make_float2(rs, rs)), w[i]);
    if (OUT == kOutF8) short_store_f8(h, static_cast<uint8_t*>(p.out), p.scale, r, at);
    else short_store<OUT == kOutF32>(h, p.out, r, at);
  }
}

// Rows of `row_warps` warps with C units each.
template <bool XF32, int RES, int OUT, bool VEC, int C>
int launch_strips(NormParams p, int row_warps, cudaStream_t st) {
  p.row_warps.set(row_warps);
  p.block_rows = std::max(8 / row_warps, 1);
  const dim3 grid((p.rows + p.block_rows - 1) / p.block_rows), block(static_cast<unsigned>(row_warps * p.block_rows * 32));
  return launch_pdl(norm_rms<XF32, RES, OUT, VEC, C>, grid, block, 0, st, 1, p) == cudaSuccess ? GL_OK : GL_ERR_CUDA;
}

template <bool XF32, int RES, int OUT, bool VEC>
int launch_norm(const NormParams& p, cudaStream_t st) {
  // Four units a warp (two of unaligned rows, which take more registers) when there are rows enough to fill the machine; a row
  // alone is spread over as many warps as it has units.
  // Eight where a row is held as bf16 and its result is F8, if that leaves no warp with less and every SM its 28 warps (and the row
  // would fit in registers by fours too): 16384 x 8192 97.6 -> 84.8 us, 16384 x 4096 51.1 -> 46.4, but 300 x 8192 4.9 -> 6.1 and
  // 2048 x 5120 11.2 -> 14.9; into bf16 16384 x 8192 80.6 -> 82.7.
  constexpr int kMost = VEC ? 4 : 2;
  constexpr bool kEight = VEC && !XF32 && RES == kNone && OUT == kOutF8;
  if (kEight && p.units % 8 == 0 && p.units <= 64 && static_cast<int64_t>(p.rows) * p.units >= static_cast<int64_t>(num_sms()) * 28 * 8)
    return launch_strips<XF32, RES, OUT, VEC, kEight ? 8 : kMost>(p, p.units / 8, st);
  const bool spread = p.rows <= static_cast<uint32_t>(num_sms());
  const int row_warps = std::min(spread ? p.units : (p.units + kMost - 1) / kMost, 32);
  const int per_warp = (p.units + row_warps - 1) / row_warps;
  if (per_warp == 1) return launch_strips<XF32, RES, OUT, VEC, 1>(p, row_warps, st);
  if (per_warp == 2) return launch_strips<XF32, RES, OUT, VEC, 2>(p, row_warps, st);
  if (VEC && row_warps <= 16) return launch_strips<XF32, RES, OUT, VEC, kMost>(p, row_warps, st);   // (then four units a warp suffice)
  return launch_pdl(norm_rms_long<XF32, RES, OUT, VEC>, dim3(p.rows), dim3(1024), 0, st, 1, p) == cudaSuccess ? GL_OK : GL_ERR_CUDA;
}

template <bool XF32, int RES, int OUT>
int launch_vec(const NormParams& p, cudaStream_t st) {
  F8View v;
  v.rows = p.rows;
  v.K = p.K;
  v.pitch = p.pitch;
  if (is_short(v)) {
    const ShortRows r = short_rows(v);
    // beside a residual one group is enough (one and four, us: 40000 x 128 into F8 5.9 and 6.6, 160000 x 128 24.2 and 25.1)
    const int groups = RES == kNone ? short_groups(r, num_sms()) : 1;
    void (*k)(NormParams, ShortRows) = groups == 4 ? norm_rms_short<XF32, RES, OUT, RES == kNone ? 4 : 1> : norm_rms_short<XF32, RES, OUT, 1>;
    return launch_pdl(k, dim3(short_blocks(r, groups)), dim3(256), 0, st, 1, p, r) == cudaSuccess ? GL_OK : GL_ERR_CUDA;
  }
  return p.K % 8 == 0 ? launch_norm<XF32, RES, OUT, true>(p, st) : launch_norm<XF32, RES, OUT, false>(p, st);
}
template <bool XF32, int RES>
int launch_out(const NormParams& p, int out, cudaStream_t st) {
  switch (out) {
    case kOutBf16: return launch_vec<XF32, RES, kOutBf16>(p, st);
    case kOutF32: return launch_vec<XF32, RES, kOutF32>(p, st);
    default: return launch_vec<XF32, RES, kOutF8>(p, st);
  }
}
template <bool XF32>
int launch_res(const NormParams& p, int res, int out, cudaStream_t st) {
  switch (res) {
    case kNone: return launch_out<XF32, kNone>(p, out, st);
    case kBf16: return launch_out<XF32, kBf16>(p, out, st);
    default: return launch_out<XF32, kF32>(p, out, st);
  }
}

int type_of(const gl_ap* a) { return !a ? kNone : a->dtype == GL_F32 ? kF32 : kBf16; }

bool same_shape(const gl_ap* a, const gl_ap* b) {
  if (a->ndim != b->ndim || a->access_ndim != b->access_ndim) return false;
  for (int i = 0; i < a->ndim; ++i)
    if (a->shape[i] != b->shape[i]) return false;
  return true;
}

// Bytes that an operand or a result takes.
struct Place {
  uintptr_t at;
  size_t bytes;
};
Place place_of(const gl_ap* a) {
  size_t n = a->dtype == GL_F32 ? 4 : 2;
  for (int i = 0; i < a->ndim; ++i) n *= static_cast<size_t>(a->shape[i]);
  return {reinterpret_cast<uintptr_t>(a->data), n};
}
bool meet(const Place& a, const Place& b) { return a.at < b.at + b.bytes && b.at < a.at + a.bytes; }
// A result of the shape of operand `in` may take its place value for value; otherwise the two have to lie apart, as a block reads
// rows while others write theirs.
bool clash(const gl_ap* in, const gl_ap* out) {
  return in && out && !(in->data == out->data && in->dtype == out->dtype) && meet(place_of(in), place_of(out));
}
bool weight_or_sum_clash(const gl_ap* weight, const gl_ap* sum, const Place& out) {
  return (weight && meet(place_of(weight), out)) || (sum && meet(place_of(sum), out));
}

// Everything but the result, which the two entry points check themselves.
int norm_params(const gl_ap* x, const gl_ap* residual, const gl_ap* weight, float eps, const gl_ap* sum, NormParams* p) {
  int rc = check_data(x);
  if (rc) return rc;
  if (x->ndim == x->access_ndim) return GL_ERR_SHAPE;   // no compute dimensions to take the mean of
  if (residual) {
    rc = check_data(residual);
    if (rc) return rc;
    if (!same_shape(x, residual)) return GL_ERR_SHAPE;
  }
  if (sum) {
    if (!residual) return GL_ERR_NULL;
    rc = check_same_meta(*residual, sum);
    if (rc) return rc;
    rc = check_data(sum);
    if (rc) return rc;
  }
  if (weight) {
    rc = check_data(weight);
    if (rc) return rc;
    if (weight->access_ndim != 0 || weight->ndim != x->ndim - x->access_ndim) return GL_ERR_SHAPE;
    for (int i = 0; i < weight->ndim; ++i)
      if (weight->shape[i] != x->shape[x->access_ndim + i]) return GL_ERR_SHAPE;
  }
  if (!(eps >= 0.f) || std::isinf(eps)) return GL_ERR_SHAPE;
  gl_f8 as_items;   // (the limits are those of the F8 format, whatever the result's type)
  std::memset(&as_items, 0, sizeof(as_items));
  as_items.ndim = x->ndim;
  as_items.access_ndim = x->access_ndim;
  for (int i = 0; i < x->ndim; ++i) as_items.shape[i] = x->shape[i];
  F8View v;
  rc = check_f8_meta(&as_items, &v);
  if (rc) return rc;
  if (clash(x, sum) || clash(residual, sum) || (sum && weight && meet(place_of(weight), place_of(sum)))) return GL_ERR_UNSUPPORTED;
  std::memset(p, 0, sizeof(*p));
  p->x = x->data;
  p->res = residual ? residual->data : nullptr;
  p->weight = weight ? weight->data : nullptr;
  p->sum = sum ? sum->data : nullptr;
  p->rows = static_cast<uint32_t>(v.rows);
  p->K = static_cast<int32_t>(v.K);
  p->pitch = static_cast<int32_t>(v.pitch);
  p->kt = static_cast<uint32_t>(v.kt);
  p->units = static_cast<int32_t>((v.nb + 1) / 2);
  p->weight_type = type_of(weight);
  p->eps = eps;
  p->inv_k = static_cast<float>(1.0 / static_cast<double>(v.K));
  return GL_OK;
}

int run_norm(const gl_ap* x, const gl_ap* residual, const NormParams& p, int out, void* stream) {
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return x->dtype == GL_F32 ? launch_res<true>(p, type_of(residual), out, st) : launch_res<false>(p, type_of(residual), out, st);
}

}  // namespace

extern "C" {

int gl_compute_norm_rms(const gl_ap* x, const gl_ap* residual, const gl_ap* weight, float eps, gl_ap* sum, gl_ap* out, void* stream) {
  NormParams p;
  int rc = norm_params(x, residual, weight, eps, sum, &p);
  if (rc) return rc;
  rc = check_data(out);
  if (rc) return rc;
  if (!same_shape(x, out)) return GL_ERR_SHAPE;
  if (clash(x, out) || clash(residual, out) || weight_or_sum_clash(weight, sum, place_of(out))) return GL_ERR_UNSUPPORTED;
  p.out = out->data;
  return run_norm(x, residual, p, out->dtype == GL_F32 ? kOutF32 : kOutBf16, stream);
}

int gl_compute_norm_rms_f8(const gl_ap* x, const gl_ap* residual, const gl_ap* weight, float eps, gl_ap* sum, gl_f8* out, void* stream) {
  NormParams p;
  int rc = norm_params(x, residual, weight, eps, sum, &p);
  if (rc) return rc;
  F8View v;
  rc = check_f8_data(out, &v);
  if (rc) return rc;
  if (!f8_same_shape(x, out)) return GL_ERR_SHAPE;
  const Place codes = {reinterpret_cast<uintptr_t>(out->data), gl_f8_data_bytes(out)};
  const Place scale = {reinterpret_cast<uintptr_t>(out->scale), gl_f8_scale_bytes(out)};
  if (meet(codes, scale)) return GL_ERR_UNSUPPORTED;
  for (const Place& to : {codes, scale})
    if (meet(place_of(x), to) || (residual && meet(place_of(residual), to)) || weight_or_sum_clash(weight, sum, to)) return GL_ERR_UNSUPPORTED;
  p.out = out->data;
  p.scale = static_cast<uint8_t*>(out->scale);
  return run_norm(x, residual, p, kOutF8, stream);
}

}  // extern "C"
