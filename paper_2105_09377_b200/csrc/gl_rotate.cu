// compute rotate: rotary positions with several axes.  Pairs of a head's values are turned by the angle
// position[axis of the pair] * frequency of the pair.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <numeric>

#include "gl_f8.cuh"
#include "gl_internal.h"
#include "gl_launch.cuh"
#include "gl_tc.cuh"
#include "gl_tmap.h"

using namespace gl;

namespace {

// Angles are 64-bit fractions of a turn: step (2^64 times the turns per position) times position, modulo 2^64.  Whole turns fall
// out of the integer product by themselves and the rest is as exact as the step, which is off by half a unit or little more; an fp32
// product of position and frequency is off by a sixteenth of a radian at a million tokens.
//
// A block takes a few tokens: cosines and sines of its tokens once into shared memory, then every thread takes one group of W
// pairs, 2W values, of head after head, kRotRows of them requested before the first is used (the first ones before the angles
// are computed).  Bound by HBM where there are heads enough to hide the angles: 8198 tokens x 40 heads x 128 bf16 30.4 us, 5.5 TB/s
// (two heads in flight 37 us), fp32 51.7 us, 6.5 TB/s; one head of 128 at 8192 tokens 5.4 us, 64 tokens x 40 heads 2.2 us.
constexpr int kRotThreads = 256;
constexpr int kRotRows = 4;           // heads of a thread in flight
constexpr int kRotAngles = 512;       // angles of a block of several tokens

struct RotateParams {
  const void* x;
  void* out;
  const int32_t* positions;    // [axes][tokens]
  int64_t tokens, pitch, out_pitch;
  int32_t d, pairs;
  int32_t groups;              // of a head: pairs / W, then (d - 2 pairs) / (2W), rounded up, that only copy
  int32_t lanes, rows;         // threads side by side on a head; heads that the block takes at a time
  int32_t per_block;           // tokens of a block
  int32_t back;
  FastDiv div_heads, div_lanes, div_pairs;
  gl_rotary plan;
};

// W values of type T as raw words.
template <int BYTES> struct Raw;
template <> struct Raw<16> { typedef uint4 type; };
template <> struct Raw<8> { typedef uint2 type; };
template <> struct Raw<4> { typedef uint32_t type; };
template <> struct Raw<2> { typedef uint16_t type; };

template <bool F32, int W>
__device__ __forceinline__ void to_floats(const typename Raw<W * (F32 ? 4 : 2)>::type& raw, float (&v)[W]) {
  if constexpr (F32) {
    const float* f = reinterpret_cast<const float*>(&raw);
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = f[i];
  } else if constexpr (W == 1) {
    v[0] = bf16_to_f32(raw);
  } else {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(&raw);
#pragma unroll
    for (int i = 0; i < W / 2; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
  }
}
template <bool F32, int W>
__device__ __forceinline__ typename Raw<W * (F32 ? 4 : 2)>::type from_floats(const float (&v)[W]) {
  typename Raw<W * (F32 ? 4 : 2)>::type raw;
  if constexpr (F32) {
    float* f = reinterpret_cast<float*>(&raw);
#pragma unroll
    for (int i = 0; i < W; ++i) f[i] = v[i];
  } else if constexpr (W == 1) {
    raw = f32_to_bf16(v[0]);
  } else {
    uint32_t* w = reinterpret_cast<uint32_t*>(&raw);
#pragma unroll
    for (int i = 0; i < W / 2; ++i) w[i] = pack_bf16x2(__float_as_uint(v[2 * i]), __float_as_uint(v[2 * i + 1]));
  }
  return raw;
}

// N pairs (u, v) turned by N consecutive angles, two at a time.
template <int N>
__device__ __forceinline__ void turn(float (&u)[N], float (&v)[N], const float* c, const float* s) {
  float cs[N], sn[N];
  if constexpr (N % 4 == 0) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      *reinterpret_cast<float4*>(cs + i) = *reinterpret_cast<const float4*>(c + i);
      *reinterpret_cast<float4*>(sn + i) = *reinterpret_cast<const float4*>(s + i);
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) { cs[i] = c[i]; sn[i] = s[i]; }
  }
  if constexpr (N % 2 == 0) {
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      const float2 a = make_float2(u[i], u[i + 1]), b = make_float2(v[i], v[i + 1]), cc = make_float2(cs[i], cs[i + 1]), ss = make_float2(sn[i], sn[i + 1]);
      const float2 x = sub2(mul2(a, cc), mul2(b, ss)), y = fma2(a, ss, mul2(b, cc));
      u[i] = x.x; u[i + 1] = x.y;
      v[i] = y.x; v[i + 1] = y.y;
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float a = u[i], b = v[i];
      u[i] = a * cs[i] - b * sn[i];
      v[i] = a * sn[i] + b * cs[i];
    }
  }
}

template <bool F32, int W>
__global__ void __launch_bounds__(kRotThreads) rotate_pairs(const __grid_constant__ RotateParams p) {
  typedef typename Raw<W * (F32 ? 4 : 2)>::type Word;
  extern __shared__ __align__(16) float trig[];   // cosines [tokens][pairs], then sines
  constexpr int kEs = F32 ? 4 : 2;
  const int64_t token0 = static_cast<int64_t>(blockIdx.x) * p.per_block;
  const int tokens = static_cast<int>(min(static_cast<int64_t>(p.per_block), p.tokens - token0));
  const uint32_t rows = static_cast<uint32_t>(tokens) * p.div_heads.d;   // heads of all of the block's tokens
  const char* in = static_cast<const char*>(p.x) + token0 * p.pitch * kEs;
  char* out = static_cast<char*>(p.out) + token0 * p.out_pitch * kEs;
  float* sines = trig + p.per_block * p.pairs;
  // Neighbouring lanes ask for different pairs: through the cache of data, not that of constants, which serves one address at a
  // time (8192 tokens of one head of 64 pairs: 11.5 -> 5.4 us).
  const gl_rotary* plan = &p.plan;
  asm volatile("" : "+l"(plan));
  uint32_t first_row, lane;
  p.div_lanes.divmod(threadIdx.x, first_row, lane);
  if (first_row >= static_cast<uint32_t>(p.rows)) first_row = rows;      // a thread too many
  pdl_wait();
  pdl_launch_dependents();
  bool angles = false;
  const int turned = p.pairs / W;
  for (int g0 = 0; g0 < p.groups; g0 += p.lanes) {
    const int g = g0 + static_cast<int>(lane);
    // the group's two times W values inside a head
    const bool turns = g < turned;
    const int one = turns ? (p.plan.adjacent ? 2 * W * g : W * g) : 2 * (p.pairs + (g - turned) * W);
    const int two = one + (turns && !p.plan.adjacent ? p.pairs : W);
    const bool has_one = g < p.groups, has_two = has_one && two < p.d;
    for (uint32_t r0 = 0; r0 < rows; r0 += kRotRows * p.rows) {
      Word a[kRotRows], b[kRotRows];
#pragma unroll
      for (int j = 0; j < kRotRows; ++j) {
        const uint32_t r = first_row + r0 + j * p.rows;
        if (r >= rows) break;
        uint32_t token, head;
        p.div_heads.divmod(r, token, head);
        const char* src = in + (static_cast<int64_t>(token) * p.pitch + static_cast<int>(head) * p.d) * kEs;
        if (has_one) a[j] = __ldcs(reinterpret_cast<const Word*>(src + one * kEs));
        if (has_two) b[j] = __ldcs(reinterpret_cast<const Word*>(src + two * kEs));
      }
      if (!angles) {
        angles = true;
        for (int i = threadIdx.x; i < tokens * p.pairs; i += kRotThreads) {
          uint32_t token, pair;
          p.div_pairs.divmod(static_cast<uint32_t>(i), token, pair);
          const int64_t at = p.positions[plan->axis[pair] * p.tokens + token0 + token];
          const int64_t phase = static_cast<int64_t>(plan->step[pair] * static_cast<uint64_t>(at));
          float s, c;
          sincospif(__ll2float_rn(phase) * 0x1p-63f, &s, &c);   // a signed fraction of half a turn
          trig[i] = c;
          sines[i] = p.back ? -s : s;
        }
        __syncthreads();
      }
#pragma unroll
      for (int j = 0; j < kRotRows; ++j) {
        const uint32_t r = first_row + r0 + j * p.rows;
        if (r >= rows) break;
        uint32_t token, head;
        p.div_heads.divmod(r, token, head);
        if (turns) {
          float u[W], v[W];
          to_floats<F32, W>(a[j], u);
          to_floats<F32, W>(b[j], v);
          const int at = static_cast<int>(token) * p.pairs + g * W;
          if (W > 1 && p.plan.adjacent) {
            // (u, v) are 2W values in a row: pairs (0, 1), (2, 3), ..
            float x[W], y[W];
#pragma unroll
            for (int i = 0; i < W; ++i) {
              x[i] = 2 * i < W ? u[2 * i & (W - 1)] : v[2 * i & (W - 1)];
              y[i] = 2 * i < W ? u[(2 * i + 1) & (W - 1)] : v[(2 * i + 1) & (W - 1)];
            }
            turn<W>(x, y, trig + at, sines + at);
#pragma unroll
            for (int i = 0; i < W; ++i) {
              (2 * i < W ? u : v)[2 * i & (W - 1)] = x[i];
              (2 * i < W ? u : v)[(2 * i + 1) & (W - 1)] = y[i];
            }
          } else {
            turn<W>(u, v, trig + at, sines + at);
          }
          a[j] = from_floats<F32, W>(u);
          b[j] = from_floats<F32, W>(v);
        }
        char* dst = out + (static_cast<int64_t>(token) * p.out_pitch + static_cast<int>(head) * p.d) * kEs;
        if (has_one) __stcs(reinterpret_cast<Word*>(dst + one * kEs), a[j]);
        if (has_two) __stcs(reinterpret_cast<Word*>(dst + two * kEs), b[j]);
      }
    }
  }
}

// Whether a token of the operand, `width` elements at i * pitch, and one of the result, at `from` + j * out_pitch, share an element; n
// tokens each.  Views of one projection may lie in each other's gaps (queries turned into where keys were).
bool tokens_meet(int64_t from, int64_t n, int64_t pitch, int64_t out_pitch, int64_t width) {
  typedef __int128 wide;
  const wide end = static_cast<wide>(n - 1) * pitch + width;          // of the operand
  if (from >= end || from + static_cast<wide>(n - 1) * out_pitch + width <= 0) return false;
  // the result's first token that ends behind the operand's beginning; the element before that end, counted in operand's tokens, is
  // less than two widths into one if and only if the two tokens meet
  const int64_t first = from + width > 0 ? 0 : -(from + width) / out_pitch + 1;
  const int64_t period = pitch / std::gcd(pitch, out_pitch);          // (tokens of the result after which the remainders repeat)
  for (int64_t j = first; j < n && j < first + period; ++j) {
    const wide last = from + static_cast<wide>(j) * out_pitch + width - 1;
    if (last - width + 1 >= end) return false;
    if (static_cast<int64_t>(last % pitch) < 2 * width - 1) return true;
  }
  return false;
}

// The whole number v, modulo 2^64.
uint64_t modulo64(long double v) { return v < 0 ? static_cast<uint64_t>(static_cast<int64_t>(v)) : static_cast<uint64_t>(v); }

// 2^64 f / (2 pi) to the nearest whole number, modulo 2^64.  The quotient is taken to twice a long double's 64 bits, as its whole
// turns would take the place of the bits that count; 2 pi = turn + rest.
uint64_t step_of(long double f) {
  if (f < 0) return 0 - step_of(-f);                            // (a fraction below one keeps its last bits, one above minus one does not)
  const long double turn = 6.283185307179586476925286766559005768L, rest = -1.00331152253366640471146541606615140276673e-19L;
  long double first = f / turn;
  long double second = (std::fma(-first, turn, f) - first * rest) / turn;
  first -= std::floor(first);                                   // whole turns per position change nothing
  if (std::abs(second) >= 0.25L) second -= std::floor(second);  // (of frequencies beyond 2^60)
  first *= 18446744073709551616.0L;
  second *= 18446744073709551616.0L;
  const long double a = std::floor(first), b = std::floor(second);
  return modulo64(a) + modulo64(b) + modulo64(std::floor((first - a) + (second - b) + 0.5L));
}

template <bool F32>
void (*rotate_kernel(int w))(RotateParams) {
  switch (w) {
    case 8: if constexpr (!F32) return rotate_pairs<F32, 8>;   // (16 bytes at most; fp32 asks for four)
    case 4: return rotate_pairs<F32, 4>;
    case 2: return rotate_pairs<F32, 2>;
    default: return rotate_pairs<F32, 1>;
  }
}

}  // namespace

extern "C" {

int gl_rotary_plan(int32_t pairs, double base, const double* freq, const int32_t* sections, int32_t axes, int32_t adjacent,
                   gl_rotary* out) {
  if (!out) return GL_ERR_NULL;
  if (pairs < 1 || pairs > GL_MAX_PAIRS || axes < 1 || axes > pairs) return GL_ERR_SHAPE;
  if (adjacent != 0 && adjacent != 1) return GL_ERR_SHAPE;
  if (!freq && !(base >= 1.0 && base <= 1e30)) return GL_ERR_SHAPE;
  if (!sections && axes != 1) return GL_ERR_NULL;
  if (sections) {
    int64_t n = 0;
    for (int i = 0; i < axes; ++i) {
      if (sections[i] < 0) return GL_ERR_SHAPE;
      n += sections[i];
    }
    if (n != pairs) return GL_ERR_SHAPE;
  }
  if (freq)
    for (int i = 0; i < pairs; ++i)
      if (!std::isfinite(freq[i])) return GL_ERR_SHAPE;
  std::memset(out, 0, sizeof(*out));
  out->pairs = pairs;
  out->axes = axes;
  out->adjacent = adjacent;
  int axis = 0, left = sections ? sections[0] : pairs;
  for (int i = 0; i < pairs; ++i) {
    while (left == 0) left = sections[++axis];
    out->axis[i] = static_cast<uint8_t>(axis);
    --left;
    out->step[i] = step_of(freq ? static_cast<long double>(freq[i])
                                : std::pow(static_cast<long double>(base), -static_cast<long double>(i) / pairs));
  }
  return GL_OK;
}

int gl_compute_rotate(const gl_ap* x, int64_t token_pitch, const gl_rotary* plan, const int32_t* positions, gl_ap* out,
                      int64_t out_pitch, uint32_t flags, void* stream) {
  int rc = check_data(x);
  if (rc) return rc;
  rc = check_data(out);
  if (rc) return rc;
  if (!plan || !positions) return GL_ERR_NULL;
  if (flags & ~GL_ROTATE_BACK) return GL_ERR_UNSUPPORTED;
  if (x->ndim != 4 || x->access_ndim != 3) return GL_ERR_NDIM;
  rc = check_same_meta(*x, out);
  if (rc) return rc;
  if (reinterpret_cast<uintptr_t>(positions) & 3u) return GL_ERR_ALIGN;
  if (plan->pairs < 1 || plan->pairs > GL_MAX_PAIRS || plan->axes < 1 || plan->axes > plan->pairs) return GL_ERR_SHAPE;
  if (plan->adjacent != 0 && plan->adjacent != 1) return GL_ERR_SHAPE;
  for (int i = 0; i < plan->pairs; ++i)
    if (plan->axis[i] >= plan->axes) return GL_ERR_SHAPE;
  const int64_t b = x->shape[0], t = x->shape[1], heads = x->shape[2], d = x->shape[3];
  if (2 * plan->pairs > d) return GL_ERR_SHAPE;
  if (b > (int64_t{1} << 31) / t || heads > (int64_t{1} << 24) / d) return GL_ERR_UNSUPPORTED;
  if (token_pitch == 0) token_pitch = heads * d;
  if (out_pitch == 0) out_pitch = heads * d;
  if (token_pitch < heads * d || out_pitch < heads * d) return GL_ERR_SHAPE;
  if (token_pitch > (int64_t{1} << 40) || out_pitch > (int64_t{1} << 40)) return GL_ERR_UNSUPPORTED;
  if (out->data == x->data && out_pitch != token_pitch) return GL_ERR_SHAPE;   // in place is the same view
  const int64_t apart = (reinterpret_cast<intptr_t>(out->data) - reinterpret_cast<intptr_t>(x->data)) / (x->dtype == GL_F32 ? 4 : 2);
  if (out->data != x->data && tokens_meet(apart, b * t, token_pitch, out_pitch, heads * d)) return GL_ERR_UNSUPPORTED;
  RotateParams p;
  std::memset(&p, 0, sizeof(p));
  p.x = x->data;
  p.out = out->data;
  p.positions = positions;
  p.tokens = b * t;
  p.pitch = token_pitch;
  p.out_pitch = out_pitch;
  p.d = static_cast<int32_t>(d);
  p.pairs = plan->pairs;
  p.back = (flags & GL_ROTATE_BACK) ? 1 : 0;
  p.plan = *plan;
  // the widest groups, up to 16 bytes, of which heads, pairs and distances between tokens are whole numbers
  const bool f32 = x->dtype == GL_F32;
  int w = f32 ? 4 : 8;
  while (w > 1 && (p.pairs % w || d % w || token_pitch % w || out_pitch % w)) w /= 2;
  const int64_t copied = d - 2 * p.pairs;
  p.groups = static_cast<int32_t>(p.pairs / w + (out->data == x->data ? 0 : (copied + 2 * w - 1) / (2 * w)));
  p.lanes = std::min(p.groups, kRotThreads);
  p.rows = kRotThreads / p.lanes;
  // tokens of a block: as many heads as its threads hold in flight, and no more angles than a few a thread; fewer while there
  // are SMs without a block
  int64_t per_block = std::min<int64_t>(static_cast<int64_t>(kRotRows) * p.rows / heads, kRotAngles / p.pairs);
  per_block = std::min(per_block, p.tokens / (2 * num_sms()));
  p.per_block = static_cast<int32_t>(std::max<int64_t>(per_block, 1));
  p.div_heads.set(heads);
  p.div_lanes.set(p.lanes);
  p.div_pairs.set(p.pairs);
  const int64_t blocks = (p.tokens + p.per_block - 1) / p.per_block;
  if (blocks > INT32_MAX) return GL_ERR_UNSUPPORTED;
  const size_t smem = static_cast<size_t>(2) * p.per_block * p.pairs * sizeof(float);
  void (*k)(RotateParams) = f32 ? rotate_kernel<true>(w) : rotate_kernel<false>(w);
  return launch_pdl(k, dim3(static_cast<unsigned>(blocks)), dim3(kRotThreads), smem, static_cast<cudaStream_t>(stream), 1, p) ==
                 cudaSuccess ? GL_OK : GL_ERR_CUDA;
}

}  // extern "C"
