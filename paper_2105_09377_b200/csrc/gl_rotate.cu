// compute rotate: rotary positions with several axes.  Pairs of a head's values are turned by the angle
// position[axis of the pair] * frequency of the pair.
#include <cuda_runtime.h>

#include <cmath>
#include <cstring>

#include "gl_internal.h"
#include "gl_launch.cuh"
#include "gl_tc.cuh"
#include "gl_tmap.h"

using namespace gl;

namespace {

// Angles are 64-bit fractions of a turn: step (2^64 times the turns per position) times position, modulo 2^64.  Whole turns fall
// out of the integer product by themselves and the rest is exact to position * 2^-65 turns, where an fp32 product of position and
// frequency is off by a sixteenth of a radian at a million tokens.
//
// A block takes a few tokens: cosines and sines of its tokens once into shared memory, then its threads take tasks of W pairs of
// a head, 2W values, all of a round requested before the first is used (the first round's before the angles are computed).
constexpr int kRotThreads = 256;
constexpr int kRotTasks = 4;          // tasks of a thread in flight
constexpr int kRotMaxTokens = 16;     // tokens of a block

struct RotateParams {
  const void* x;
  void* out;
  const int32_t* positions;    // [axes][tokens]
  int64_t tokens, pitch, out_pitch;
  int32_t heads, d, pairs;
  int32_t per_head;            // tasks of a head: pairs / W, then (d - 2 pairs) / (2W), rounded up, that only copy
  int32_t per_block;           // tokens of a block
  int32_t back;
  FastDiv div_head, div_token; // tasks of a head; tasks of a token
  FastDiv div_pairs;
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
  } else {
    const uint16_t* h = reinterpret_cast<const uint16_t*>(&raw);
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = bf16_to_f32(h[i]);
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

struct TaskAt {
  int64_t in, out;    // element of the token's start
  int first, second;  // elements of the two groups of W values inside the token; second < 0: there is none
  int angle;          // index of the first pair's cosine, < 0: values to copy
  bool live;
};

template <int W>
__device__ __forceinline__ TaskAt task_at(const RotateParams& p, uint32_t task, uint32_t tasks, int64_t token0) {
  TaskAt t;
  t.live = task < tasks;
  uint32_t token, in_token, head, i;
  p.div_token.divmod(t.live ? task : 0u, token, in_token);
  p.div_head.divmod(in_token, head, i);
  t.in = (token0 + token) * p.pitch;
  t.out = (token0 + token) * p.out_pitch;
  const int base = static_cast<int>(head) * p.d, turned = p.pairs / W;
  if (static_cast<int>(i) < turned) {
    const int pair = static_cast<int>(i) * W;
    t.first = base + (p.plan.adjacent ? 2 * pair : pair);
    t.second = t.first + (p.plan.adjacent ? W : p.pairs);
    t.angle = static_cast<int>(token) * p.pairs + pair;
  } else {
    const int at = 2 * p.pairs + (static_cast<int>(i) - turned) * 2 * W;
    t.first = base + at;
    t.second = at + W < p.d ? t.first + W : -1;
    t.angle = -1;
  }
  return t;
}

template <bool F32, int W>
__global__ void __launch_bounds__(kRotThreads) rotate_pairs(const __grid_constant__ RotateParams p) {
  typedef typename Raw<W * (F32 ? 4 : 2)>::type Word;
  extern __shared__ float trig[];   // cosines [tokens][pairs], then sines
  constexpr int kEs = F32 ? 4 : 2;
  const int64_t token0 = static_cast<int64_t>(blockIdx.x) * p.per_block;
  const int tokens = static_cast<int>(min(static_cast<int64_t>(p.per_block), p.tokens - token0));
  const uint32_t tasks = static_cast<uint32_t>(tokens) * p.div_token.d;
  const char* in = static_cast<const char*>(p.x);
  char* out = static_cast<char*>(p.out);
  float* sines = trig + p.per_block * p.pairs;
  pdl_wait();
  pdl_launch_dependents();
  for (uint32_t round = 0; round < tasks; round += kRotThreads * kRotTasks) {
    Word a[kRotTasks], b[kRotTasks];
#pragma unroll
    for (int j = 0; j < kRotTasks; ++j) {
      const TaskAt t = task_at<W>(p, round + j * kRotThreads + threadIdx.x, tasks, token0);
      if (t.live) {
        a[j] = *reinterpret_cast<const Word*>(in + (t.in + t.first) * kEs);
        if (t.second >= 0) b[j] = *reinterpret_cast<const Word*>(in + (t.in + t.second) * kEs);
      }
    }
    if (round == 0) {
      for (int i = threadIdx.x; i < tokens * p.pairs; i += kRotThreads) {
        uint32_t token, pair;
        p.div_pairs.divmod(static_cast<uint32_t>(i), token, pair);
        const int64_t at = p.positions[p.plan.axis[pair] * p.tokens + token0 + token];
        const int64_t phase = static_cast<int64_t>(p.plan.step[pair] * static_cast<uint64_t>(at));
        float s, c;
        sincospif(__ll2float_rn(phase) * 0x1p-63f, &s, &c);   // a signed fraction of half a turn
        trig[i] = c;
        sines[i] = p.back ? -s : s;
      }
      __syncthreads();
    }
#pragma unroll
    for (int j = 0; j < kRotTasks; ++j) {
      const TaskAt t = task_at<W>(p, round + j * kRotThreads + threadIdx.x, tasks, token0);
      if (!t.live) continue;
      if (t.angle >= 0) {
        float u[W], v[W];
        to_floats<F32, W>(a[j], u);
        to_floats<F32, W>(b[j], v);
        if (p.plan.adjacent && W > 1) {
          // pairs (0,1), (2,3), ... of the 2W values in u, v
#pragma unroll
          for (int i = 0; i < W; i += 2) {
            const int pu = t.angle + i / 2, pv = pu + W / 2;
            const float cu = trig[pu], su = sines[pu], cv = trig[pv], sv = sines[pv];
            const float u0 = u[i], u1 = u[i + 1 < W ? i + 1 : i], v0 = v[i], v1 = v[i + 1 < W ? i + 1 : i];
            u[i] = u0 * cu - u1 * su;
            u[i + 1 < W ? i + 1 : i] = u0 * su + u1 * cu;
            v[i] = v0 * cv - v1 * sv;
            v[i + 1 < W ? i + 1 : i] = v0 * sv + v1 * cv;
          }
        } else {
#pragma unroll
          for (int i = 0; i < W; ++i) {
            const float c = trig[t.angle + i], s = sines[t.angle + i];
            const float x0 = u[i], x1 = v[i];
            u[i] = x0 * c - x1 * s;
            v[i] = x0 * s + x1 * c;
          }
        }
        a[j] = from_floats<F32, W>(u);
        b[j] = from_floats<F32, W>(v);
      }
      *reinterpret_cast<Word*>(out + (t.out + t.first) * kEs) = a[j];
      if (t.second >= 0) *reinterpret_cast<Word*>(out + (t.out + t.second) * kEs) = b[j];
    }
  }
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
  const long double turn = 6.283185307179586476925286766559005768L;
  int axis = 0, left = sections ? sections[0] : pairs;
  for (int i = 0; i < pairs; ++i) {
    while (left == 0) left = sections[++axis];
    out->axis[i] = static_cast<uint8_t>(axis);
    --left;
    const long double f = freq ? static_cast<long double>(freq[i])
                               : std::pow(static_cast<long double>(base), -static_cast<long double>(i) / pairs);
    long double part = f / turn;
    part -= std::floor(part);                                  // whole turns per position change nothing
    const long double scaled = std::floor(part * 18446744073709551616.0L + 0.5L);
    out->step[i] = scaled >= 18446744073709551616.0L ? 0 : static_cast<uint64_t>(scaled);
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
  RotateParams p;
  std::memset(&p, 0, sizeof(p));
  p.x = x->data;
  p.out = out->data;
  p.positions = positions;
  p.tokens = b * t;
  p.pitch = token_pitch;
  p.out_pitch = out_pitch;
  p.heads = static_cast<int32_t>(heads);
  p.d = static_cast<int32_t>(d);
  p.pairs = plan->pairs;
  p.back = (flags & GL_ROTATE_BACK) ? 1 : 0;
  p.plan = *plan;
  // the widest groups, up to 16 bytes, of which heads, pairs and distances between tokens are whole numbers
  const bool f32 = x->dtype == GL_F32;
  int w = f32 ? 4 : 8;
  while (w > 1 && (p.pairs % w || d % w || token_pitch % w || out_pitch % w)) w /= 2;
  const int64_t copied = d - 2 * p.pairs;
  p.per_head = static_cast<int32_t>(p.pairs / w + (out->data == x->data ? 0 : (copied + 2 * w - 1) / (2 * w)));
  const int64_t per_token = heads * p.per_head;
  // tokens of a block: a round of tasks for its threads
  p.per_block = 1;
  while (p.per_block * 2 <= kRotMaxTokens && p.per_block * 2 * per_token <= kRotThreads * kRotTasks) p.per_block *= 2;
  while (p.per_block > 1 && (p.tokens + p.per_block - 1) / p.per_block < 2 * num_sms()) p.per_block /= 2;
  p.div_head.set(p.per_head);
  p.div_token.set(per_token);
  p.div_pairs.set(p.pairs);
  const int64_t blocks = (p.tokens + p.per_block - 1) / p.per_block;
  if (blocks > INT32_MAX) return GL_ERR_UNSUPPORTED;
  const size_t smem = static_cast<size_t>(2) * p.per_block * p.pairs * sizeof(float);
  void (*k)(RotateParams) = f32 ? rotate_kernel<true>(w) : rotate_kernel<false>(w);
  return launch_pdl(k, dim3(static_cast<unsigned>(blocks)), dim3(kRotThreads), smem, static_cast<cudaStream_t>(stream), 1, p) ==
                 cudaSuccess ? GL_OK : GL_ERR_CUDA;
}

}  // extern "C"
