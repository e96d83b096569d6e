// Pages of 4-bit keys and values (gl_cache4) and the attention that reads them.
// The order of a page's bytes and where a token lies: gl_cache4.cuh.
#include <cuda.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cstring>
#include <type_traits>

#include "gl_cache4.cuh"
#include "gl_internal.h"
#include "gl_launch.cuh"
#include "gl_mx4.cuh"
#include "gl_tc.cuh"
#include "gl_tmap.h"

using namespace gl;

namespace {

// ------------------------------------------------------------------------
// Storing and reading back
// ------------------------------------------------------------------------

// Eight dims of K and of V of one token and head per item.  Neighbouring threads have neighbouring items: D / 8 of them
// (8, 16 or 32, inside a warp) share a token and head.  U items per thread, 256 apart, are requested before the first is
// used.  What bounds both kernels are the instructions that find an item's place: K and V share them (apart, 14 us each
// way for 8192 tokens of 8 heads of 128).

// Scale exponent and codes of a thread's eight values, four neighbouring threads a block.  (Every thread of the warp.)
__device__ __forceinline__ void quantize8(const uint4& raw, uint32_t& e, uint32_t& word) {
  const uint32_t in[4] = {raw.x, raw.y, raw.z, raw.w};
  float x[8];
  uint32_t two = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(in[i] << 16);
    x[2 * i + 1] = __uint_as_float(in[i] & 0xFFFF0000u);
    two = __vmaxu2(two, in[i] & 0x7FFF7FFFu);
  }
  uint32_t top = max(two << 16, two & 0xFFFF0000u);
  top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
  top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
  e = mx4_exponent(top);
  word = mx4_codes8(x, e);
}
// Words of the lanes of blocks b & ~1 and b | 1, same j: their low halves, or their high ones.
__device__ __forceinline__ uint32_t halves_of_pair(uint32_t word, bool high) {
  const int even = static_cast<int>(threadIdx.x & 31u) & ~4;
  const uint32_t w0 = __shfl_sync(0xFFFFFFFFu, word, even), w1 = __shfl_sync(0xFFFFFFFFu, word, even | 4);
  return __byte_perm(w0, w1, high ? 0x7632 : 0x5410);
}

template <int U>
__global__ void __launch_bounds__(256) cache4_append(const uint16_t* __restrict__ k, const uint16_t* __restrict__ v,
                                                     const TokensParams p) {
  pdl_wait();
  pdl_launch_dependents();
  TokenAt at[U];
  uint4 raw_k[U], raw_v[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t item = (blockIdx.x * U + u) * 256u + threadIdx.x;
    at[u] = token_at(p, item);
    // (does not wait for the page: a token that is not stored is read all the same)
    raw_k[u] = raw_v[u] = make_uint4(0, 0, 0, 0);
    if (item < p.items) {
      raw_k[u] = __ldcs(reinterpret_cast<const uint4*>(k + at[u].dense));
      raw_v[u] = __ldcs(reinterpret_cast<const uint4*>(v + at[u].dense));
    }
  }
  const int NB = p.D / 32;
#pragma unroll
  for (int u = 0; u < U; ++u) {   // (every thread goes through the shuffles)
    uint32_t ek, ev, wk, wv;
    quantize8(raw_k[u], ek, wk);
    quantize8(raw_v[u], ev, wv);
    const int b = at[u].w >> 2, j = at[u].w & 3, tok = at[u].tok;
    wv = halves_of_pair(wv, b & 1);
    uint8_t* group = at[u].group;
    if (group) {
      const int codes = tok * (p.D / 2), scales = tok * NB + b;
      *reinterpret_cast<uint32_t*>(group + codes + (j * NB + b) * 4) = wk;
      *reinterpret_cast<uint32_t*>(group + v_codes_at(p.D) + codes + v_offset(NB, b, j, tok)) = wv;
      if (j == 0) {
        group[k_scales_at(p.D) + scales] = static_cast<uint8_t>(ek);
        group[v_scales_at(p.D) + scales] = static_cast<uint8_t>(ev);
      }
    }
  }
}

template <int U>
__global__ void __launch_bounds__(256) cache4_read(uint16_t* __restrict__ k, uint16_t* __restrict__ v, const TokensParams p) {
  pdl_wait();
  pdl_launch_dependents();
  const int NB = p.D / 32;
  TokenAt at[U];
  uint32_t wk[U], wv[U], ek[U], ev[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    at[u] = token_at(p, (blockIdx.x * U + u) * 256u + threadIdx.x);
    wk[u] = wv[u] = ek[u] = ev[u] = 0;
    if (at[u].group) {
      const int b = at[u].w >> 2, j = at[u].w & 3, tok = at[u].tok, codes = tok * (p.D / 2), scales = tok * NB + b;
      wk[u] = *reinterpret_cast<const uint32_t*>(at[u].group + codes + (j * NB + b) * 4);
      wv[u] = *reinterpret_cast<const uint32_t*>(at[u].group + v_codes_at(p.D) + codes + v_offset(NB, b, j, tok));
      ek[u] = at[u].group[k_scales_at(p.D) + scales];
      ev[u] = at[u].group[v_scales_at(p.D) + scales];
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    // of V, dims 8 j .. + 3 come from the lane of the even block, + 4 .. + 7 from that of the odd one
    wv[u] = halves_of_pair(wv[u], at[u].w & 4);
    if ((blockIdx.x * U + u) * 256u + threadIdx.x < p.items) {
      uint32_t w[4];
      mx4_words_bf16(wk[u], ek[u], w);
      __stcs(reinterpret_cast<uint4*>(k + at[u].dense), make_uint4(w[0], w[1], w[2], w[3]));
      mx4_words_bf16(wv[u], ev[u], w);
      __stcs(reinterpret_cast<uint4*>(v + at[u].dense), make_uint4(w[0], w[1], w[2], w[3]));
    }
  }
}

// ------------------------------------------------------------------------
// Attention
// ------------------------------------------------------------------------
//
// out = sum_t p_t V_t / sum_t p_t, p_t = 2^((s_t - roof) cf), s = q K_t, cf = scale log2(e), in one pass over the tokens with a
// running reference `roof`, 8 / cf above the largest score that it was set by.  The reference is held in units of the scores
// and subtracted before the product with cf: of scores beyond 2^24 / cf the rounded product roof cf would be off by more than
// the largest weight can bear (from 2^31 on all weights became 0 or Inf).
//
// Rows are the T * group query rows that share a kv head, 8 * NT of them per work item; scores are computed transposed,
// S^T = K Q^T with tokens as the 16-row side of mma.m16n8k16, so that eight rows (a usual group) fill an instruction.
// Codes become fp16 by the conversion instruction (exact).  The scale of a block of K multiplies the fp32 result of that
// block's two instructions, so no scale ever meets fp16's range.  Q is scaled per row by a power of two for the same reason;
// the scales of K get 2^-24 for it, or keys beyond 2^100 would leave fp32's range although the scores do not.  (Scales of K
// below 2^-109 become zeros by it.)
// Of V, a token's scale varies along the result, so it goes into the weights: w = 2^15 p * 2^(e - top), top the largest
// exponent that the block has met (and one more); the sums refer to it.  Tokens more than seven binades below it take
// a turn of their own.  fp16 weights keep 11 bits, which a bf16 result cannot show; for fp32 results (HILO) the rounded-off
// part of the weights is multiplied in a second instruction.  The reference moves only when a weight would pass 2^15: then
// the largest one becomes 2^7.
//
// The work is cut along the tokens of all sequences: tiles of 64 (32) tokens of all (sequence, kv head, row block) in one
// list, the same number to every block.  A block's four warps take turns in the tiles of a segment, each with its own
// ring of bulk copies, running reference, sum and result; the block joins its warps, and a second kernel joins the
// blocks where a segment was cut.  A part is stored divided by its own sum of weights and joined as an average, so that
// nothing is larger than the values themselves (weights of up to 2^15 over many tokens took values beyond 2^100 to Inf).
//
// 64 sequences of 4096 tokens, 32 heads over 8 of 128: 75 us, 3.8 TB/s of cache (0.58 of the copy rate), bound by issue: about
// 610 instructions per 32 tokens and warp, of which 128 convert codes and 32 are matrix instructions, at 0.55 instructions
// per cycle and scheduler.  Four blocks per SM (128 registers) instead of three: 95 us.  fp32 results 82 us.
// 32 rows per kv head (NT = 4, 255 registers, some spilled): 32 sequences of 4096 tokens, 64 heads over 8, 4 tokens each:
// 106 us, fp32 results 134 us.  256-wide heads, 16 rows (NT = 2, some spilled), 32 sequences: 114 us and 161 us; 8 rows 76 and
// 80 us.

constexpr int kSubTok = 32;       // tokens that a warp computes with at a time
constexpr int kWarps = 4;

struct AttendParams {
  CacheView c;
  const uint16_t* q;
  void* out;
  float* part;           // partial results: per block two slots of rows * (D + 2) floats: reference, sum of weights, averages
  int64_t q_pitch;
  int T, heads, group;   // group = heads / kv_heads
  int rows, row_blocks;  // rows = T * group
  int R, tile_log2;      // rows per row block, tokens per tile (a power of two)
  FastDiv div_group;
  int grid;
  int min_share;         // list entries that a block takes at least
  int lead;              // what a segment costs beyond its tiles, in tiles (see Walk)
  int alone;             // a block per segment, no list, nothing to join: caches of a few tiles
  float scale_log2;      // softmax scale * log2(e)
  float step;            // 8 / scale_log2
  int out_bf16;
};

// Tokens that the rows of row block rb can see at most, and the tiles that hold them.
__device__ __forceinline__ int seen_by(const AttendParams& p, int len, int rb) {
  const int last = min(p.rows, (rb + 1) * p.R) - 1;
  return min(max(len - p.T + static_cast<int>(p.div_group.div(static_cast<uint32_t>(last))) + 1, 0), len);
}
__device__ __forceinline__ int seen_tiles(const AttendParams& p, int len, int rb) {
  return (seen_by(p, len, rb) + (1 << p.tile_log2) - 1) >> p.tile_log2;
}

// Entries of the work list for a row block and for one kv head of sequence b: its tiles, with `lead` empty entries before
// them that stand for what every segment costs (fragments of Q, filling the ring, joining the warps).  Without them a
// block that meets many short sequences gets as many tiles as the others and ends last.  One token per sequence, us with none,
// 4, 8, 16 and 32 empty entries:
//   16 sequences of 17 .. 16384 tokens, 128 wide: 79, 54, 46, 47, 50;  64 wide: 53, 38, 32, 33, 35;  256 wide: 142, 91, 86, 79, 81
//   64 sequences of 100 .. 2000 tokens:           57, 39, 35, 36, 37;           41, 29, 27, 27, 28;            126, 95, 81, 71, 71
//   32 sequences of 4096 tokens:                  47, 45, 46, 49, 54;           33, 32, 33, 35, 38;            77, 77, 76, 77, 78
// (so 8, and 16 for 256-wide heads).  attend_many has one; none would cost 3 to 25 % (two prompts of 512 tokens behind 5001 and
// 8192: 181 us against 174), two or four would gain on ragged prompts (168 and 164 us).
__device__ __forceinline__ int seen_entries(const AttendParams& p, int len, int rb) {
  const int n = seen_tiles(p, len, rb);
  return n ? n + p.lead : 0;
}
__device__ __forceinline__ int64_t head_entries(const AttendParams& p, int b) {
  const int len = clamped_length(p.c, b);
  int64_t n = 0;
  for (int rb = 0; rb < p.row_blocks; ++rb) n += seen_entries(p, len, rb);
  return n;
}

// Sum of head_entries over the sequences before `upto` and over all of them, by the whole block.
template <int THREADS>
__device__ __forceinline__ void sum_entries(const AttendParams& p, int upto, int64_t* before, int64_t* all, int64_t* scratch) {
  int64_t a = 0, b = 0;
  for (int i = threadIdx.x; i < p.c.batch; i += THREADS) {
    const int64_t n = head_entries(p, i);
    a += n;
    if (i < upto) b += n;
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    a += __shfl_xor_sync(0xFFFFFFFFu, a, o);
    b += __shfl_xor_sync(0xFFFFFFFFu, b, o);
  }
  if ((threadIdx.x & 31) == 0) {
    scratch[2 * (threadIdx.x >> 5)] = a;
    scratch[2 * (threadIdx.x >> 5) + 1] = b;
  }
  __syncthreads();
  a = b = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 32; ++w) { a += scratch[2 * w]; b += scratch[2 * w + 1]; }
  *all = a * p.c.kv_heads;
  *before = b * p.c.kv_heads;
}

// Entries per block: an even share, but no less than min_share.
__device__ __forceinline__ int64_t block_share(const AttendParams& p, int64_t all) {
  const int64_t n = (all + p.grid - 1) / p.grid;
  return n < p.min_share ? p.min_share : n;
}

// A block's way through its part of the list: one (sequence, kv head, row block) after the other, tiles t0 .. t1 of the
// n_seg that it has.
struct Walk {
  int64_t at, end, seg0, per_head;
  int b, h, rb, t0, t1, n_seg, len, seen;

  // Finds the block's part, by the whole block (scratch: 2 * THREADS / 32 + 4 words): the sequences' tiles are counted by a
  // thread each and scanned.  (One thread that walks along 64 sequences takes 3 us.)
  template <int THREADS>
  __device__ __forceinline__ void start(const AttendParams& p, int block, int64_t* scratch) {
    if (p.alone) {
      rb = block % p.row_blocks;
      h = block / p.row_blocks;
      b = h / p.c.kv_heads;
      h -= b * p.c.kv_heads;
      len = clamped_length(p.c, b);
      seen = seen_by(p, len, rb);
      t0 = 0;
      t1 = n_seg = seen_tiles(p, len, rb);
      at = 0;
      end = n_seg ? 1 : 0;
      __syncthreads();
      return;
    }
    int64_t all, before;
    sum_entries<THREADS>(p, 0, &before, &all, scratch);
    const int64_t share = block_share(p, all);
    at = block * share;
    end = min(all, at + share);
    b = 0;
    seg0 = per_head = 0;
    if (at >= end) return;   // (block-uniform)
    int64_t* found = scratch + 2 * (THREADS / 32);
    int64_t done = 0;        // tiles of the sequences before this round
    for (int first = 0; first < p.c.batch; first += THREADS) {
      const int i = first + static_cast<int>(threadIdx.x), lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
      const int64_t heads = i < p.c.batch ? head_entries(p, i) : 0, mine = heads * p.c.kv_heads;
      int64_t upto = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int64_t x = __shfl_up_sync(0xFFFFFFFFu, upto, o);
        if (lane >= o) upto += x;
      }
      __syncthreads();
      if (lane == 31) scratch[warp] = upto;
      __syncthreads();
      int64_t total = 0, off = 0;
#pragma unroll
      for (int w = 0; w < THREADS / 32; ++w) {
        if (w < warp) off += scratch[w];
        total += scratch[w];
      }
      const int64_t from = done + off + upto - mine;
      if (from <= at && at < from + mine) { found[0] = i; found[1] = from; found[2] = heads; }
      done += total;
      if (done > at) break;
    }
    __syncthreads();
    b = static_cast<int>(found[0]);
    seg0 = found[1];
    per_head = found[2];
  }
  __device__ __forceinline__ bool next(const AttendParams& p) {
    if (p.alone) return at++ < end;
    while (at < end) {
      while (seg0 + per_head * p.c.kv_heads <= at) {
        if (b + 1 >= p.c.batch) return false;   // (only if lengths changed under the kernel)
        seg0 += per_head * p.c.kv_heads;
        per_head = head_entries(p, ++b);
      }
      len = clamped_length(p.c, b);
      h = static_cast<int>((at - seg0) / per_head);
      int64_t s0 = seg0 + h * per_head;
      int n = 0;
      for (rb = 0;; ++rb) {
        n = seen_entries(p, len, rb);
        if (s0 + n > at || rb + 1 == p.row_blocks) break;
        s0 += n;
      }
      const int64_t stop = min(end, s0 + n);
      if (stop <= at) return false;             // (the same)
      n_seg = n - p.lead;
      t0 = max(static_cast<int>(at - s0) - p.lead, 0);
      t1 = static_cast<int>(stop - s0) - p.lead;
      seen = seen_by(p, len, rb);
      at = stop;
      if (t1 > t0) return true;
    }
    return false;
  }
  __device__ __forceinline__ bool whole() const { return t0 == 0 && t1 == n_seg; }
  // where this block's part of a segment that it does not have to itself goes: it is the block's last or its first
  __device__ __forceinline__ float* slot(const AttendParams& p, int D) const {
    return p.part + (static_cast<int64_t>(blockIdx.x) * 2 + (t0 == 0 ? 1 : 0)) * p.R * (D + 2);
  }
};

// Token of a query row, and element 0 of the row's result and of the row itself.
__device__ __forceinline__ int row_token(const AttendParams& p, int row) {
  return static_cast<int>(p.div_group.div(static_cast<uint32_t>(row)));
}
__device__ __forceinline__ int64_t out_row(const AttendParams& p, int b, int h, int row, int D) {
  const int t = row_token(p, row);
  return ((static_cast<int64_t>(b) * p.T + t) * p.heads + static_cast<int64_t>(h) * p.group + row - t * p.group) * D;
}
__device__ __forceinline__ const uint16_t* q_row(const AttendParams& p, int b, int h, int row, int D) {
  const int t = row_token(p, row);
  return p.q + (static_cast<int64_t>(b) * p.T + t) * p.q_pitch + (static_cast<int64_t>(h) * p.group + row - t * p.group) * D;
}

// Zeros for a segment without a tile, by its own block (blocks that share a list leave that to the joining kernel).
template <int THREADS>
__device__ __forceinline__ void store_empty(const AttendParams& p, const Walk& w, int D) {
  if (!p.alone || w.n_seg) return;
  const int rows = min(p.rows - w.rb * p.R, p.R);
  for (int e = threadIdx.x; e < rows * (D / 4); e += THREADS) {
    const int r = e / (D / 4), d = e % (D / 4) * 4;
    const int64_t to = out_row(p, w.b, w.h, w.rb * p.R + r, D) + d;
    if (p.out_bf16) *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.out) + to) = make_uint2(0, 0);
    else *reinterpret_cast<float4*>(static_cast<float*>(p.out) + to) = make_float4(0.f, 0.f, 0.f, 0.f);
  }
}

__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(v));
  return d;
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}
// What brings sums that refer to the exact ref cf to its rounded value, which is what the joining goes by.  (Beyond 2^24 that
// says no more than which part is ahead.)
__device__ __forceinline__ float rounded_off(float ref, float cf) {
  const float rest = fmaf(ref, cf, -(ref * cf));
  return fabsf(rest) < 1.f ? ex2(rest) : 1.f;
}
// lo += low half, hi += high half
__device__ __forceinline__ void add_halves_f16(uint32_t two, float& lo, float& hi) {
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tadd.f32.f16 %0, l, %0;\n\tadd.f32.f16 %1, h, %1;\n\t}"
      : "+f"(lo), "+f"(hi) : "r"(two));
}
// Token (0..15) of the group that row i of a 16-row fragment stands for: spreads the tokens that a warp reads in one
// access over the banks.  Rows come in pairs (2i, 2i+1) -> (i, 4 + (i ^ 1)), the upper eight likewise.
__device__ __forceinline__ int token_of_row(int i) {
  const int j = i & 7;
  return (i & 8) + ((j & 1) ? 4 + ((j >> 1) ^ 1) : (j >> 1));
}

__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// The codes of a word's bytes as fp16 pairs (low code, high code): one conversion instruction a byte, 1.2 cycles of an SM
// per word of a warp; moving the bits with shifts and masks takes 3.6.
__device__ __forceinline__ void mx4_bytes_f16(uint32_t w, uint32_t (&h)[4]) {
  asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
      "mov.b32 {b0, b1, b2, b3}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, b0;\n\t"
      "cvt.rn.f16x2.e2m1x2 %1, b1;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, b2;\n\t"
      "cvt.rn.f16x2.e2m1x2 %3, b3;\n\t}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(w));
}
// N consecutive words, or half words, or scale bytes of a token (shared-memory addresses)
template <int N>
__device__ __forceinline__ void load_shared(uint32_t at, uint32_t (&w)[N]) {
  static_assert(N == 1 || N == 2 || N % 4 == 0, "1, 2 or whole 16 bytes");
  if constexpr (N == 1) {
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w[0]) : "r"(at));
  } else if constexpr (N == 2) {
    asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(at));
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 4)
      asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                   : "=r"(w[i]), "=r"(w[i + 1]), "=r"(w[i + 2]), "=r"(w[i + 3]) : "r"(at + 4 * i));
  }
}
template <int NB>
__device__ __forceinline__ void load_words(uint32_t at, uint32_t (&w)[NB]) { load_shared<NB>(at, w); }
template <int NB>
__device__ __forceinline__ void load_halves(uint32_t at, uint32_t (&w)[NB / 2]) { load_shared<NB / 2>(at, w); }
template <int NB>
__device__ __forceinline__ void load_scales(uint32_t at, uint32_t (&w)[(NB + 3) / 4]) {
  if constexpr (NB == 2) {
    uint16_t x;
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(x) : "r"(at));
    w[0] = x;
  } else {
    load_shared<NB / 4>(at, w);
  }
}
// Scale bytes of K as 2^(e - 127 - 24), NaN for 255: two a conversion, by way of bf16
template <int NB>
__device__ __forceinline__ void scale_floats(const uint32_t (&w)[(NB + 3) / 4], float (&f)[NB]) {
#pragma unroll
  for (int i = 0; i < NB; i += 2) {
    uint32_t two;
    const uint16_t bytes = static_cast<uint16_t>(w[i >> 2] >> (8 * (i & 2)));
    asm("cvt.rn.bf16x2.ue8m0x2 %0, %1;" : "=r"(two) : "h"(bytes));
    two = mul_bf16x2(two, 0x33803380u);
    f[i] = __uint_as_float(two << 16);
    f[i + 1] = __uint_as_float(two & 0xFFFF0000u);
  }
}
// Byte i of two words as the high bytes of two halves, zeros below (the bytes' top bits are clear: their sign is zeros)
__device__ __forceinline__ uint32_t high_bytes(uint32_t a, uint32_t b, int i) {
  uint32_t d;
  asm("prmt.b32 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"((8u | i) | i << 4 | (8u | (4u + i)) << 8 | (4u + i) << 12));
  return d;
}
// V of two neighbouring blocks as 16-row operands: x0..x3 hold dims 4 g .. + 3 of both blocks (low and high half) of the
// tokens in columns 2 tq, 2 tq + 1, 2 tq + 8, 2 tq + 9.  Bytes with one token's code in each half become fp16 pairs.
__device__ __forceinline__ void v_operands(uint32_t x0, uint32_t x1, uint32_t x2, uint32_t x3, uint32_t (&va)[2][2][4]) {
  uint32_t e0[4], o0[4], e1[4], o1[4];   // even and odd dims of both blocks: (block 0: 0 1, block 1: 2 3)
  mx4_bytes_f16((x0 & 0x0F0F0F0Fu) | ((x1 << 4) & 0xF0F0F0F0u), e0);
  mx4_bytes_f16(((x0 >> 4) & 0x0F0F0F0Fu) | (x1 & 0xF0F0F0F0u), o0);
  mx4_bytes_f16((x2 & 0x0F0F0F0Fu) | ((x3 << 4) & 0xF0F0F0F0u), e1);
  mx4_bytes_f16(((x2 >> 4) & 0x0F0F0F0Fu) | (x3 & 0xF0F0F0F0u), o1);
#pragma unroll
  for (int hb = 0; hb < 2; ++hb)
#pragma unroll
    for (int k = 0; k < 2; ++k) {   // instruction k: row g = dim 2 k, row g + 8 = dim 2 k + 1
      va[hb][k][0] = e0[2 * hb + k];
      va[hb][k][1] = o0[2 * hb + k];
      va[hb][k][2] = e1[2 * hb + k];
      va[hb][k][3] = o1[2 * hb + k];
    }
}

template <int NB, int NT>
struct AttCfg {
  static constexpr int D = 32 * NB;
  static constexpr int R = 8 * NT;
  // Tokens per tile (what a warp waits for and asks for at a time) and tiles in a warp's ring: 64 and 2, but 32 and 3 for
  // 256-wide heads, whose rings would leave room for one block per SM (32 x 4096 tokens: 96 us, 77 us with two blocks).
  static constexpr int kTileTok = NB == 8 ? 32 : 64;
  static constexpr int kStagesAt = NB == 8 ? 3 : 2;
  static constexpr int kStage = kTileTok / kGroup * group_bytes(D);  // one tile
  static constexpr int kRing = kWarps * kStagesAt * kStage;
  static constexpr int kQ = NB * 2 * NT * 32 * 8;                    // fragments of Q
  // results of a warp, in the place of its ring: rows of D floats, then maxima and sums.  Rows are kept apart by their
  // order in the banks (a pitch of D + 4 floats) where the ring has the room.
  static constexpr int kWarpRing = kStagesAt * kStage;
  static constexpr int kAccPitch = R * (D + 6) * 4 <= kWarpRing ? D + 4 : D;
  static constexpr int kSmem = kRing + kQ + R * 4 + 2 * kWarps * R * 4 + 256;
  static_assert(R * kAccPitch * 4 <= kWarpRing, "results fit in the ring");
};

template <int NB, int NT, bool HILO>
__global__ void __launch_bounds__(kWarps * 32) attend_cache4(const AttendParams p) {
  using Cfg = AttCfg<NB, NT>;
  constexpr int D = Cfg::D, R = Cfg::R, kTileTok = Cfg::kTileTok, kStagesAt = Cfg::kStagesAt;
  extern __shared__ __align__(128) unsigned char smem[];
  uint2* qfrag = reinterpret_cast<uint2*>(smem + Cfg::kRing);
  float* qfac = reinterpret_cast<float*>(smem + Cfg::kRing + Cfg::kQ);
  float* jm = qfac + R;             // [kWarps][R] references and sums of the warps
  float* jl = jm + kWarps * R;
  unsigned char* tail = smem + Cfg::kRing + Cfg::kQ + R * 4 + 2 * kWarps * R * 4;
  uint64_t* bars = reinterpret_cast<uint64_t*>(tail);                          // [kWarps][kStagesAt]
  int64_t* scratch = reinterpret_cast<int64_t*>(tail + 8 * kWarps * kStagesAt);   // [2 * kWarps + 4]
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tail + 8 * kWarps * kStagesAt + 16 * kWarps + 32);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, tq = lane & 3;

  if (threadIdx.x == 0) {
    for (int i = 0; i < kWarps * kStagesAt; ++i) mbar_init(smem_u32(bars + i), 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  pdl_wait();
  pdl_launch_dependents();
  Walk w;
  w.start<kWarps * 32>(p, blockIdx.x, scratch);   // (its barriers also publish the ones set up above)
  store_empty<kWarps * 32>(p, w, D);

  const uint32_t my_ring = smem_u32(smem) + warp * kStagesAt * Cfg::kStage;
  const uint32_t my_bar = smem_u32(bars + warp * kStagesAt);
  uint32_t slot_in = 0, slot_out = 0, phase_out = 0;
  constexpr int kScaleWords = (NB + 3) / 4;
  const float ninf = __uint_as_float(0xFF800000u);
  bool ok = true;

  while (w.next(p)) {
    const int b = w.b, h = w.h, rb = w.rb, t0 = w.t0, t1 = w.t1, len = w.len, seen = w.seen;

    // ---- ring of this warp: tiles t0 + warp, + kWarps, ...
    // The previous segment's fragments and joined results (which lie in the rings) are read.  A block that gave up ends here:
    // it cannot use a barrier again whose copies are still out.
    if (__syncthreads_or(!ok)) break;
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    constexpr int kGroupsAt = kTileTok / kGroup;
    constexpr uint32_t kAllThere = (1u << kGroupsAt) - 1u;
    uint32_t there = 0;   // kGroupsAt bits per tile in flight: its groups that have a page (oldest tile lowest)
    int in_flight = 0;
    int next = t0 + warp;
    int32_t page = -1;    // lane g < kGroupsAt: page of group g of tile `next`, -1 where there is none
    auto fetch_pages = [&]() {
      const int pos = next * kTileTok + lane * kGroup;
      page = -1;
      if (next < t1 && lane < kGroupsAt && pos < seen)
        page = p.c.table[static_cast<int64_t>(b) * p.c.width + p.c.div_page.div(static_cast<uint32_t>(pos))];
    };
    auto issue = [&]() {   // copies of tile `next`: lane g asks for group g
      if (next >= t1) return;
      const bool mine = page >= 0 && page < p.c.pages;
      const uint32_t have = __ballot_sync(0xFFFFFFFFu, mine);
      const uint32_t bar = my_bar + 8 * slot_in;
      if (lane == 0) mbar_expect_tx(bar, __popc(have) * group_bytes(D));
      __syncwarp();
      if (mine) {
        uint32_t slot, in_page;
        p.c.div_page.divmod(static_cast<uint32_t>(next * kTileTok + lane * kGroup), slot, in_page);
        bulk_copy_g2s(my_ring + slot_in * Cfg::kStage + lane * group_bytes(D),
                      p.c.data + page * p.c.page_stride + h * p.c.head_stride + static_cast<int64_t>(in_page / kGroup) * group_bytes(D),
                      group_bytes(D), bar);
      }
      there |= have << (kGroupsAt * in_flight);
      ++in_flight;
      slot_in = slot_in + 1 == kStagesAt ? 0 : slot_in + 1;
      next += kWarps;
      fetch_pages();
    };
    fetch_pages();
#pragma unroll
    for (int i = 0; i < kStagesAt; ++i) issue();

    // ---- Q as fragments in shared memory, row r scaled by a power of two into [2^14, 2^15)
    for (int r = warp; r < R; r += kWarps) {
      const int row = rb * R + r;
      const bool live = row < p.rows;
      const uint16_t* src = nullptr;
      if (live) src = q_row(p, b, h, row, D);
      float x[NB];
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        x[i] = live ? bf16_to_f32(src[i * 32 + lane]) : 0.f;
        top = max(top, __float_as_uint(x[i]) & 0x7FFFFFFFu);
      }
      top = __reduce_max_sync(0xFFFFFFFFu, top);
      const int e = max(static_cast<int>(top >> 23), 27) - 127;                 // floor(log2) of the largest, not below -100
      const float f = __uint_as_float(static_cast<uint32_t>(14 - e + 127 > 0 ? 14 - e + 127 : 0) << 23);
      // lane = dim % 32: word j = lane / 8, byte (lane / 2) % 4 of the word; byte 2i + s is register s of instruction i
      const int j = lane >> 3, byte = (lane >> 1) & 3, half = lane & 1;
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        __half* dst = reinterpret_cast<__half*>(qfrag + ((i * 2 + (byte >> 1)) * NT + (r >> 3)) * 32 + (r & 7) * 4 + j);
        dst[(byte & 1) * 2 + half] = __float2half_rn(x[i] * f);
      }
      // scores carry the 2^(14 - e) of Q and the 2^-24 of K (queries beyond 2^117 may need more than fp32 has)
      if (lane == 0)
        qfac[r] = fminf(__uint_as_float(static_cast<uint32_t>(min(e + 127 - 14 + 24, 254)) << 23) * p.scale_log2, 1.7014118e38f);
    }
    __syncthreads();
    // roof: what a row's weights refer to; a weight is 2^15 p = 2^((s - roof) cf + 15), roof -Inf until there is one.
    // top_e: the scale exponents that the blocks' results refer to, four to a word, 8 at least.
    float roof[NT][2], l[NT][2], cf[NT][2];
    int limit[NT][2], all_see = INT32_MAX, any_sees = 0;
    uint32_t top_e[kScaleWords];
    float acc[NT][NB][2][4];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int row = rb * R + n * 8 + tq * 2 + c;
        roof[n][c] = ninf;
        l[n][c] = 0.f;
        cf[n][c] = qfac[n * 8 + tq * 2 + c];
        limit[n][c] = row < p.rows ? min(len, len - p.T + row_token(p, row) + 1) : seen;   // (rows past the end: anything)
        all_see = min(all_see, limit[n][c]);
        any_sees = max(any_sees, limit[n][c]);
      }
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[n][i][0][c] = acc[n][i][1][c] = 0.f;
    }
    all_see = __reduce_min_sync(0xFFFFFFFFu, all_see);
    any_sees = __reduce_max_sync(0xFFFFFFFFu, any_sees);
#pragma unroll
    for (int i = 0; i < kScaleWords; ++i) top_e[i] = NB == 2 ? 0x0808u : 0x08080808u;
    // where this lane's tokens start in a group: K rows g and (8 tokens on) g + 8; V columns 2 tq, 2 tq + 1 and 8 tokens on
    const uint32_t tok_k = token_of_row(g), tok_v0 = token_of_row(2 * tq), tok_v1 = token_of_row(2 * tq + 1);
    const uint32_t at_k = tok_k * (D / 2) + tq * (NB * 4), at_ks = k_scales_at(D) + tok_k * NB;
    const uint32_t at_v0 = v_codes_at(D) + tok_v0 * (D / 2) + (g ^ ((tok_v0 & 2) ? 4 : 0)) * NB * 2;
    const uint32_t at_v1 = v_codes_at(D) + tok_v1 * (D / 2) + (g ^ ((tok_v1 & 2) ? 4 : 0)) * NB * 2;
    const uint32_t at_vs0 = v_scales_at(D) + tok_v0 * NB, at_vs1 = v_scales_at(D) + tok_v1 * NB;

    for (int tile = t0 + warp; tile < t1; tile += kWarps) {
      if (!mbar_wait(my_bar + 8 * slot_out, phase_out, abort_flag)) { ok = false; break; }
      const uint32_t tile_have = there & kAllThere;
#pragma unroll 1
      for (int sub = 0; sub < kTileTok / kSubTok; ++sub) {
      const uint32_t st = my_ring + slot_out * Cfg::kStage + sub * 2 * group_bytes(D);
      const uint32_t have = tile_have >> (2 * sub) & 3u;
      const int pos0 = tile * kTileTok + sub * kSubTok;
      if (pos0 >= any_sees) break;
      const bool masked = have != 3u || pos0 + kSubTok > all_see;

      // ---- scores: s[mt][n] = 16 tokens x 8 rows; thread: tokens of rows g and g + 8, query rows 2 tq and 2 tq + 1
      float s[2][NT][4];
      {
        uint32_t wa[2][NB], wb[2][NB];
        float fa[2][NB], fb[2][NB];
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
          const uint32_t grp = st + mt * group_bytes(D);
          load_words<NB>(grp + at_k, wa[mt]);
          load_words<NB>(grp + at_k + 8 * (D / 2), wb[mt]);
          uint32_t sa[kScaleWords], sb[kScaleWords];
          load_scales<NB>(grp + at_ks, sa);
          load_scales<NB>(grp + at_ks + 8 * NB, sb);
          scale_floats<NB>(sa, fa[mt]);
          scale_floats<NB>(sb, fb[mt]);
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int c = 0; c < 4; ++c) s[mt][n][c] = 0.f;
        }
#pragma unroll
        for (int i = 0; i < NB; ++i) {
          uint32_t a[2][2][4];
#pragma unroll
          for (int mt = 0; mt < 2; ++mt) {
            uint32_t ha[4], hb[4];
            mx4_bytes_f16(wa[mt][i], ha);
            mx4_bytes_f16(wb[mt][i], hb);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              a[mt][k][0] = ha[2 * k]; a[mt][k][1] = hb[2 * k]; a[mt][k][2] = ha[2 * k + 1]; a[mt][k][3] = hb[2 * k + 1];
            }
          }
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            const uint2 b0 = qfrag[((i * 2) * NT + n) * 32 + lane], b1 = qfrag[((i * 2 + 1) * NT + n) * 32 + lane];
#pragma unroll
            for (int mt = 0; mt < 2; ++mt) {
              float c[4] = {0.f, 0.f, 0.f, 0.f};
              mma_f16(c, a[mt][0], b0.x, b0.y);
              mma_f16(c, a[mt][1], b1.x, b1.y);
              s[mt][n][0] = fmaf(c[0], fa[mt][i], s[mt][n][0]);
              s[mt][n][1] = fmaf(c[1], fa[mt][i], s[mt][n][1]);
              s[mt][n][2] = fmaf(c[2], fb[mt][i], s[mt][n][2]);
              s[mt][n][3] = fmaf(c[3], fb[mt][i], s[mt][n][3]);
            }
          }
        }
      }
      if (masked) {   // what lies behind the end or on a missing page is never looked at
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              const int pos = pos0 + mt * kGroup + static_cast<int>(tok_k) + 8 * (c >> 1);
              if (!(pos < limit[n][c & 1] && (have >> mt & 1u))) s[mt][n][c] = ninf;
            }
      }

      // ---- the reference moves only when a weight would pass 2^15: a vote, no shuffles, in most tiles
      bool above = false;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
          for (int c = 0; c < 4; ++c) above |= s[mt][n][c] > roof[n][c & 1];
      if (__any_sync(0xFFFFFFFFu, above)) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float top = fmaxf(fmaxf(s[0][n][c], s[0][n][2 + c]), fmaxf(s[1][n][c], s[1][n][2 + c]));
            top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 4));
            top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 8));
            top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 16));
            // (a step of 2^120 stands for more: all scores are the same to such a cf)
            const float now = fmaxf(roof[n][c], top + fminf(__fdividef(8.f, cf[n][c]), 1.329228e36f));
            // (roof = -Inf, nothing seen so far: sum and result are zeros)
            const float f = now == roof[n][c] ? 1.f : ex2((roof[n][c] - now) * cf[n][c]);
            roof[n][c] = now;
            l[n][c] *= f;
#pragma unroll
            for (int i = 0; i < NB; ++i)
#pragma unroll
              for (int k = 0; k < 2; ++k) { acc[n][i][k][c] *= f; acc[n][i][k][2 + c] *= f; }
          }
      }
      // weights, and as the 8-column operand: register hf holds rows 8 hf + 2 tq and + 1 of the 16 tokens, query row g
      uint32_t wh[2][NT][2], wl[2][NT][2];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const float w15 = ex2(fmaf(s[mt][n][c] - roof[n][c & 1], cf[n][c & 1], 15.f));
            s[mt][n][c] = masked && s[mt][n][c] == ninf ? 0.f : w15;
            if (HILO) l[n][c & 1] += s[mt][n][c];
          }
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            const float x = s[mt][n][2 * hf], y = s[mt][n][2 * hf + 1];
            const uint32_t packed = pack_f16x2(x, y);
            wh[mt][n][hf] = transpose8x8(packed);
            if (!HILO) add_halves_f16(packed, l[n][0], l[n][1]);   // (the sum is that of the weights as they are used)
            if (HILO) {
              const __half2 r = *reinterpret_cast<const __half2*>(&packed);
              wl[mt][n][hf] = transpose8x8(pack_f16x2(x - __low2float(r), y - __high2float(r)));
            }
          }
        }

      // ---- result: acc += V^T w.  Thread: dims 4 g .. + 3 of every block for the tokens of rows 2 tq, 2 tq + 1 and
      // those 8 further on, k = 0..3
      uint32_t vw[2][4][NB / 2], vs[2][4][kScaleWords];
#pragma unroll
      for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t grp = st + mt * group_bytes(D) + (k >> 1) * 8 * (D / 2);
          load_halves<NB>(grp + (k & 1 ? at_v1 : at_v0), vw[mt][k]);
          load_scales<NB>(st + mt * group_bytes(D) + (k >> 1) * 8 * NB + (k & 1 ? at_vs1 : at_vs0), vs[mt][k]);
        }
      // Distance of every scale from its block's reference, byte by byte: 0..7 all over is the plain case.  (References are 8 at
      // least: no distance that is none of these looks like one after the borrow.)
      uint32_t fs[2][4][kScaleWords];   // high bytes of fp16 2^-d
      const auto plain = [&]() {
        uint32_t far = 0;
#pragma unroll
        for (int k2 = 0; k2 < kScaleWords; ++k2)
#pragma unroll
          for (int mt = 0; mt < 2; ++mt)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const uint32_t d = top_e[k2] - vs[mt][k][k2];
              far |= d & 0xF8F8F8F8u;
              fs[mt][k][k2] = 0x3C3C3C3Cu - 4u * d;
            }
        return !__any_sync(0xFFFFFFFFu, far != 0);
      };
      // Brings block i's reference up to `top`, one binade more than needed so that the next larger scale finds room.
      const auto raise = [&](int i, uint32_t top) {
        const uint32_t base = top_e[i >> 2] >> (8 * (i & 3)) & 255u;
        if (top <= base) return base;
        top = min(top + 1u, 254u);
        const float f = top - base > 126u ? 0.f : __uint_as_float((127u - (top - base)) << 23);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int c = 0; c < 4; ++c) { acc[n][i][0][c] *= f; acc[n][i][1][c] *= f; }
        top_e[i >> 2] += (top - base) << (8 * (i & 3));
        return top;
      };
      bool easy = !masked && plain();
      if (!easy && !masked) {
#pragma unroll
        for (int i = 0; i < NB; ++i) {
          uint32_t top = 0;
#pragma unroll
          for (int mt = 0; mt < 2; ++mt)
#pragma unroll
            for (int k = 0; k < 4; ++k) top = max(top, vs[mt][k][i >> 2] >> (8 * (i & 3)) & 255u);
          top = __reduce_max_sync(0xFFFFFFFFu, top);
          if (top < 255u) raise(i, top);
        }
        easy = plain();
      }
      if (easy) {
#pragma unroll
        for (int w2 = 0; w2 < NB / 2; ++w2) {
#pragma unroll
          for (int mt = 0; mt < 2; ++mt) {
            uint32_t va[2][2][4];   // [block of the pair][instruction][register]
            v_operands(vw[mt][0][w2], vw[mt][1][w2], vw[mt][2][w2], vw[mt][3][w2], va);
#pragma unroll
            for (int hb = 0; hb < 2; ++hb) {
              const int i = 2 * w2 + hb;
              const uint32_t f0 = high_bytes(fs[mt][0][i >> 2], fs[mt][1][i >> 2], i & 3);
              const uint32_t f1 = high_bytes(fs[mt][2][i >> 2], fs[mt][3][i >> 2], i & 3);
#pragma unroll
              for (int n = 0; n < NT; ++n) {
                const uint32_t b0 = mul_f16x2(wh[mt][n][0], f0), b1 = mul_f16x2(wh[mt][n][1], f1);
                mma_f16(acc[n][i][0], va[hb][0], b0, b1);
                mma_f16(acc[n][i][1], va[hb][1], b0, b1);
                if (HILO) {
                  const uint32_t c0 = mul_f16x2(wl[mt][n][0], f0), c1 = mul_f16x2(wl[mt][n][1], f1);
                  mma_f16(acc[n][i][0], va[hb][0], c0, c1);
                  mma_f16(acc[n][i][1], va[hb][1], c0, c1);
                }
              }
            }
          }
        }
      } else {
        // The end of a sequence, missing pages, NaN, or scales far apart: per block, the tokens within seven binades of the
        // largest scale left, then the next ones.
#pragma unroll
        for (int i = 0; i < NB; ++i) {
          uint32_t ex[2][4];   // 256: not seen, or done
          uint32_t top = 0, nan_here = 0;
#pragma unroll
          for (int mt = 0; mt < 2; ++mt)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const int tok = static_cast<int>(k & 1 ? tok_v1 : tok_v0) + 8 * (k >> 1);
              uint32_t e = vs[mt][k][i >> 2] >> (8 * (i & 3)) & 255u;
              if (!(have >> mt & 1u) || pos0 + mt * kGroup + tok >= any_sees) e = 256u;
              if (e == 255u) { nan_here |= 1u << (4 * mt + k); e = 256u; }
              ex[mt][k] = e;
              if (e < 255u) top = max(top, e);
            }
          top = __reduce_max_sync(0xFFFFFFFFu, top);
          const uint32_t base = raise(i, top);
          bool more;
          do {
            uint32_t f2[2][2];
            uint32_t rest = 0;
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
              for (int hf = 0; hf < 2; ++hf) {
                f2[mt][hf] = 0;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                  uint32_t& e = ex[mt][2 * hf + k];
                  if (e <= top && e + 7u >= top) {
                    f2[mt][hf] |= (15u - (top - e)) << (10 + 16 * k);
                    e = 256u;
                  }
                  // (e = 0 next to a larger scale: zeros, or values below 2^-124, which are left out here)
                  if (e < 255u) rest = max(rest, e);
                }
              }
            rest = __reduce_max_sync(0xFFFFFFFFu, rest);
            more = rest > 0u;
            const uint32_t below = base - top;
            const float f = below > 126u ? 0.f : __uint_as_float((127u - below) << 23);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              float c0[4] = {0.f, 0.f, 0.f, 0.f}, c1[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
              for (int mt = 0; mt < 2; ++mt) {
                uint32_t va[2][2][4];
                v_operands(vw[mt][0][i >> 1], vw[mt][1][i >> 1], vw[mt][2][i >> 1], vw[mt][3][i >> 1], va);
                const uint32_t b0 = mul_f16x2(wh[mt][n][0], f2[mt][0]), b1 = mul_f16x2(wh[mt][n][1], f2[mt][1]);
                mma_f16(c0, va[i & 1][0], b0, b1);
                mma_f16(c1, va[i & 1][1], b0, b1);
                if (HILO) {
                  const uint32_t d0 = mul_f16x2(wl[mt][n][0], f2[mt][0]), d1 = mul_f16x2(wl[mt][n][1], f2[mt][1]);
                  mma_f16(c0, va[i & 1][0], d0, d1);
                  mma_f16(c1, va[i & 1][1], d0, d1);
                }
              }
#pragma unroll
              for (int c = 0; c < 4; ++c) {
                acc[n][i][0][c] = fmaf(c0[c], f, acc[n][i][0][c]);
                acc[n][i][1][c] = fmaf(c1[c], f, acc[n][i][1][c]);
              }
            }
            top = rest;
          } while (more);
          if (__any_sync(0xFFFFFFFFu, nan_here != 0)) {   // NaN for the rows that see such a token, and for no others
            int from = INT32_MAX;
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
              for (int k = 0; k < 4; ++k)
                if (nan_here >> (4 * mt + k) & 1u)
                  from = min(from, pos0 + mt * kGroup + static_cast<int>(k & 1 ? tok_v1 : tok_v0) + 8 * (k >> 1));
            from = __reduce_min_sync(0xFFFFFFFFu, from);
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
              for (int c = 0; c < 2; ++c)
                if (from < limit[n][c])
#pragma unroll
                  for (int k = 0; k < 2; ++k) acc[n][i][k][c] = acc[n][i][k][2 + c] = __uint_as_float(0x7FC00000u);
          }
        }
      }
      }   // (sub)
      __syncwarp();   // every lane has read the stage
      there >>= kGroupsAt;
      --in_flight;
      if (++slot_out == kStagesAt) { slot_out = 0; phase_out ^= 1u; }
      issue();
    }

    // ---- join the warps
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        l[n][c] += __shfl_xor_sync(0xFFFFFFFFu, l[n][c], 4);
        l[n][c] += __shfl_xor_sync(0xFFFFFFFFu, l[n][c], 8);
        l[n][c] += __shfl_xor_sync(0xFFFFFFFFu, l[n][c], 16);
      }
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int r = n * 8 + tq * 2 + c;
        if (g == 0) {
          jm[warp * R + r] = roof[n][c] * cf[n][c];
          jl[warp * R + r] = l[n][c] * rounded_off(roof[n][c], cf[n][c]);
        }
        const float inv = l[n][c] == 0.f ? 0.f : __fdividef(1.f, l[n][c]);
        float* row = reinterpret_cast<float*>(smem + warp * Cfg::kWarpRing) + r * Cfg::kAccPitch;
#pragma unroll
        for (int i = 0; i < NB; ++i) {
          const float back = mx4_scale(top_e[i >> 2] >> (8 * (i & 3)) & 255u);
#pragma unroll
          for (int k = 0; k < 2; ++k)
            *reinterpret_cast<float2*>(row + i * 32 + 4 * g + 2 * k) =
                make_float2(acc[n][i][k][c] * inv * back, acc[n][i][k][2 + c] * inv * back);
        }
      }
    __syncthreads();
    const bool whole = w.whole();
    float* slot = w.slot(p, D);
    for (int e = threadIdx.x; e < R * (D / 4); e += kWarps * 32) {
      const int r = e / (D / 4), d = e % (D / 4) * 4;
      const int row = rb * R + r;
      float top = jm[r];
#pragma unroll
      for (int w = 1; w < kWarps; ++w) top = fmaxf(top, jm[w * R + r]);
      const float base = top == __uint_as_float(0xFF800000u) ? 0.f : top;
      float sum = 0.f, f[kWarps];
#pragma unroll
      for (int w = 0; w < kWarps; ++w) sum += f[w] = jl[w * R + r] * ex2(jm[w * R + r] - base);
      const float inv = sum == 0.f ? 0.f : __fdividef(1.f, sum);
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float4 x = *reinterpret_cast<const float4*>(smem + w * Cfg::kWarpRing + (r * Cfg::kAccPitch + d) * 4);
        f[w] *= inv;
        o.x += x.x * f[w]; o.y += x.y * f[w]; o.z += x.z * f[w]; o.w += x.w * f[w];
      }
      if (!whole) {
        *reinterpret_cast<float2*>(slot + r * (D + 2) + d + 2) = make_float2(o.x, o.y);
        *reinterpret_cast<float2*>(slot + r * (D + 2) + d + 4) = make_float2(o.z, o.w);
        if (d == 0) *reinterpret_cast<float2*>(slot + r * (D + 2)) = make_float2(top, sum);
      } else if (row < p.rows) {
        const int64_t to = out_row(p, b, h, row, D) + d;
        if (p.out_bf16)
          *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.out) + to) =
              make_uint2(pack_bf16x2(__float_as_uint(o.x), __float_as_uint(o.y)), pack_bf16x2(__float_as_uint(o.z), __float_as_uint(o.w)));
        else
          *reinterpret_cast<float4*>(static_cast<float*>(p.out) + to) = o;
      }
    }
  }
  if (!ok || *abort_flag) {   // copies in flight land before the block leaves
    const uint64_t wait0 = global_timer();
    while (global_timer() - wait0 < 20000000ull) { }
  }
}

// Segments that several blocks share, joined in a fixed order; zeros for segments without a tile.  `wpr` warps share a row:
// each adds up every wpr-th part (lane = D / 32 neighbouring dims, four parts requested before the first is used), then
// they meet in shared memory.  Eight to a row when there are few rows in all (a long sequence has a part from every block
// of the grid: one warp that takes 296 of them by itself needs 120 us), else as few as fill a block.
constexpr int kJoinWarps = 8;

struct JoinShape { int wpr, rows_per_block; };

template <int NB>
__global__ void __launch_bounds__(32 * kJoinWarps) attend_join(const AttendParams p, const JoinShape js) {
  constexpr int D = 32 * NB;
  __shared__ int64_t scratch[2 * kJoinWarps];
  __shared__ float meet[kJoinWarps][D + 2];
  pdl_wait();
  pdl_launch_dependents();
  const int rb = static_cast<int>(blockIdx.x) % p.row_blocks, bh = static_cast<int>(blockIdx.x) / p.row_blocks;
  const int b = bh / p.c.kv_heads, h = bh % p.c.kv_heads;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int64_t all, first;
  sum_entries<32 * kJoinWarps>(p, b, &first, &all, scratch);
  const int64_t share = block_share(p, all);
  const int len = clamped_length(p.c, b);
  first += h * head_entries(p, b);
  for (int i = 0; i < rb; ++i) first += seen_entries(p, len, i);
  const int n = seen_tiles(p, len, rb);
  const int64_t c0 = (first + p.lead) / share, c1 = n ? (first + p.lead + n - 1) / share : c0;
  if (n && c0 == c1) return;   // written by the block that had all of it
  const float ninf = __uint_as_float(0xFF800000u);
  const int sub = warp % js.wpr, r0 = static_cast<int>(blockIdx.y) * js.rows_per_block;
  for (int r1 = 0; r1 < js.rows_per_block; r1 += kJoinWarps / js.wpr) {   // (block-uniform)
    if (rb * p.R + r0 + r1 >= p.rows) break;
    const int r = r0 + r1 + warp / js.wpr, row = rb * p.R + r;
    const bool live = r < r0 + js.rows_per_block && row < p.rows;
    float top = ninf, sum = 0.f, o[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i) o[i] = 0.f;
    // the average so far and K parts, each with its weight in the sum of all
    const auto add = [&](auto parts, const float2* ml, const float (*x)[NB]) {
      constexpr int K = decltype(parts)::value;
      float t = top, f[K];
#pragma unroll
      for (int k = 0; k < K; ++k) t = fmaxf(t, ml[k].x);
      const float base = t == ninf ? 0.f : t;
      float fo = sum * ex2(top - base);
      sum = fo;
#pragma unroll
      for (int k = 0; k < K; ++k) sum += f[k] = ml[k].y * ex2(ml[k].x - base);
      const float inv = sum == 0.f ? 0.f : __fdividef(1.f, sum);   // (to 1 ulp; the sums are ordinary numbers)
      fo *= inv;
#pragma unroll
      for (int k = 0; k < K; ++k) f[k] *= inv;
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        o[i] *= fo;
#pragma unroll
        for (int k = 0; k < K; ++k) o[i] = fmaf(x[k][i], f[k], o[i]);
      }
      top = t;
    };
    if (n && live) {
      for (int64_t c = c0 + sub; c <= c1; c += 4 * js.wpr) {
        float2 ml[4];
        float x[4][NB];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int64_t part = c + k * js.wpr;
          ml[k] = make_float2(ninf, 0.f);
#pragma unroll
          for (int i = 0; i < NB; ++i) x[k][i] = 0.f;
          if (part <= c1) {
            const float* slot = p.part + ((part * 2 + (part == c0 ? 1 : 0)) * p.R + r) * (D + 2);
            ml[k] = *reinterpret_cast<const float2*>(slot);
#pragma unroll
            for (int i = 0; i < NB; i += 2) {
              const float2 v = *reinterpret_cast<const float2*>(slot + 2 + lane * NB + i);
              x[k][i] = v.x;
              x[k][i + 1] = v.y;
            }
          }
        }
        add(std::integral_constant<int, 4>{}, ml, x);
      }
    }
    if (js.wpr > 1) {
      __syncthreads();   // the previous row's sums are read
      if (lane == 0) { meet[warp][D] = top; meet[warp][D + 1] = sum; }
#pragma unroll
      for (int i = 0; i < NB; ++i) meet[warp][lane * NB + i] = o[i];
      __syncthreads();
      if (sub != 0) continue;
      for (int w = warp + 1; w < warp + js.wpr; ++w) {
        float x[1][NB];
#pragma unroll
        for (int i = 0; i < NB; ++i) x[0][i] = meet[w][lane * NB + i];
        const float2 ml = make_float2(meet[w][D], meet[w][D + 1]);
        add(std::integral_constant<int, 1>{}, &ml, x);
      }
    }
    if (!live) continue;
    const int64_t to = out_row(p, b, h, row, D) + lane * NB;
#pragma unroll
    for (int i = 0; i < NB; i += 2) {
      if (p.out_bf16)
        *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(p.out) + to + i) =
            pack_bf16x2(__float_as_uint(o[i]), __float_as_uint(o[i + 1]));
      else
        *reinterpret_cast<float2*>(static_cast<float*>(p.out) + to + i) = make_float2(o[i], o[i + 1]);
    }
  }
}

}  // namespace

#include "gl_attend_many.cuh"

namespace {

// ---- host side ----

int check_cache_meta(const gl_cache4* c) {
  if (!c) return GL_ERR_NULL;
  if (c->pages < 1 || c->kv_heads < 1 || c->page_tokens < 1) return GL_ERR_SHAPE;
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return GL_ERR_UNSUPPORTED;
  if (c->page_tokens % kGroup) return GL_ERR_UNSUPPORTED;
  return GL_OK;
}

int check_cache(const gl_cache4* c, const gl_pages* at, CacheView* v) {
  const int rc = check_cache_meta(c);
  if (rc) return rc;
  if (!c->data || !at || !at->page_table || !at->lengths) return GL_ERR_NULL;
  if (reinterpret_cast<uintptr_t>(c->data) & 15u) return GL_ERR_ALIGN;
  if ((reinterpret_cast<uintptr_t>(at->page_table) | reinterpret_cast<uintptr_t>(at->lengths)) & 3u) return GL_ERR_ALIGN;
  if (at->batch < 1 || at->table_width < 1) return GL_ERR_SHAPE;
  const int64_t cap = static_cast<int64_t>(at->table_width) * c->page_tokens;
  if (cap > INT32_MAX - 4096) return GL_ERR_UNSUPPORTED;
  v->data = static_cast<uint8_t*>(c->data);
  v->table = at->page_table;
  v->lengths = at->lengths;
  v->pages = c->pages;
  v->head_stride = static_cast<int64_t>(c->page_tokens / kGroup) * group_bytes(c->head_dim);
  v->page_stride = v->head_stride * c->kv_heads;
  v->kv_heads = c->kv_heads;
  v->page_tokens = c->page_tokens;
  v->batch = at->batch;
  v->width = at->table_width;
  v->capacity = static_cast<int>(cap);
  v->div_page.set(c->page_tokens);
  return GL_OK;
}

// x is ((batch, T, heads),(head_dim)), bf16; pitch 0 stands for dense.
int check_tokens(const gl_ap* x, const gl_cache4* c, const gl_pages* at, int64_t* pitch) {
  const int rc = check_data(x);
  if (rc) return rc;
  if (x->dtype != GL_BF16) return GL_ERR_DTYPE;
  if (x->ndim != 4 || x->access_ndim != 3) return GL_ERR_NDIM;
  if (x->shape[0] != at->batch || x->shape[3] != c->head_dim) return GL_ERR_SHAPE;
  if (x->shape[1] > INT32_MAX || x->shape[2] > INT32_MAX) return GL_ERR_UNSUPPORTED;
  const int64_t dense = x->shape[2] * x->shape[3];
  if (*pitch == 0) *pitch = dense;
  if (*pitch < dense) return GL_ERR_SHAPE;
  if (*pitch % 8) return GL_ERR_ALIGN;
  return GL_OK;
}

int tokens_params(const gl_cache4* cache, const gl_ap* k, const gl_ap* v, int64_t pitch, const gl_pages* at, TokensParams* p) {
  int rc = check_cache(cache, at, &p->c);
  if (rc) return rc;
  int64_t pk = pitch, pv = pitch;
  rc = check_tokens(k, cache, at, &pk);
  if (rc) return rc;
  rc = check_tokens(v, cache, at, &pv);
  if (rc) return rc;
  if (k->shape[1] != v->shape[1] || k->shape[2] != cache->kv_heads || v->shape[2] != cache->kv_heads) return GL_ERR_SHAPE;
  const int64_t items = k->shape[0] * k->shape[1] * k->shape[2] * (cache->head_dim / 8);
  if (items > INT32_MAX - 256) return GL_ERR_UNSUPPORTED;
  p->T = static_cast<int>(k->shape[1]);
  p->D = cache->head_dim;
  p->pitch = pk;
  p->items = static_cast<uint32_t>(items);
  p->div_row.set(cache->head_dim / 8);
  p->div_heads.set(cache->kv_heads);
  p->div_T.set(p->T);
  return GL_OK;
}

// Several items per thread only when every SM has blocks to hold.
constexpr int kTokenItems = 2;
bool several_items(const TokensParams& p) { return p.items >= static_cast<uint32_t>(num_sms()) * 4u * 256u * kTokenItems; }
dim3 token_grid(const TokensParams& p, bool many) {
  const uint32_t per_block = 256u * (many ? kTokenItems : 1);
  return dim3((p.items + per_block - 1) / per_block);
}

// Which kernel runs, and its numbers.
struct AttKernel {
  void (*fn)(AttendParams);
  int smem, threads;
  int rows, tile, min_share;   // rows per work item, tokens per tile, tiles that a block takes at least
  int lead;                    // what a segment costs beyond its tiles, in tiles
  int per_sm;                  // most blocks per SM
};

template <int NB, int NT>
AttKernel few_kernel(bool hilo) {
  return {hilo ? attend_cache4<NB, NT, true> : attend_cache4<NB, NT, false>, AttCfg<NB, NT>::kSmem, kWarps * 32, 8 * NT,
          AttCfg<NB, NT>::kTileTok, kWarps, NB == 8 ? 16 : 8, 4};
}
template <int NB>
AttKernel many_kernel(bool f32) {
  if (f32) return {attend_many<NB, 3>, ManyCfg<NB, 3>::kSmem, ManyCfg<NB, 3>::kThreads, ManyCfg<NB, 3>::kRows, ManyCfg<NB, 3>::TT, 1, 1, 1};
  return {attend_many<NB, 1>, ManyCfg<NB, 1>::kSmem, ManyCfg<NB, 1>::kThreads, ManyCfg<NB, 1>::kRows, ManyCfg<NB, 1>::TT, 1, 1, 1};
}

constexpr int kAloneTiles = 4;

// Up to 32 rows that share a kv head: 8, 16 or 32 of them per warp tile (256-wide heads: 16, two items for more);
// more rows: 128 or 256 per block on tcgen05.
AttKernel pick_kernel(int64_t rows, int d, bool f32) {
  if (rows > 32) return d == 64 ? many_kernel<2>(f32) : d == 128 ? many_kernel<4>(f32) : many_kernel<8>(f32);
  const int nt = rows <= 8 ? 1 : rows <= 16 || d == 256 ? 2 : 4;
  if (d == 64) return nt == 1 ? few_kernel<2, 1>(f32) : nt == 2 ? few_kernel<2, 2>(f32) : few_kernel<2, 4>(f32);
  if (d == 128) return nt == 1 ? few_kernel<4, 1>(f32) : nt == 2 ? few_kernel<4, 2>(f32) : few_kernel<4, 4>(f32);
  return nt == 1 ? few_kernel<8, 1>(f32) : few_kernel<8, 2>(f32);
}

// Blocks of the persistent grid: what is resident at once.
int att_grid(const AttKernel& k, int d, bool f32, int* grid) {
  static std::atomic<int> cached[64][3][5][2];   // per device, 0: not asked yet (threads may ask at once: the calls are idempotent)
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return GL_ERR_CUDA;
  std::atomic<int>& known = cached[dev][d == 64 ? 0 : d == 128 ? 1 : 2][k.rows <= 8 ? 0 : k.rows <= 16 ? 1 : k.rows <= 32 ? 2 : k.rows <= 128 ? 3 : 4][f32];
  int n = known.load(std::memory_order_acquire);
  if (!n) {
    if (cudaFuncSetAttribute(k.fn, cudaFuncAttributeMaxDynamicSharedMemorySize, k.smem) != cudaSuccess) return GL_ERR_CUDA;
    int per = 0;
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per, k.fn, k.threads, k.smem) != cudaSuccess || per < 1) return GL_ERR_CUDA;
    n = std::min(per, k.per_sm) * num_sms();
    known.store(n, std::memory_order_release);
  }
  *grid = n;
  return GL_OK;
}

}  // namespace

namespace gl {
int take_status_attend() {
  unsigned int v = 0;
  if (cudaMemcpyFromSymbol(&v, g_status, sizeof(v)) != cudaSuccess) return GL_ERR_CUDA;
  if (!v) return GL_OK;
  const unsigned int zero = 0;
  if (cudaMemcpyToSymbol(g_status, &zero, sizeof(zero)) != cudaSuccess) return GL_ERR_CUDA;
  return GL_ERR_TIMEOUT;
}
}  // namespace gl

extern "C" {

size_t gl_cache4_bytes(const gl_cache4* c) {
  if (check_cache_meta(c)) return 0;
  return static_cast<size_t>(c->pages) * c->kv_heads * (c->page_tokens / kGroup) * group_bytes(c->head_dim);
}

int gl_cache4_append(const gl_cache4* cache, const gl_ap* k, const gl_ap* v, int64_t token_pitch, const gl_pages* at, void* stream) {
  TokensParams p;
  const int rc = tokens_params(cache, k, v, token_pitch, at, &p);
  if (rc) return rc;
  const bool many = several_items(p);
  return launch_pdl(many ? cache4_append<kTokenItems> : cache4_append<1>, token_grid(p, many), dim3(256), 0,
                    static_cast<cudaStream_t>(stream), 1, static_cast<const uint16_t*>(k->data),
                    static_cast<const uint16_t*>(v->data), p) == cudaSuccess ? GL_OK : GL_ERR_CUDA;
}

int gl_cache4_read(const gl_cache4* cache, const gl_pages* at, gl_ap* k, gl_ap* v, void* stream) {
  TokensParams p;
  const int rc = tokens_params(cache, k, v, 0, at, &p);
  if (rc) return rc;
  const bool many = several_items(p);
  return launch_pdl(many ? cache4_read<kTokenItems> : cache4_read<1>, token_grid(p, many), dim3(256), 0,
                    static_cast<cudaStream_t>(stream), 1, static_cast<uint16_t*>(k->data), static_cast<uint16_t*>(v->data), p) ==
                 cudaSuccess ? GL_OK : GL_ERR_CUDA;
}

size_t gl_attend_cache4_workspace(const gl_ap* q, const gl_cache4* cache) {
  if (check_meta(q) || check_cache_meta(cache) || q->ndim != 4 || q->shape[2] % cache->kv_heads) return 0;
  const int64_t rows = q->shape[1] * (q->shape[2] / cache->kv_heads);
  size_t most = 0;
  for (const bool f32 : {false, true}) {
    const AttKernel k = pick_kernel(rows, cache->head_dim, f32);
    most = std::max(most, static_cast<size_t>(k.per_sm) * num_sms() * 2 * k.rows * (cache->head_dim + 2) * sizeof(float));
  }
  return most;
}

int gl_attend_cache4(const gl_ap* q, int64_t token_pitch, const gl_cache4* cache, const gl_pages* at, float scale, gl_ap* out,
                     uint32_t flags, void* workspace, size_t workspace_bytes, void* stream) {
  AttendParams p;
  int rc = check_cache(cache, at, &p.c);
  if (rc) return rc;
  if (flags & ~GL_OUT_BF16) return GL_ERR_UNSUPPORTED;
  int64_t pitch = token_pitch;
  rc = check_tokens(q, cache, at, &pitch);
  if (rc) return rc;
  if (q->shape[2] % cache->kv_heads) return GL_ERR_SHAPE;
  if (!(scale > 0.f) || !(scale <= 1.7014118e38f)) return GL_ERR_SHAPE;   // (2^127: times log2(e) it is still finite)
  gl_ap want = *q;
  want.dtype = (flags & GL_OUT_BF16) ? GL_BF16 : GL_F32;
  rc = check_same_meta(want, out);
  if (rc) return rc;
  rc = check_data(out);
  if (rc) return rc;
  const size_t need = gl_attend_cache4_workspace(q, cache);
  if (!workspace || workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 1023u)) return GL_ERR_WORKSPACE;
  const int64_t group = q->shape[2] / cache->kv_heads, rows = q->shape[1] * group;
  const bool f32 = !(flags & GL_OUT_BF16);
  const AttKernel k = pick_kernel(rows, cache->head_dim, f32);
  const int64_t row_blocks = (rows + k.rows - 1) / k.rows, segments = q->shape[0] * cache->kv_heads * row_blocks;
  if (rows > INT32_MAX - 512 || segments > INT32_MAX) return GL_ERR_UNSUPPORTED;
  rc = att_grid(k, cache->head_dim, f32, &p.grid);
  if (rc) return rc;
  p.q = static_cast<const uint16_t*>(q->data);
  p.out = out->data;
  p.part = static_cast<float*>(workspace);
  p.q_pitch = pitch;
  p.T = static_cast<int>(q->shape[1]);
  p.heads = static_cast<int>(q->shape[2]);
  p.group = static_cast<int>(group);
  p.rows = static_cast<int>(rows);
  p.row_blocks = static_cast<int>(row_blocks);
  p.scale_log2 = scale * 1.4426950408889634f;
  p.step = std::min(8.f / p.scale_log2, 1.329228e36f);   // (2^120 stands for more: all scores are the same to such a scale)
  p.out_bf16 = f32 ? 0 : 1;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  p.R = k.rows;
  p.tile_log2 = k.tile == 32 ? 5 : k.tile == 64 ? 6 : 7;
  p.div_group.set(group);
  // (no more than a segment can have: a block that takes several short segments takes them one after the other)
  p.lead = k.lead;
  p.min_share = k.lead + std::min<int>(k.min_share, (p.c.capacity + k.tile - 1) / k.tile);
  // A cache of at most four tiles per sequence: a block per segment, one launch (8 sequences of 100 tokens, 8 heads: 11.2 us
  // with the list and the joining kernel, 7.0 us without; 64 of 256, 32 heads: 19.3 and 12.1).  Longer ones have warps with
  // several tiles, which the list spreads over the blocks.
  p.alone = p.c.capacity <= kAloneTiles * k.tile ? 1 : 0;
  const int64_t blocks = p.alone ? segments : p.grid;
  if (launch_pdl(k.fn, dim3(static_cast<unsigned>(blocks)), dim3(static_cast<unsigned>(k.threads)), static_cast<size_t>(k.smem), st, 1, p) !=
      cudaSuccess)
    return GL_ERR_CUDA;
  if (p.alone) return GL_OK;
  JoinShape js = {kJoinWarps, 1};
  int64_t live = std::min<int64_t>(rows, k.rows), row_groups = live;
  if (segments * live > 4 * num_sms()) {   // (four blocks per SM at once)
    js.wpr = live <= 1 ? 8 : live <= 2 ? 4 : live <= 4 ? 2 : 1;
    js.rows_per_block = static_cast<int>(std::min<int64_t>(live, 64));
    row_groups = (live + js.rows_per_block - 1) / js.rows_per_block;
  }
  void (*const join)(AttendParams, JoinShape) = cache->head_dim == 64 ? attend_join<2> : cache->head_dim == 128 ? attend_join<4> : attend_join<8>;
  return launch_pdl(join, dim3(static_cast<unsigned>(segments), static_cast<unsigned>(row_groups)), dim3(32 * kJoinWarps), 0, st, 1, p,
                    js) == cudaSuccess ? GL_OK : GL_ERR_CUDA;
}

}  // extern "C"
