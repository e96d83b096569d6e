// Attention over 4-bit pages for many query rows (prompts read in pieces): the two products on tcgen05.
// Included by gl_attend.cu, whose cache layout, work list and joining it uses.
//
// A block has MT x 128 rows that share a kv head and walks along the tokens in tiles of TT.  Eight warps widen the
// tile's codes to bf16, scales included (two significant bits times a power of two: exact), into the swizzled shared-
// memory layouts of the MMA operands: K as [token][dim] (K-major B of S = Q K^T), V as [token][dim] too, which is the
// MN-major B of O = P V.  Scores come back from tensor memory a row per thread, are turned into weights and go back
// into the columns they came from, as the A operand of the second product.  The maximum that the weights refer to is
// moved only when a weight would pass 2^-8: then the largest one becomes 2^-16, so that O is rarely rescaled, and their
// sum over all tokens is about 1 at most, so that O is not much larger than the values.  It is one of the scores, subtracted
// before the product with the softmax scale, two values to an instruction: scores of any size keep their differences.
// MT = 2: while the softmax warps of one half work, the tensor core works for the other.
// TERMS = 1 rounds the weights to bf16 (8 bits; the result is bf16 too); TERMS = 3 carries them as three bf16 terms
// for fp32 results.
//
// 512 tokens behind 5001 and 8192 cached ones, 32 heads over 8 of 128, channels of unequal size: 175 us, 610 TFLOP/s, 0.37
// of the measured bf16 rate; fp32 results 369 us.  Heads 64 wide 146 us, 256 wide 500 us, fp32 results 674 us.  Per pair of 128-row tiles and 128 tokens (5.5 k cycles): 2 k of matrix instructions; the
// exponentials of 256 rows take 2 k cycles of their unit; a widening warp is busy 4.2 k (1.3 k each for K and V, 1.6 k to ask
// for the next tile).  What is left is waiting for one another: the scores of a half are only there after its turn
// on the tensor core.  Before: widening by four warps with a condition per word 259 us.
//
// Dims appear in operand order: the conversion of a 32-bit word yields pairs (i, i + 4) for K, where Q's rows are
// stored in the same order, and pairs of neighbouring blocks for V, undone when the result is stored.
#pragma once

#include <type_traits>

namespace {

template <int NB, int TERMS>
struct ManyCfg {
  static constexpr int D = 32 * NB;
  static constexpr int MT = (NB <= 4 && TERMS == 1) ? 2 : 1;
  static constexpr int TT = NB == 8 ? 64 : 128;                 // tokens per tile
  static constexpr int kRows = 128 * MT;
  static constexpr int kQ = D == 64 ? 32768 : 128 * D * 2;      // bytes of one Q tile (results are staged in its rows)
  static constexpr int kKV = TT * D * 2;                        // bytes of a K or V tile
  static constexpr int kStages = 2;
  static constexpr int kWidenWarps = 8;
  static constexpr int kWarps = 4 * MT + kWidenWarps + 1;
  static constexpr int kThreads = 32 * kWarps;
  static constexpr int kSmem = MT * kQ + kStages * 2 * kKV + 1024 + 640;
  // tensor memory: scores (weights take their place), third terms, results
  static constexpr int kS = 0;
  static constexpr int kLow = MT * TT;
  static constexpr int kO = 512 - MT * D;
  static_assert(kLow + (TERMS == 3 ? TT / 2 : 0) <= kO, "tensor memory");
  static_assert(kSmem <= 232448, "shared memory");
};

// D[tmem] (+)= A[tmem] * B[smem]: A is a row per lane, two bf16 values per column
__device__ __forceinline__ void tc_mma_bf16_ta(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tc_store_16cols(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tc_load_8cols(uint32_t taddr, uint32_t (&r)[8]) {   // (waits for nothing)
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tc_wait_load() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
// Byte of 16-byte piece `piece` (0..15) of staged row `row`: 128 bytes in each of the Q tile's first two chunks, in that
// row's own place, so that no warp touches another's rows.
__device__ __forceinline__ uint32_t stage_piece(int row, int piece) {
  return (piece >> 3) * 16384 + row * 128 + (((piece & 7) ^ (row & 7)) << 4);
}
__device__ __forceinline__ void tc_wait_store() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Scales of four blocks, a byte each: is one of them above 2^1 (e > 128)?
__device__ __forceinline__ bool any_above_128(uint32_t e4) { return (((e4 & 0x7F7F7F7Fu) + 0x7F7F7F7Fu) & e4 & 0x80808080u) != 0u; }

// Is one of them NaN (e = 255)?
__device__ __forceinline__ bool any_255(uint32_t e4) { return ((((~e4) & 0x7F7F7F7Fu) + 0x7F7F7F7Fu) | ~e4 | 0x7F7F7F7Fu) != 0xFFFFFFFFu; }

// Eight codes (pairs: code i of the low and of the high half) -> four bf16 pairs times the scales of bytes lo and hi of e4.
// 2^(e - 1), the factor that the moved codes lack, is a bf16 up to e = 128.  ABOVE: some scale may be larger; 2^126 and
// 2^(e - 127) one after the other (Inf for e = 255: a NaN block's codes are zeros, and zero times Inf is NaN).
template <bool ABOVE>
__device__ __forceinline__ uint4 mx4_pairs_bf16(uint32_t z, uint32_t e4, int lo, int hi) {
  uint32_t h[4];
  mx4_pairs_moved(z, h);
  const uint32_t pair = __byte_perm(e4, 0u, lo | 4 << 4 | hi << 8 | 4 << 12);
  if constexpr (ABOVE) {
    const uint32_t f = __vmaxu2(pair * 128u, 0x00400040u);   // (e = 0: 2^-127 is subnormal)
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = mul_bf16x2(mul_bf16x2(h[i], 0x7E807E80u), f);
  } else {
    const uint32_t f = pair * 128u + 0x3F003F00u;            // 2^(e - 1) in both halves
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = mul_bf16x2(h[i], f);
  }
  return make_uint4(h[0], h[1], h[2], h[3]);
}

// What a widening thread holds of a tile: its codes and scales of one of K and V.
template <int NB, int ITEMS>
struct Held {
  uint32_t word[ITEMS][NB];
  uint32_t exps[ITEMS][NB <= 4 ? 1 : 2];
};
// Item i: NB words and NB scale bytes.
template <int NB, int ITEMS>
__device__ __forceinline__ void get(Held<NB, ITEMS>& x, int i, const uint8_t* codes, const uint8_t* scales) {
  if constexpr (NB == 2) {
    const uint2 a = *reinterpret_cast<const uint2*>(codes);
    x.word[i][0] = a.x; x.word[i][1] = a.y;
    x.exps[i][0] = *reinterpret_cast<const uint16_t*>(scales);
  } else {
#pragma unroll
    for (int k = 0; k < NB / 4; ++k) {
      const uint4 a = *reinterpret_cast<const uint4*>(codes + 16 * k);
      x.word[i][4 * k] = a.x; x.word[i][4 * k + 1] = a.y; x.word[i][4 * k + 2] = a.z; x.word[i][4 * k + 3] = a.w;
    }
    if constexpr (NB == 4) {
      x.exps[i][0] = *reinterpret_cast<const uint32_t*>(scales);
    } else {
      const uint2 a = *reinterpret_cast<const uint2*>(scales);
      x.exps[i][0] = a.x; x.exps[i][NB == 8 ? 1 : 0] = a.y;
    }
  }
}
// lo += low half, hi += high half
__device__ __forceinline__ void add_halves_bf16(uint32_t two, float& lo, float& hi) {
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tadd.f32.bf16 %0, l, %0;\n\tadd.f32.bf16 %1, h, %1;\n\t}"
      : "+f"(lo), "+f"(hi) : "r"(two));
}
// (a + b) * c + d of two values at a time
__device__ __forceinline__ float2 add_mul_add2(float a0, float a1, float b, float c, float d) {
  float2 y;
  asm("{\n\t.reg .b64 a, b, c, d;\n\t"
      "mov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %4};\n\tmov.b64 c, {%5, %5};\n\tmov.b64 d, {%6, %6};\n\t"
      "add.rn.f32x2 a, a, b;\n\tfma.rn.f32x2 a, a, c, d;\n\t"
      "mov.b64 {%0, %1}, a;\n\t}"
      : "=f"(y.x), "=f"(y.y) : "f"(a0), "f"(a1), "f"(b), "f"(c), "f"(d));
  return y;
}
// A token that does not exist or is not seen by any row.
template <int NB, int ITEMS>
__device__ __forceinline__ void clear(Held<NB, ITEMS>& x, int i) {
#pragma unroll
  for (int k = 0; k < NB; ++k) x.word[i][k] = 0;
#pragma unroll
  for (int k = 0; k < (NB <= 4 ? 1 : 2); ++k) x.exps[i][k] = 0;
}

template <int NB, int TERMS>
__global__ void __launch_bounds__(ManyCfg<NB, TERMS>::kThreads, 1) attend_many(const AttendParams p) {
  using Cfg = ManyCfg<NB, TERMS>;
  constexpr int D = Cfg::D, MT = Cfg::MT, TT = Cfg::TT, kGroups = TT / 16;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  unsigned char* gen = smem_raw + (base - raw);
  const uint32_t q_at = base, kv_at = base + MT * Cfg::kQ;       // stage s: K at kv_at + 2 s kKV, V behind it
  unsigned char* tail = gen + MT * Cfg::kQ + Cfg::kStages * 2 * Cfg::kKV;
  uint64_t* bars = reinterpret_cast<uint64_t*>(tail);
  const uint32_t bar = smem_u32(bars);
  const uint32_t b_kfull = bar, b_kempty = bar + 16, b_vfull = bar + 32, b_vempty = bar + 48, b_q = bar + 64, b_s = bar + 80,
                 b_p = bar + 96, b_o = bar + 112;                // two each
  const uint32_t b_item = bar + 280;                             // one
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 16);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  volatile uint32_t* have = reinterpret_cast<volatile uint32_t*>(tmem_slot + 2);   // [4] groups of a tile that have a page
  int* nan_from = reinterpret_cast<int*>(tmem_slot + 6);                           // [4][NB] first token whose V block is NaN
  int64_t* scratch = reinterpret_cast<int64_t*>(tail + 288);                       // [2 * kWarps + 4]
  static_assert(288 + 16 * Cfg::kWarps + 32 <= 640 && 128 + 24 + 16 * 8 <= 280, "tail");
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr int kWiden = 4 * MT, kMma = kWiden + Cfg::kWidenWarps;

  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(b_kfull + 8 * i, Cfg::kWidenWarps);
      mbar_init(b_vfull + 8 * i, Cfg::kWidenWarps);
      mbar_init(b_kempty + 8 * i, 1);
      mbar_init(b_vempty + 8 * i, 1);
      mbar_init(b_q + 8 * i, 4);
      mbar_init(b_s + 8 * i, 1);
      mbar_init(b_p + 8 * i, 4);
      mbar_init(b_o + 8 * i, 1);
    }
    mbar_init(b_item, Cfg::kWidenWarps);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == kMma) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(tmem_slot)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();   // tensor memory is there before the next kernel, which may want some and wait for this one, can start
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  pdl_wait();
  pdl_launch_dependents();
  Walk w;
  w.start<Cfg::kThreads>(p, blockIdx.x, scratch);
  store_empty<Cfg::kThreads>(p, w, D);
  uint32_t it = 0;     // tiles so far, the same for every role
  uint32_t item = 0;
  bool ok = true;

  if (warp < kWiden) {
    // ---------------- softmax: thread = row ----------------
    const int m = warp >> 2, r = (warp & 3) * 32 + lane;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t s_col = tmem + lanes + Cfg::kS + m * TT, o_col = tmem + lanes + Cfg::kO + m * D;
    const uint32_t low_col = tmem + lanes + Cfg::kLow;
    const float cf = p.scale_log2, ninf = __uint_as_float(0xFF800000u);
    for (; ok && w.next(p); ++item) {
      const int row = w.rb * Cfg::kRows + m * 128 + r;
      const bool live = row < p.rows;
      // Q: the warp's 32 rows, 16 bytes a lane along the rows; dims 8c .. 8c + 7 in the order 0 4 1 5 2 6 3 7, 128-byte swizzle
      {
        constexpr int kLanes = D / 8, kAtOnce = kLanes < 32 ? 32 / kLanes : 1;   // lanes to a row, rows to an access
        const int c = lane % kLanes;
#pragma unroll 8
        for (int i = 0; i < 32; i += kAtOnce) {
          const int r1 = (warp & 3) * 32 + i + lane / kLanes, row1 = w.rb * Cfg::kRows + m * 128 + r1;
          uint4 x = make_uint4(0, 0, 0, 0);
          if (row1 < p.rows) x = *reinterpret_cast<const uint4*>(q_row(p, w.b, w.h, row1, D) + 8 * c);
          const uint4 y = make_uint4(__byte_perm(x.x, x.z, 0x5410), __byte_perm(x.x, x.z, 0x7632), __byte_perm(x.y, x.w, 0x5410),
                                     __byte_perm(x.y, x.w, 0x7632));
          *reinterpret_cast<uint4*>(gen + m * Cfg::kQ + (c >> 3) * 16384 + r1 * 128 + (((c & 7) ^ (r1 & 7)) << 4)) = y;
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(b_q + 8 * m);
      }
      const int limit = live ? min(w.len, w.len - p.T + row_token(p, row) + 1) : 0;
      float ref = ninf, sum = 0.f;   // weights are 2^((s - ref) cf - 16)
      for (int tile = w.t0; tile < w.t1; ++tile, ++it) {
        if (!mbar_wait(b_s + 8 * m, it & 1u, abort_flag)) { ok = false; break; }
        tc_fence_after();
        const int open = limit - tile * TT;           // columns that this row sees
        const uint32_t groups = have[it & 3u];
        const bool masked = __any_sync(0xFFFFFFFFu, open < TT) || groups != (1u << kGroups) - 1u;
        float top = ninf;
#pragma unroll 1
        for (int j = 0; j < TT / 32; ++j) {
          uint32_t x[32];
          tc_load_32cols(s_col + 32 * j, x);
          if (masked) {
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (32 * j + i < open && (groups >> (2 * j + (i >> 4)) & 1u)) top = fmaxf(top, __uint_as_float(x[i]));
          } else {
            float t1 = ninf, t2 = ninf, t3 = ninf;
#pragma unroll
            for (int i = 0; i < 32; i += 4) {
              top = fmaxf(top, __uint_as_float(x[i]));
              t1 = fmaxf(t1, __uint_as_float(x[i + 1]));
              t2 = fmaxf(t2, __uint_as_float(x[i + 2]));
              t3 = fmaxf(t3, __uint_as_float(x[i + 3]));
            }
            top = fmaxf(fmaxf(top, t1), fmaxf(t2, t3));
          }
        }
        const bool move = top > ref + p.step;         // (ref = -Inf: whenever the row sees something)
        if (__any_sync(0xFFFFFFFFu, move) && tile > w.t0) {
          // O holds the tiles before this one: bring it to the new reference
          if (!mbar_wait(b_o + 8 * m, (it - 1) & 1u, abort_flag)) { ok = false; break; }
          tc_fence_after();
          const float f = move ? ex2((ref - top) * cf) : 1.f;
          sum *= f;
#pragma unroll 1
          for (int j = 0; j < D / 16; ++j) {
            uint32_t x[16];
            tc_load_16cols(o_col + 16 * j, x);
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = __float_as_uint(__uint_as_float(x[i]) * f);
            tc_store_16cols(o_col + 16 * j, x);
          }
        }
        if (move) ref = top;
        const float down = ref == ninf ? 0.f : -ref;
        float part[2] = {0.f, 0.f};
        // (two copies of the loop: a test of `masked` per weight would cost as much as the weight)
        const auto weigh = [&](auto with_mask) {
#pragma unroll 1
          for (int j = 0; j < TT / 32; ++j) {
            uint32_t x[32], hi[16], mid[16], lo[16];
            tc_load_32cols(s_col + 32 * j, x);
#pragma unroll
            for (int i = 0; i < 32; i += 2) {
              const float2 y = add_mul_add2(__uint_as_float(x[i]), __uint_as_float(x[i + 1]), down, cf, -16.f);
              float a = ex2(y.x), b = ex2(y.y);
              if constexpr (decltype(with_mask)::value) {
                const bool there = groups >> (2 * j + (i >> 4)) & 1u;
                a = there && 32 * j + i < open ? a : 0.f;
                b = there && 32 * j + i + 1 < open ? b : 0.f;
              }
              hi[i / 2] = pack_bf16x2(__float_as_uint(a), __float_as_uint(b));
              if (TERMS == 1) {
                add_halves_bf16(hi[i / 2], part[0], part[1]);   // (the sum is that of the weights as they are used)
              } else {
                part[0] += a;
                part[1] += b;
                a -= __uint_as_float(hi[i / 2] << 16);
                b -= __uint_as_float(hi[i / 2] & 0xFFFF0000u);
                mid[i / 2] = pack_bf16x2(__float_as_uint(a), __float_as_uint(b));
                a -= __uint_as_float(mid[i / 2] << 16);
                b -= __uint_as_float(mid[i / 2] & 0xFFFF0000u);
                lo[i / 2] = pack_bf16x2(__float_as_uint(a), __float_as_uint(b));
              }
            }
            tc_store_16cols(s_col + 32 * j, hi);
            if (TERMS == 3) {
              tc_store_16cols(s_col + 32 * j + 16, mid);
              tc_store_16cols(low_col + 16 * j, lo);
            }
          }
        };
        if (masked) weigh(std::true_type{});
        else weigh(std::false_type{});
        sum += part[0] + part[1];
        tc_wait_store();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(b_p + 8 * m);
      }
      if (!ok) break;
      // ---- result of the item
      if (!mbar_wait(b_o + 8 * m, (it - 1) & 1u, abort_flag)) { ok = false; break; }
      tc_fence_after();
      const bool whole = w.whole();
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      float* slot = w.slot(p, D) + static_cast<int64_t>(m * 128) * (D + 2);
      if (!whole) *reinterpret_cast<float2*>(slot + r * (D + 2)) = make_float2(ref * cf, sum * rounded_off(ref, cf));
      const int* nan_at = nan_from + (item & 3u) * NB;
      // 64 dims at a time (a pair of blocks), by way of the warp's rows of its Q tile, which no product reads any more:
      // written a row per lane, stored along the rows.  Columns (g * NB/2 + pair) * 8 + 2 i + half hold dims
      // 32 (2 pair + half) + 4 g + i.
      const uint32_t rows_at = q_at + m * Cfg::kQ;
#pragma unroll 1
      for (int pair = 0; pair < NB / 2; ++pair) {
#pragma unroll
        for (int hg = 0; hg < 2; ++hg) {   // four g at a time
          uint32_t x[4][8];
#pragma unroll
          for (int k = 0; k < 4; ++k) tc_load_8cols(o_col + ((4 * hg + k) * (NB / 2) + pair) * 8, x[k]);
          tc_wait_load();
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const bool bad = nan_at[2 * pair + half] < limit;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              uint32_t v[4];
#pragma unroll
              for (int i = 0; i < 4; ++i) v[i] = bad ? 0x7FC00000u : __float_as_uint(__uint_as_float(x[k][2 * i + half]) * inv);
              asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(rows_at + stage_piece(r, half * 8 + 4 * hg + k)),
                           "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
            }
          }
        }
        __syncwarp();
#pragma unroll 4
        for (int i = 0; i < 32; ++i) {
          const int r1 = (warp & 3) * 32 + i, row1 = w.rb * Cfg::kRows + m * 128 + r1, d = 64 * pair + 2 * lane;
          float2 v;
          asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(rows_at + stage_piece(r1, lane >> 1) + (lane & 1) * 8));
          if (!whole) {
            *reinterpret_cast<float2*>(slot + static_cast<int64_t>(r1) * (D + 2) + 2 + d) = v;
          } else if (row1 < p.rows) {
            const int64_t to = out_row(p, w.b, w.h, row1, D) + d;
            if (p.out_bf16)
              *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(p.out) + to) = pack_bf16x2(__float_as_uint(v.x), __float_as_uint(v.y));
            else
              *reinterpret_cast<float2*>(static_cast<float*>(p.out) + to) = v;
          }
        }
        __syncwarp();
      }
      tc_fence_before();
    }
  } else if (warp < kMma) {
    // ---------------- widening: codes from the pages to bf16 operands ----------------
    // Thread: a fourth of a token's codes, tokens 64 apart.  Codes and scales of the next tile are asked for before those of
    // the current one are widened, its pages a tile earlier still.
    constexpr int kItems = TT / 64;
    const int dw = warp - kWiden, j = lane >> 3;
    for (; ok && w.next(p); ++item) {
      // the item's NaN positions are cleared before any warp of this role notes one
      if (dw == 0 && lane < NB) nan_from[(item & 3u) * NB + lane] = INT32_MAX;
      __syncwarp();
      if (lane == 0) mbar_arrive(b_item);
      if (!mbar_wait(b_item, item & 1u, abort_flag)) { ok = false; break; }
      Held<NB, kItems> hk[2], hv[2];
      uint32_t tile_have[2];
      int32_t page = -1;        // of group `lane` of the tile to be asked for next
      auto find = [&](int tile) {
        const int pos = tile * TT + lane * 16;
        page = -1;
        if (lane < kGroups && tile < w.t1 && pos < w.seen)
          page = p.c.table[static_cast<int64_t>(w.b) * p.c.width + p.c.div_page.div(static_cast<uint32_t>(pos))];
      };
      auto fetch = [&](int tile, Held<NB, kItems>& k, Held<NB, kItems>& v, uint32_t& groups) {
        const bool there = page >= 0 && page < p.c.pages;
        groups = __ballot_sync(0xFFFFFFFFu, there);
        uint32_t slot, in_page;   // lane g: where group g lies
        p.c.div_page.divmod(static_cast<uint32_t>(tile * TT + (lane & 7) * 16), slot, in_page);
        const uint64_t mine = reinterpret_cast<uint64_t>(p.c.data) + static_cast<int64_t>(page) * p.c.page_stride +
                              w.h * p.c.head_stride + (in_page / kGroup) * group_bytes(D);
        // (the plain case is a branch of its own: a condition per load costs more than the load)
        const bool plain = groups == (1u << kGroups) - 1u && (tile + 1) * TT <= w.seen;
        const int in_group = (dw * 8 + (lane & 7)) & 15, jv = j ^ ((in_group & 2) ? 2 : 0);
        const uint8_t* grp[kItems];
#pragma unroll
        for (int i = 0; i < kItems; ++i) grp[i] = reinterpret_cast<const uint8_t*>(__shfl_sync(0xFFFFFFFFu, mine, 4 * i + (dw >> 1)));
        if (plain) {
#pragma unroll
          for (int i = 0; i < kItems; ++i) {
            get(k, i, grp[i] + in_group * (D / 2) + j * NB * 4, grp[i] + k_scales_at(D) + in_group * NB);
            get(v, i, grp[i] + v_codes_at(D) + in_group * (D / 2) + jv * NB * 4, grp[i] + v_scales_at(D) + in_group * NB);
          }
        } else {
#pragma unroll
          for (int i = 0; i < kItems; ++i) {
            clear(k, i);
            clear(v, i);
            if ((groups >> (4 * i + (dw >> 1)) & 1u) && tile * TT + 64 * i + dw * 8 + (lane & 7) < w.seen) {
              get(k, i, grp[i] + in_group * (D / 2) + j * NB * 4, grp[i] + k_scales_at(D) + in_group * NB);
              get(v, i, grp[i] + v_codes_at(D) + in_group * (D / 2) + jv * NB * 4, grp[i] + v_scales_at(D) + in_group * NB);
            }
          }
        }
      };
      const auto widen_k = [&](auto above, unsigned char* kt, const Held<NB, kItems>& x) {
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
          const int tok = 64 * i + dw * 8 + (lane & 7);
#pragma unroll
          for (int b = 0; b < NB; ++b) {
            const int c = b * 4 + j;
            *reinterpret_cast<uint4*>(kt + (c >> 3) * (TT * 128) + tok * 128 + (((c & 7) ^ (tok & 7)) << 4)) =
                mx4_pairs_bf16<decltype(above)::value>(x.word[i][b], x.exps[i][b >> 2], b & 3, b & 3);
          }
        }
      };
      const auto widen_v = [&](auto above, unsigned char* vt, const Held<NB, kItems>& x) {
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
          const int tok = 64 * i + dw * 8 + (lane & 7);
#pragma unroll
          for (int k = 0; k < NB; ++k) {
            const int b = 2 * (k % (NB / 2)), c = j * NB + k;
            *reinterpret_cast<uint4*>(vt + (c >> 3) * (TT * 128) + tok * 128 + (((c & 7) ^ (tok & 7)) << 4)) =
                mx4_pairs_bf16<decltype(above)::value>(x.word[i][k], x.exps[i][b >> 2], b & 3, (b & 3) + 1);
          }
        }
      };
      // V blocks that are NaN: zeros in their place; the NaN goes to the rows that see the token when the result is stored
      const auto take_nan = [&](Held<NB, kItems>& x, int tile) {
#pragma unroll
        for (int i = 0; i < kItems; ++i)
#pragma unroll
          for (int b = 0; b < NB; ++b)
            if ((x.exps[i][b >> 2] >> (8 * (b & 3)) & 255u) == 255u) {
              atomicMin(nan_from + (item & 3u) * NB + b, tile * TT + 64 * i + dw * 8 + (lane & 7));
              x.exps[i][b >> 2] &= ~(255u << (8 * (b & 3)));
#pragma unroll
              for (int k = 0; k < NB; ++k)   // words of the block pair that b is in: its half
                if (2 * (k % (NB / 2)) == (b & ~1)) x.word[i][k] &= b & 1 ? 0x0000FFFFu : 0xFFFF0000u;
            }
      };
      auto widen = [&](int tile, Held<NB, kItems>& hk, Held<NB, kItems>& hv, uint32_t groups) {
        const uint32_t st = it & 1u, ph = (it >> 1) & 1u;
        bool large = false, nan = false;
#pragma unroll
        for (int i = 0; i < kItems; ++i)
#pragma unroll
          for (int k = 0; k < (NB <= 4 ? 1 : 2); ++k) {
            large |= any_above_128(hk.exps[i][k]) || any_above_128(hv.exps[i][k]);
            nan |= any_255(hv.exps[i][k]);
          }
        large = __any_sync(0xFFFFFFFFu, large);
        if (__any_sync(0xFFFFFFFFu, nan)) take_nan(hv, tile);
        if (!mbar_wait(b_kempty + 8 * st, ph ^ 1u, abort_flag)) return false;
        if (dw == 0 && lane == 0) have[it & 3u] = groups;
        unsigned char* kt = gen + MT * Cfg::kQ + 2 * st * Cfg::kKV;
        if (large) widen_k(std::true_type{}, kt, hk);
        else widen_k(std::false_type{}, kt, hk);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(b_kfull + 8 * st);
        if (!mbar_wait(b_vempty + 8 * st, ph ^ 1u, abort_flag)) return false;
        if (large) widen_v(std::true_type{}, kt + Cfg::kKV, hv);
        else widen_v(std::false_type{}, kt + Cfg::kKV, hv);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(b_vfull + 8 * st);
        return true;
      };
      find(w.t0);
      fetch(w.t0, hk[0], hv[0], tile_have[0]);
      find(w.t0 + 1);
      for (int tile = w.t0; tile < w.t1 && ok; tile += 2) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          if (tile + u >= w.t1 || !ok) break;
          if (tile + u + 1 < w.t1) {
            fetch(tile + u + 1, hk[u ^ 1], hv[u ^ 1], tile_have[u ^ 1]);
            find(tile + u + 2);
          }
          ok = widen(tile + u, hk[u], hv[u], tile_have[u]);
          ++it;
        }
      }
      if (!ok) break;
    }
  } else {
    // ---------------- MMA issuer ----------------
    const bool leader = elect_one();
    constexpr uint32_t idesc_s = make_idesc(128, TT), idesc_o = make_idesc(128, D) | (1u << 16);   // V is MN-major
    const uint64_t dq = make_desc(q_at, 16, 1024, 2), dk = make_desc(kv_at, 16, 1024, 2);
    const uint64_t dv = make_desc(kv_at + Cfg::kKV, TT * 128, 1024, 2);
    // S_m of tile number n (0-based over the block's life)
    auto scores = [&](uint32_t n, int m) {
      const uint32_t st = n & 1u;
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        const uint64_t a = dq + ((m * Cfg::kQ + (k >> 2) * 16384 + (k & 3) * 32) >> 4);
        const uint64_t b = dk + ((2 * st * Cfg::kKV) >> 4) + (((k >> 2) * (TT * 128) + (k & 3) * 32) >> 4);
        if (leader) tc_mma_bf16(tmem + Cfg::kS + m * TT, a, b, idesc_s, k ? 1u : 0u);
      }
      if (leader) tc_commit(b_s + 8 * m);
    };
    for (; ok && w.next(p); ++item) {
      const int n = w.t1 - w.t0;
      for (int m = 0; m < MT && ok; ++m) ok = mbar_wait(b_q + 8 * m, item & 1u, abort_flag);
      if (ok) ok = mbar_wait(b_kfull + 8 * (it & 1u), (it >> 1) & 1u, abort_flag);
      if (!ok) break;
      tc_fence_after();
      for (int m = 0; m < MT; ++m) scores(it, m);
      if (leader) tc_commit(b_kempty + 8 * (it & 1u));
      for (int t = 0; t < n && ok; ++t, ++it) {
        const uint32_t st = it & 1u;
        if (!mbar_wait(b_vfull + 8 * st, (it >> 1) & 1u, abort_flag)) { ok = false; break; }
        if (t + 1 < n && !mbar_wait(b_kfull + 8 * (st ^ 1u), ((it + 1) >> 1) & 1u, abort_flag)) { ok = false; break; }
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          if (ok && !mbar_wait(b_p + 8 * m, it & 1u, abort_flag)) ok = false;
          if (!ok) break;
          tc_fence_after();
#pragma unroll
          for (int k = 0; k < TT / 16; ++k) {
            const uint64_t b = dv + ((2 * st * Cfg::kKV) >> 4) + ((k * 2048) >> 4);
            const uint32_t s = tmem + Cfg::kS + m * TT + 32 * (k >> 1) + 8 * (k & 1), o = tmem + Cfg::kO + m * D;
            if (leader) {
              tc_mma_bf16_ta(o, s, b, idesc_o, t > 0 || k > 0 ? 1u : 0u);
              if (TERMS == 3) {
                tc_mma_bf16_ta(o, s + 16, b, idesc_o, 1u);
                tc_mma_bf16_ta(o, tmem + Cfg::kLow + 8 * k, b, idesc_o, 1u);
              }
            }
          }
          if (leader) tc_commit(b_o + 8 * m);
          if (t + 1 < n) scores(it + 1, m);
        }
        if (ok && leader) {
          tc_commit(b_vempty + 8 * st);
          if (t + 1 < n) tc_commit(b_kempty + 8 * (st ^ 1u));
        }
      }
    }
  }
  __syncwarp();
  if (*abort_flag) {   // a block that gave up lets its matrix instructions in flight end before it leaves
    const uint64_t t0 = global_timer();
    while (global_timer() - t0 < 20000000ull) { }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kMma) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

}  // namespace
