// fqt_gated.cuh -- the activations of a gated feed-forward block, and what its product
// kernel does with the sums of both projections.
#pragma once

#include <type_traits>

#include "fqt_fp8_core.cuh"

namespace fqt {

// ---------------------------------------------------------------------------
// Activations
// ---------------------------------------------------------------------------
// sigma(z) = 1 / (1 + 2^(-z log2 e)) by the hardware's base-2 exponential and reciprocal, for
// fp32 outputs too: the epilogue that waits for them bounds the kernel with codes.  They
// themselves are 2 units off, and the exponential's argument is rounded, which counts where
// sigma is small (measured: 2e-7 of sigma at z > -2, 9e-7 at -20, 3.6e-6 at -87).  Below
// 2^-126 (z < -87.3) sigma is 0.  tanh.approx would leave 5e-4.
constexpr float kLog2E = 1.4426950408889634f;
__device__ __forceinline__ float exp2_of(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float inverse_of(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float sigmoid_of(float z) {
  return inverse_of(__fadd_rn(1.0f, exp2_of(__fmul_rn(z, -kLog2E))));
}

// gelu's tanh form is g sigma(z(g)), z = 2 sqrt(2 / pi) (g + 0.044715 g^3).  Past |g| = 64
// sigma is 0 or 1, and g^2 times a slope of 0 would be no number.
constexpr float kTanhScale = 1.5957691216057308f, kTanhCube = 0.044715f;
__device__ __forceinline__ float tanh_arg(float g) { return fminf(fmaxf(g, -64.0f), 64.0f); }
__device__ __forceinline__ float tanh_z(float c) {
  return __fmul_rn(kTanhScale, fmaf(__fmul_rn(__fmul_rn(kTanhCube, c), c), c, c));
}

// gelu's Phi(-x) e^(x^2/2), x >= 0, is t P(t) with t = 1 / (1 + 0.35 x): P, of degree 8, is the
// polynomial whose largest relative error over 0 <= x <= 14 is least (3.2e-8, 3e-7 in fp32
// arithmetic; found by reweighted least squares).  Unlike an approximation of erf, it is as good
// in the tail, and its factor e^(-x^2/2) is the density that the slope needs.  That factor's
// argument is rounded like sigma's: gelu is off by 4e-7 of itself for |g| < 2, 1.3e-6 at -6,
// 3.6e-6 at -12 (0.5 erfc(-g / sqrt 2) in fp32 by 3e-7, 1.6e-6 and 1e-5).  (With CUDA's
// normcdff 8192 x 4096 x 1024 took 139 us.)
constexpr float kCdfScale = 0.35f;
constexpr int kCdfTerms = 9;
__device__ constexpr float kCdf[kCdfTerms] = {
    0.13962140679359436f, 0.1398618370294571f,   0.1198330670595169f,
    0.10550717264413834f, -0.023107722401618958f, 0.15917086601257324f,
    -0.255711168050766f,  0.1439700871706009f,   -0.029145577922463417f};

// Phi(g), and e^(-g^2/2).
__device__ __forceinline__ float cdf_of(float g, float &bell) {
  const float t = inverse_of(fmaf(fabsf(g), kCdfScale, 1.0f));
  float p = kCdf[kCdfTerms - 1];
#pragma unroll
  for (int i = kCdfTerms - 2; i >= 0; --i) p = fmaf(p, t, kCdf[i]);
  bell = exp2_of(__fmul_rn(__fmul_rn(g, g), -0.5f * kLog2E));
  const float q = __fmul_rn(__fmul_rn(p, t), bell);
  return g < 0.0f ? q : __fsub_rn(1.0f, q);
}

// act(g) and act'(g).  1 - sigma is e^-z sigma where it is the slope's factor on its own, so
// that it loses no digits where it is small.  e^-z is held at 2^126 there, and only there:
// past it sigma is 0, and a value that kept 2^-126 would be g 2^-126 far to the left (-3.5 at
// g = -3e38).  silu's slope is s + a (1 - s): there 1 - s is a difference, which is off by
// 2^-24 where the slope is next to 1.
constexpr float kPow126 = 8.507059173023462e37f;
template <int ACT>
__device__ __forceinline__ void act_and_slope(float g, float &a, float &d) {
  if constexpr (ACT == FQT_RELU) {
    a = g <= 0.0f ? 0.0f : g;  // NaN stays
    d = g > 0.0f ? 1.0f : a;   // (as here: a checkpoint that is no number shows in dg)
  } else if constexpr (ACT == FQT_GELU) {
    float bell;
    const float cdf = cdf_of(g, bell);
    a = __fmul_rn(g, cdf);
    d = fmaf(__fmul_rn(g, 0.3989422804014327f), bell, cdf);
  } else if constexpr (ACT == FQT_SILU) {
    const float s = sigmoid_of(g);
    a = __fmul_rn(g, s);
    d = fmaf(a, __fsub_rn(1.0f, s), s);
  } else {
    const float c = ACT == FQT_GELU_TANH ? tanh_arg(g) : g;
    const float z = ACT == FQT_GELU_TANH ? tanh_z(c) : g;
    const float t = exp2_of(__fmul_rn(z, -kLog2E)), s = inverse_of(__fadd_rn(1.0f, t));
    const float r = __fmul_rn(fminf(t, kPow126), s);  // 1 - s, and 0 where s is 0
    if constexpr (ACT == FQT_SIGMOID) {
      a = s;
      d = __fmul_rn(s, r);
    } else {
      a = __fmul_rn(g, s);
      const float dz = __fmul_rn(kTanhScale, fmaf(__fmul_rn(3.0f * kTanhCube, c), c, 1.0f));
      d = fmaf(__fmul_rn(__fmul_rn(c, r), s), dz, s);
      if (g != g) d = g;  // the limits take NaN away
    }
  }
}

__device__ __forceinline__ f32x2 both(float v) { return pack2(v, v); }

// Of two values at a time; silu's and gelu's in packed arithmetic, with the same roundings.
template <int ACT>
__device__ __forceinline__ void act_and_slope2(f32x2 g, f32x2 &a, f32x2 &d) {
  if constexpr (ACT == FQT_SILU) {
    float x, y;
    unpack2(mul2(g, both(-kLog2E)), x, y);
    unpack2(add2(pack2(exp2_of(x), exp2_of(y)), both(1.0f)), x, y);
    const f32x2 s = pack2(inverse_of(x), inverse_of(y));
    a = mul2(g, s);
    d = fma2(a, fma2(s, both(-1.0f), both(1.0f)), s);
  } else if constexpr (ACT == FQT_GELU) {
    float x, y, g0, g1;
    unpack2(g, g0, g1);
    unpack2(fma2(pack2(fabsf(g0), fabsf(g1)), both(kCdfScale), both(1.0f)), x, y);
    const f32x2 t = pack2(inverse_of(x), inverse_of(y));
    f32x2 p = both(kCdf[kCdfTerms - 1]);
#pragma unroll
    for (int i = kCdfTerms - 2; i >= 0; --i) p = fma2(p, t, both(kCdf[i]));
    unpack2(mul2(mul2(g, g), both(-0.5f * kLog2E)), x, y);
    const f32x2 bell = pack2(exp2_of(x), exp2_of(y)), q = mul2(mul2(p, t), bell);
    float q0, q1, r0, r1;
    unpack2(q, q0, q1);
    unpack2(fma2(q, both(-1.0f), both(1.0f)), r0, r1);
    const f32x2 cdf = pack2(g0 < 0.0f ? q0 : r0, g1 < 0.0f ? q1 : r1);
    a = mul2(g, cdf);
    d = fma2(mul2(g, both(0.3989422804014327f)), bell, cdf);
  } else {
    float g0, g1, a0, a1, d0, d1;
    unpack2(g, g0, g1);
    act_and_slope<ACT>(g0, a0, d0);
    act_and_slope<ACT>(g1, a1, d1);
    a = pack2(a0, a1);
    d = pack2(d0, d1);
  }
}

template <int ACT>
__device__ __forceinline__ f32x2 act2(f32x2 g) {
  f32x2 a, unused;
  act_and_slope2<ACT>(g, a, unused);
  return a;
}

template <typename F>
__device__ __forceinline__ void with_act(int act, F f) {
  switch (act) {
    case FQT_SILU: f(std::integral_constant<int, FQT_SILU>()); break;
    case FQT_GELU: f(std::integral_constant<int, FQT_GELU>()); break;
    case FQT_GELU_TANH: f(std::integral_constant<int, FQT_GELU_TANH>()); break;
    case FQT_RELU: f(std::integral_constant<int, FQT_RELU>()); break;
    default: f(std::integral_constant<int, FQT_SIGMOID>());
  }
}

// ---------------------------------------------------------------------------
// The product kernel's operands
// ---------------------------------------------------------------------------
// The right operand of a tile are 128 rows of the gate's weights (64 in a narrow tile) and the
// same of the up projection's (of a pair's CTAs, each loads one).  With few tokens the left operand are
// g.part rows of each, and what is left of its 128 rows is not used.
template <int NT, bool PAIR>
__device__ __forceinline__ void f8_load_gated(const F8Of<F8_GATED>::Maps &maps,
                                              const F8GatedArgs &g, uint8_t *stage,
                                              const F8Item &t, int kb, int rank, uint64_t *full) {
  const int32_t k = kb * kF8Block, m = (int32_t)t.m0, n = (int32_t)(t.n0 / 2);
  if constexpr (NT <= 64) {
    const uint32_t half = (uint32_t)g.part * kF8Block;
    mbar_expect_tx(full, 2 * half + NT * kF8Block);
    tma_load_2d(stage, &maps.a, k, m, full);
    tma_load_2d(stage + half, &maps.b2, k, m, full);
    tma_load_2d(stage + kTileBytes, &maps.b, k, 0, full);
  } else if constexpr (PAIR) {  // the leader's barrier counts both CTAs' bytes
    if (rank == 0) mbar_expect_tx(full, (uint32_t)(4 * kTileBytes));
    const uint32_t bar = leader_addr(full);
    tma_load_2d_pair(stage, &maps.a, k, m, bar);
    tma_load_2d_pair(stage + kTileBytes, rank ? &maps.b2 : &maps.b, k, n, bar);
  } else {
    mbar_expect_tx(full, (uint32_t)kTileBytes + NT * kF8Block);
    tma_load_2d(stage, &maps.a, k, m, full);
    tma_load_2d(stage + kTileBytes, &maps.b, k, n, full);
    tma_load_2d(stage + kTileBytes + NT / 2 * kF8Block, &maps.b2, k, n, full);
  }
}

// The scales of four K blocks for row 32 i + lane of the left operand (i < 4) or row
// 32 (i - 4) + lane of the right one; 1 past the ends, where the codes are zeros, so that
// such rows' sums are zeros too.
template <int NT>
__device__ __forceinline__ uint32_t f8_gated_scales(const F8GatedArgs &g, const F8Item &t,
                                                    int64_t group, int i, int lane) {
  const uint32_t *from;
  int64_t r, rows, pitch;
  if constexpr (NT <= 64) {
    const int at = 32 * i;
    if (i >= 4) {
      from = g.sb, pitch = g.spb, rows = g.N, r = at - BM + lane;
    } else {
      from = at < g.part ? g.sa : g.s2, pitch = g.spa;
      rows = at < 2 * g.part ? g.M : 0, r = t.m0 + at % g.part + lane;
    }
  } else if (i < 4) {
    from = g.sa, pitch = g.spa, rows = g.M, r = t.m0 + 32 * i + lane;
  } else {
    const int at = 32 * (i - 4);
    from = at < NT / 2 ? g.sb : g.s2, pitch = g.spb, rows = g.N;
    r = t.n0 / 2 + at % (NT / 2) + lane;
  }
  return r < rows ? __ldg(from + group * pitch + r) : 0x7F7F7F7Fu;
}

// ---------------------------------------------------------------------------
// The product kernel's epilogue
// ---------------------------------------------------------------------------
// The largest magnitude (NaN if one is).
__device__ __forceinline__ float top3(float a, float b, float c) {
  float r;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ bool is_odd(float top) {
  return (__float_as_uint(top) & 0x7FFFFFFFu) >= 0x7F800000u;
}

// The largest finite magnitude of N values (fp32 bits); odd: some are not finite.
template <int N>
__device__ __forceinline__ uint32_t f8_top(const uint32_t *v, bool &odd) {
  float m[2] = {0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < N; i += 2) {
    float &t = m[N > 4 ? i / 2 % 2 : 0];
    t = top3(t, __uint_as_float(v[i]), i + 1 < N ? __uint_as_float(v[i + 1]) : 0.0f);
  }
  m[0] = top3(m[0], m[1], 0.0f);
  odd = is_odd(m[0]);
  if (odd) {
    m[0] = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (!is_odd(__uint_as_float(v[i]))) m[0] = fmaxf(m[0], fabsf(__uint_as_float(v[i])));
  }
  return __float_as_uint(m[0]);
}

// Four codes of fp32 values (bits) times inv; ODD: infinities take the NaN code (y + 0 y).
template <bool ODD>
__device__ __forceinline__ uint32_t f8_codes4(const uint32_t *v, float inv) {
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; i += 2)
    unpack2(mul2(pack2(__uint_as_float(v[i]), __uint_as_float(v[i + 1])), both(inv)), y[i], y[i + 1]);
  if constexpr (ODD)
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = fmaf(y[i], 0.0f, y[i]);
  return f8_four(y[0], y[1], y[2], y[3]);
}

// A lane's 32 codes of its row (part h of the block's 128) in a box of 32 rows of 128 bytes with
// the 128-byte swizzle: no bank conflicts.
template <bool ODD>
__device__ __forceinline__ void f8_box_codes(uint8_t *box, int lane, int h, const uint32_t *v,
                                             float inv) {
#pragma unroll
  for (int k = 0; k < 2; ++k)
    *reinterpret_cast<uint4 *>(box + lane * 128 + (((2 * h + k) ^ (lane & 7)) << 4)) =
        make_uint4(f8_codes4<ODD>(v + 16 * k, inv), f8_codes4<ODD>(v + 16 * k + 4, inv),
                   f8_codes4<ODD>(v + 16 * k + 8, inv), f8_codes4<ODD>(v + 16 * k + 12, inv));
}
__device__ __forceinline__ void f8_put_box(uint8_t *box, int lane, int h, const uint32_t *v,
                                           float inv, bool odd) {
  if (__any_sync(0xffffffffu, odd)) f8_box_codes<true>(box, lane, h, v, inv);
  else f8_box_codes<false>(box, lane, h, v, inv);
}

// A barrier of the four warps that hold a quadrant's rows; true if any says so.
__device__ __forceinline__ bool f8_any(int quadrant, bool mine) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %2, 0;\n\t"
      "barrier.cta.red.or.pred q, %1, 128, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r)
      : "r"(quadrant + 1), "r"((uint32_t)mine)
      : "memory");
  return r != 0;
}

// The scale of a block of 128 columns from its four warps' maxima.
__device__ __forceinline__ uint32_t f8_block_scale(const uint32_t *tops, float &inv) {
  return f8_scale(max(max(tops[0], tops[BM]), max(tops[2 * BM], tops[3 * BM])), inv);
}

// A tile's sums of this warp's CW columns of g and of u, when they are there; false if they do
// not come.  The accumulator is handed back.
template <int NT, int CW, int ACCS, bool PAIR, bool FOLD>
__device__ __forceinline__ bool f8_gated_sums(const F8GatedArgs &g, const F8Item &t,
                                              uint32_t lane_base, uint64_t *accf, uint64_t *acce,
                                              volatile int *abort_flag, int lane, uint32_t &c,
                                              uint32_t (&v)[CW], uint32_t (&w)[CW]) {
  if constexpr (FOLD)
#pragma unroll
    for (int i = 0; i < CW; ++i) v[i] = w[i] = 0u;
  for (int kb = t.kb0; kb < t.kb1; kb = FOLD ? kb + g.chunk : t.kb1, ++c) {
    const int buf = c % ACCS;
    if (!f8_wait(&accf[buf], (c / ACCS) & 1u, g.status)) {
      *abort_flag = 1;
      return false;
    }
    tc_fence_after();
    const uint32_t from = lane_base + (uint32_t)(buf * NT);
    if constexpr (!FOLD) {
#pragma unroll
      for (int j = 0; j < CW; j += 32) {
        tmem_ld32_nw(from + j, *reinterpret_cast<uint32_t(*)[32]>(v + j));
        tmem_ld32_nw(from + NT / 2 + j, *reinterpret_cast<uint32_t(*)[32]>(w + j));
      }
#pragma unroll
      for (int j = 0; j < CW; j += 32) {
        tmem_wait_ld(*reinterpret_cast<uint32_t(*)[32]>(v + j));
        tmem_wait_ld(*reinterpret_cast<uint32_t(*)[32]>(w + j));
      }
    } else {
#pragma unroll
      for (int j = 0; j < 2 * CW; j += 16) {  // 16 columns at a time: registers
        uint32_t r[16];
        tmem_ld16_nw(from + (j < CW ? j : NT / 2 + j - CW), r);
        tmem_wait_ld(r);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          uint32_t &x = j < CW ? v[j + i] : w[j - CW + i];
          x = __float_as_uint(__uint_as_float(x) + __uint_as_float(r[i]));
        }
      }
    }
    tc_fence_before();
    __syncwarp();
    if (lane == 0) f8_release<PAIR>(&acce[buf]);
  }
  return true;
}

// v = act(v) w
template <int CW>
__device__ __forceinline__ void f8_form(int act, uint32_t (&v)[CW], const uint32_t (&w)[CW]) {
  with_act(act, [&](auto a) {
#pragma unroll
    for (int i = 0; i < CW; i += 2) {
      float x, y;
      unpack2(mul2(act2<a.value>(pack2(__uint_as_float(v[i]), __uint_as_float(v[i + 1]))),
                   pack2(__uint_as_float(w[i]), __uint_as_float(w[i + 1]))),
              x, y);
      v[i] = __float_as_uint(x), v[i + 1] = __float_as_uint(y);
    }
  });
}

// A warp's 32 rows x CW columns of the dense output, by way of its box.
template <int CW>
__device__ __forceinline__ void f8_put_dense(const F8Of<F8_GATED>::Maps &maps, const F8GatedArgs &g,
                                             float *box, int lane, int64_t m0, int64_t n,
                                             const uint32_t (&v)[CW]) {
#pragma unroll
  for (int j = 0; j < CW; j += 32) {
    const auto &x = *reinterpret_cast<const uint32_t(*)[32]>(v + j);
    if (g.boxes && g.bf16)
      f8_store_box<__nv_bfloat16>(g, &maps.out, box, lane, m0, n + j, x);
    else if (g.boxes)
      f8_store_box<float>(g, &maps.out, box, lane, m0, n + j, x);
    else if (g.bf16)
      f8_store_rows<__nv_bfloat16>(g, static_cast<__nv_bfloat16 *>(g.out), g.ldo, box, lane, m0,
                                   n + j, x);
    else
      f8_store_rows<float>(g, static_cast<float *>(g.out), g.ldo, box, lane, m0, n + j, x);
  }
}

// One super tile's (or tile's) accumulator holds g in its first half of columns and u in the
// others, for the same 128 hidden columns (64 in a narrow tile).  A warp takes half of them of
// both for its 32 rows (a lane a row), so a is formed in registers.  This one is for a dense
// output alone: its fewer warps hand the accumulator back sooner than 16 (8192 x 4096 x 1024: 47
// us, 2.9 PFLOP/s, and 54; an item's products take 4500 of the 5100 cycles from one to the next,
// its epilogue 3200 under them); and for tiles whose K blocks a cluster shares, with any outputs.
template <int NT, int ACCS, bool PAIR, bool FOLD>
__device__ __forceinline__ void f8_gated_dense(const F8Of<F8_GATED>::Maps &maps,
                                               const F8GatedArgs &g, uint32_t tmem, uint64_t *accf,
                                               uint64_t *acce, volatile int *abort_flag, float *box,
                                               float *part, int q, int h, int lane, int64_t first,
                                               int64_t step) {
  constexpr int CW = NT / 4;
  uint32_t c = 0;
  for (int64_t it = first; it < g.items && !*abort_flag; it += step) {
    const F8Item t = f8_item<NT, PAIR, uint32_t>(g, it);
    uint32_t v[CW], w[CW];  // g (then a) and u
    if (!f8_gated_sums<NT, CW, ACCS, PAIR, FOLD>(
            g, t, tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(h * CW), accf, acce, abort_flag,
            lane, c, v, w))
      break;
    if constexpr (!PAIR && NT == 256)
      if (g.splits > 1) {  // the products are done with the operand stages
        float *to = part + (q * 32 + lane) * (256 + 4) + h * CW;
#pragma unroll
        for (int i = 0; i < CW; i += 4) {
          *reinterpret_cast<uint4 *>(to + i) = make_uint4(v[i], v[i + 1], v[i + 2], v[i + 3]);
          *reinterpret_cast<uint4 *>(to + 128 + i) = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
        }
        break;
      }
    f8_form<CW>(g.act, v, w);
    f8_put_dense<CW>(maps, g, box, lane, t.m0 + q * 32, t.n0 / 2 + h * CW, v);
  }
  if (lane == 0) bulk_wait_all();
}

// With codes among the outputs a warp takes 32 columns, and a row's block of 128 is four
// lanes', which exchange their maxima through shared memory: g and u leave first, then a takes
// g's registers.  Codes leave by TMA in boxes of 32 rows x 128 bytes that a quadrant's four
// warps fill (straight from registers, 32 bytes a row, they took 90 us).  The warps meet at
// named barriers, for the maxima: what is in a box by then leaves after it, so a's codes leave
// in the next round.  Whatever makes one of the warps stop, all four leave the loop at the same
// barrier.  DENSE: a leaves densely as well.
//
// 8192 x 4096 x 1024: a's codes 50 us, those of a, g and u 59 (2.3 PFLOP/s), 67 with gelu, 62
// with gelu_tanh, where a dense output takes 47.  An item's products take 5000 cycles; this
// epilogue, next to them, 7000: 16 warps issue at 43% of the rate, waiting for their own
// arithmetic, the shared memory and one another.  Registers decide (96 a thread, 20 to 40 bytes
// of others spilled): with eight warps and twice the columns 78 us; sums taken all at once
// instead of 16 columns at a time 72, with more spilled; kernels without a dense output are
// without its code.  Maxima taken along with the sums, or 8 columns at a time while the next are
// on their way: 62; half of the reciprocals by Newton's iteration: no difference.
template <int ACCS, bool PAIR, bool DENSE>
__device__ __forceinline__ void f8_gated_codes(const F8Of<F8_GATED>::Maps &maps,
                                               const F8GatedArgs &g, uint32_t tmem, uint64_t *accf,
                                               uint64_t *acce, volatile int *abort_flag,
                                               uint8_t *boxes, uint32_t *tops, int q, int h,
                                               int lane, int64_t first, int64_t step) {
  const bool keeps = g.gate.codes || g.up.codes, makes = g.q.codes, leads = h == 0 && lane == 0;
  boxes += q * kF8QuadBoxes;
  // a warp's box of a dense output, where those of g and u have been
  [[maybe_unused]] float *dense = reinterpret_cast<float *>(boxes + h * kF8BoxBytes);
  constexpr size_t kBox = kF8QuadBoxes / 3;
  tops += q * 32 + lane;  // a row's maxima, tops[(slot * 4 + part) * 128]: g's, u's, a's, a's
  uint32_t c = 0, parity = 0;
  int32_t q_row = 0, q_col = -1;  // a's codes that have not left
  uint8_t *q_box = nullptr;
  bool bad = false;
  auto send_q = [&]() {
    if (leads && q_col >= 0 && q_row < g.M) {
      tma_store_2d(&maps.q, q_col, q_row, q_box);
      bulk_commit();
    }
    q_col = -1;
  };
  for (int64_t it = first; it < g.items; it += step, parity ^= 1u) {
    const F8Item t = f8_item<256, PAIR, uint32_t>(g, it);
    uint32_t v[32], w[32];  // g (then a) and u
    const bool ok = f8_gated_sums<256, 32, ACCS, PAIR, true>(
        g, t, tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(h * 32), accf, acce, abort_flag, lane,
        c, v, w);
    const int64_t m0 = t.m0 + q * 32, n0 = t.n0 / 2;
    const bool row = h == 0 && m0 + lane < g.M;
    const int64_t scale = scale_at(n0 / kF8Block, g.sp, m0 + lane);
    float inv;
    if (keeps) {
      bool odd_g, odd_u;
      tops[h * BM] = f8_top<32>(v, odd_g);
      tops[(4 + h) * BM] = f8_top<32>(w, odd_u);
      if ((odd_g && g.gate.codes) || (odd_u && g.up.codes)) record_status(g.status, FQT_ENONFINITE);
      if (lane == 0) bulk_wait_read(0);  // what left the boxes of g and u
      if ((bad = f8_any(q, !ok || *abort_flag))) break;
      send_q();
      if (g.gate.codes) {
        const uint32_t e = f8_block_scale(tops, inv);
        f8_put_box(boxes, lane, h, v, inv, odd_g);
        if (row) g.gate.scales[scale] = (uint8_t)e;
      }
      if (g.up.codes) {
        const uint32_t e = f8_block_scale(tops + 4 * BM, inv);
        f8_put_box(boxes + kBox, lane, h, w, inv, odd_u);
        if (row) g.up.scales[scale] = (uint8_t)e;
      }
      fence_proxy_async_smem();
    }
    f8_form<32>(g.act, v, w);
    // (two slots in turn: without g and u there is one barrier a round)
    uint32_t *top_a = tops + (8 + (keeps ? 0 : 4 * parity)) * BM;
    bool odd = false;
    if (makes) {
      top_a[h * BM] = f8_top<32>(v, odd);
      if (odd) record_status(g.status, FQT_ENONFINITE);
    }
    if (lane == 0) bulk_wait_read(0);  // what left a's box
    if ((bad = f8_any(q, !ok || *abort_flag))) break;
    if (!keeps) send_q();
    if (keeps && leads && m0 < g.M) {
      if (g.gate.codes) tma_store_2d(&maps.gate, (int32_t)n0, (int32_t)m0, boxes);
      if (g.up.codes) tma_store_2d(&maps.up, (int32_t)n0, (int32_t)m0, boxes + kBox);
      bulk_commit();
    }
    if constexpr (DENSE) {
      if (keeps) {  // not before they have left
        if (leads) bulk_wait_read(0);
        f8_any(q, false);
      }
      f8_put_dense<32>(maps, g, dense, lane, m0, n0 + h * 32, v);
    }
    if (makes) {
      // (alone, two boxes in turn: one may be leaving)
      q_box = boxes + (keeps || DENSE || parity ? 2 : 0) * kBox;
      q_row = (int32_t)m0;
      q_col = (int32_t)n0;
      const uint32_t e = f8_block_scale(top_a, inv);
      f8_put_box(q_box, lane, h, v, inv, odd);
      if (row) g.q.scales[scale] = (uint8_t)e;
      fence_proxy_async_smem();
      if (DENSE && !keeps) {
        f8_any(q, false);
        send_q();
      }
    }
  }
  if (!bad && makes) {
    f8_any(q, false);
    send_q();
  }
  if (lane == 0) bulk_wait_all();
}

// W consecutive entries of the shared memory of a cluster's CTA.
template <int W>
__device__ __forceinline__ void f8_remote(const float *p, int cta, uint32_t (&v)[W]) {
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(cta));
  if constexpr (W == 4)
    asm volatile("ld.shared::cluster.v4.b32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3])
                 : "r"(a)
                 : "memory");
  else if constexpr (W == 2)
    asm volatile("ld.shared::cluster.v2.b32 {%0, %1}, [%2];" : "=r"(v[0]), "=r"(v[1]) : "r"(a)
                 : "memory");
  else
    asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(v[0]) : "r"(a) : "memory");
}

// The sums over a cluster's K splits of W consecutive entries at p and at q, in their order
// (all on their way at once: one after the other, 1523 x 336 x 1201 took 12.4 us).
template <int W>
__device__ __forceinline__ void f8_parts(const float *p, const float *q, int cta, int step,
                                         int splits, uint32_t (&a)[W], uint32_t (&u)[W]) {
  if (splits == 1) {
    f8_remote<W>(p, cta, a);
    f8_remote<W>(q, cta, u);
    return;
  }
  uint32_t x[kF8Parts][W], y[kF8Parts][W];
#pragma unroll
  for (int k = 0; k < kF8Parts; ++k)
    if (k < splits) {
      f8_remote<W>(p, cta + k * step, x[k]);
      f8_remote<W>(q, cta + k * step, y[k]);
    }
#pragma unroll
  for (int i = 0; i < W; ++i) {
    float s = __uint_as_float(x[0][i]), t = __uint_as_float(y[0][i]);
#pragma unroll
    for (int k = 1; k < kF8Parts; ++k)
      if (k < splits) {
        s += __uint_as_float(x[k][i]);
        t += __uint_as_float(y[k][i]);
      }
    a[i] = __float_as_uint(s);
    u[i] = __float_as_uint(t);
  }
}

// A lane's four codes of a block of 128 columns that the warp holds.
__device__ __forceinline__ void f8_put_codes(const F8Codes &o, const F8GatedArgs &g, int64_t token,
                                             int64_t j, int64_t cols, const uint32_t (&v)[4],
                                             int lane) {
  if (!o.codes) return;
  bool odd;
  const uint32_t m = __reduce_max_sync(0xffffffffu, f8_top<4>(v, odd));
  if (odd) record_status(g.status, FQT_ENONFINITE);
  float inv;
  const uint32_t e = f8_scale(m, inv);
  // (rows of codes are whole 16 bytes)
  if (j < cols)
    *reinterpret_cast<uint32_t *>(o.codes + token * o.pitch + j) = f8_codes4<true>(v, inv);
  if (lane == 0) o.scales[scale_at(j / kF8Block, g.sp, token)] = (uint8_t)e;
}

// What is left to do where sums of g and u lie in the shared memory of a cluster's CTAs, which
// share a tile's K blocks (g.splits / g.holds of them) and, with few tokens, blocks of 128
// hidden columns (g.holds CTAs of g.part columns each).  A warp takes a token, a lane W of its
// 32 W columns.  With few tokens a token's sums lie in a row of 128 (g, then u), else in a row
// of 256 and four more (bank conflicts).  A token of 4096 x 1024: 5.3 us, with codes, for which
// four CTAs meet, 6.6; what a call of one K block takes is 5.
template <int W, bool FEW>
__device__ __forceinline__ void f8_gated_join(const F8GatedArgs &g, const float *part) {
  const int ctas = g.splits, self = (int)(blockIdx.x % (unsigned)ctas);
  const int holds = FEW ? g.holds : 1, splits = ctas / holds;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t cols = FEW ? g.M : g.N;
  int64_t t0 = 0, j = (int64_t)(blockIdx.x / (unsigned)ctas) * 32 * W, tokens = g.N;
  int pitch = BM, second = g.part, cta = 0, at = lane * W;
  if constexpr (FEW) {
    cta = at / g.part;
    at %= g.part;
  } else {
    const F8Item t = f8_item<256, false, uint32_t>(g, blockIdx.x);
    t0 = t.m0;
    j = t.n0 / 2;
    tokens = min((int64_t)BM, g.M - t0);
    pitch = 256 + 4;
    second = 128;
  }
  j += lane * W;
  for (int64_t r = self + ctas * warp; r < tokens; r += ctas * (kF8Threads / 32)) {
    uint32_t a[W], u[W];
    f8_parts<W>(part + r * pitch + at, part + r * pitch + second + at, cta, holds, splits, a, u);
    const int64_t token = t0 + r;
    if constexpr (W == 4) {
      f8_put_codes(g.gate, g, token, j, cols, a, lane);
      f8_put_codes(g.up, g, token, j, cols, u, lane);
    }
    with_act(g.act, [&](auto act) {
#pragma unroll
      for (int i = 0; i < W; ++i) {
        float x, unused;
        act_and_slope<act.value>(__uint_as_float(a[i]), x, unused);
        a[i] = __float_as_uint(__fmul_rn(x, __uint_as_float(u[i])));
      }
    });
    if (g.out) {
      const int64_t o = token * g.ldo + j;
#pragma unroll
      for (int i = 0; i < W; ++i)
        if (j + i < cols) {
          if (g.bf16)
            static_cast<__nv_bfloat16 *>(g.out)[o + i] = __float2bfloat16_rn(__uint_as_float(a[i]));
          else
            static_cast<float *>(g.out)[o + i] = __uint_as_float(a[i]);
        }
    }
    if constexpr (W == 4) f8_put_codes(g.q, g, token, j, cols, a, lane);
  }
}

template <int NT>
__device__ __forceinline__ void f8_gated_join(const F8GatedArgs &g, const float *part) {
  if constexpr (NT == 256) {
    f8_gated_join<4, false>(g, part);
  } else if constexpr (NT <= 64) {
    if (g.holds * g.part == kF8Block) f8_gated_join<4, true>(g, part);
    else if (g.part == 64) f8_gated_join<2, true>(g, part);
    else f8_gated_join<1, true>(g, part);
  }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
inline F8Codes codes_of(const fqt_fp8 *q) {
  return q ? F8Codes{q->codes, q->scales, q->pitch} : F8Codes{nullptr, nullptr, 0};
}

inline bool act_known(fqt_act act) { return act >= FQT_SILU && act <= FQT_SIGMOID; }

// An output of rows x cols codes: its pointers and its pitch; then its sizes.
inline bool codes_fit(const fqt_fp8 *q, int64_t rows, int64_t cols) {
  if (!q) return true;
  fqt_fp8 v = *q;
  v.rows = rows;
  v.cols = cols;
  return f8_good(&v);
}
inline void set_codes(fqt_fp8 *q, int64_t rows, int64_t cols) {
  if (!q) return;
  q->rows = rows;
  q->cols = cols;
  q->block_rows = 1;
}

}  // namespace fqt
