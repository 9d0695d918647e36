// fqt_gated.cuh -- the activations of a gated feed-forward block, and what its product
// kernel does with the sums of both projections.
#pragma once

#include <type_traits>

#include "fqt_fp8_core.cuh"

namespace fqt {

// ---------------------------------------------------------------------------
// Activations
// ---------------------------------------------------------------------------
// sigma(z) = 1 / (1 + 2^(-z log2 e)) by the hardware's base-2 exponential and reciprocal:
// the exponential's argument is rounded (relative error |z| 2^-24 of the result), they
// themselves are 2 units off; tanh.approx would leave 5e-4.
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
// arithmetic; found by reweighted least squares).  Unlike an approximation of erf, it loses no
// digits in the tail, and its factor e^(-x^2/2) is the density that the slope needs.  (With
// CUDA's normcdff 8192 x 4096 x 1024 took 139 us.)
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

// act(g) and act'(g).  1 - sigma is e^-z sigma where it is the slope's factor on its own
// (e^-z held below 2^126, so that neither loses digits where it is small); silu's slope is
// s + a (1 - s), which a rounded 1 - s does not harm.
template <int ACT>
__device__ __forceinline__ void act_and_slope(float g, float &a, float &d) {
  if constexpr (ACT == FQT_RELU) {
    a = g <= 0.0f ? 0.0f : g;  // NaN stays
    d = g > 0.0f ? 1.0f : 0.0f;
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
    const float t = exp2_of(fminf(__fmul_rn(z, -kLog2E), 126.0f));
    const float s = inverse_of(__fadd_rn(1.0f, t)), r = __fmul_rn(t, s);  // r = 1 - s
    if constexpr (ACT == FQT_SIGMOID) {
      a = s;
      d = __fmul_rn(s, r);
    } else {
      a = __fmul_rn(g, s);
      const float dz = __fmul_rn(kTanhScale, fmaf(__fmul_rn(3.0f * kTanhCube, c), c, 1.0f));
      d = fmaf(__fmul_rn(__fmul_rn(c, r), s), dz, s);
    }
    if (g != g) a = d = g;  // the limits take NaN away
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
// The right operand of a tile are 128 rows of the gate's weights and the same 128 of the up
// projection's (of a pair's CTAs, each loads one).  With few tokens the left operand are
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
    mbar_expect_tx(full, (uint32_t)(3 * kTileBytes));
    tma_load_2d(stage, &maps.a, k, m, full);
    tma_load_2d(stage + kTileBytes, &maps.b, k, n, full);
    tma_load_2d(stage + 2 * kTileBytes, &maps.b2, k, n, full);
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
    from = i < 8 ? g.sb : g.s2, pitch = g.spb, rows = g.N, r = t.n0 / 2 + 32 * (i & 3) + lane;
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
// The same of the numbers among them.
__device__ __forceinline__ float top3_number(float a, float b, float c) {
  float r;
  asm("max.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
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

// 64 columns of a warp's 32 rows as codes, by way of its box and TMA.
template <bool ODD>
__device__ __forceinline__ void f8_box_codes(float *box, int lane, const uint32_t *v, float inv) {
#pragma unroll
  for (int k = 0; k < 4; ++k)
    *reinterpret_cast<uint4 *>(box + box_off(lane, k) / 4) =
        make_uint4(f8_codes4<ODD>(v + 16 * k, inv), f8_codes4<ODD>(v + 16 * k + 4, inv),
                   f8_codes4<ODD>(v + 16 * k + 8, inv), f8_codes4<ODD>(v + 16 * k + 12, inv));
}

__device__ __forceinline__ void f8_store_codes(const CUtensorMap *map, float *&box, float *&spare,
                                               int lane, int64_t m0, int64_t n, const uint32_t *v,
                                               float inv, bool odd) {
  if (lane == 0) bulk_wait_read(1);  // all but the last store, from the other box, have read theirs
  __syncwarp();
  if (__any_sync(0xffffffffu, odd)) f8_box_codes<true>(box, lane, v, inv);
  else f8_box_codes<false>(box, lane, v, inv);
  fence_proxy_async_smem();
  __syncwarp();
  if (lane == 0) {
    tma_store_2d(map, (int32_t)n, (int32_t)m0, box);
    bulk_commit();
  }
  float *const used = box;
  box = spare;
  spare = used;
}

// A barrier of the two warps that hold a quadrant's rows; true if either says so.
__device__ __forceinline__ bool f8_either(int quadrant, bool mine) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %2, 0;\n\t"
      "barrier.cta.red.or.pred q, %1, 64, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r)
      : "r"(quadrant + 1), "r"((uint32_t)mine)
      : "memory");
  return r != 0;
}

// One super tile's (or tile's) accumulator holds g in its first 128 columns and u in the
// others, for the same 128 hidden columns.  A warp takes 64 columns of both for its 32 rows
// (a lane a row), so a is formed in registers, and a row's block of 128 is two lanes' 64,
// which exchange their maxima through shared memory.  g and u leave first, then a takes g's
// registers.  Both warps of a quadrant leave the loop together, whatever made one of them
// stop: they meet at named barriers.
template <int ACCS, bool PAIR, bool FOLD>
__device__ __forceinline__ void f8_gated_epilogue(const F8Of<F8_GATED>::Maps &maps,
                                                  const F8GatedArgs &g, uint32_t tmem,
                                                  uint64_t *accf, uint64_t *acce,
                                                  volatile int *abort_flag, float *box,
                                                  uint32_t *tops, int q, int h, int lane,
                                                  int64_t first, int64_t step) {
  constexpr int NT = 256;
  const uint32_t lane_base = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(h * 64);
  const bool keeps = g.gate.codes || g.up.codes, codes = keeps || g.q.codes;
  // of a row's halves: tops[(tensor * 2 + half) * 128 + row]
  float *spare = box + (g.boxes_each - 1) * (kF8BoxBytes / 4);
  uint32_t *mine = tops + h * 128 + q * 32 + lane, *other = tops + (1 - h) * 128 + q * 32 + lane;
  uint32_t c = 0;
  for (int64_t it = first; it < g.items; it += step) {
    if (codes ? f8_either(q, *abort_flag) : *abort_flag) break;
    const F8Item t = f8_item<NT, PAIR>(g, it);
    uint32_t v[4][32];  // 64 columns of g, 64 of u
    bool ok = true;
    if constexpr (FOLD)
#pragma unroll
      for (int i = 0; i < 128; ++i) v[i / 32][i % 32] = 0u;
    for (int kb = t.kb0; kb < t.kb1; kb = FOLD ? kb + g.chunk : t.kb1, ++c) {
      const int buf = c % ACCS;
      if (!f8_wait(&accf[buf], (c / ACCS) & 1u, g.status)) {
        *abort_flag = 1;
        ok = false;
        break;
      }
      tc_fence_after();
      const uint32_t from = lane_base + (uint32_t)(buf * NT);
      if constexpr (!FOLD) {
#pragma unroll
        for (int p = 0; p < 4; ++p) tmem_ld32_nw(from + (p >> 1) * 128 + (p & 1) * 32, v[p]);
#pragma unroll
        for (int p = 0; p < 4; ++p) tmem_wait_ld(v[p]);
      } else {
#pragma unroll
        for (int j = 0; j < 128; j += 16) {  // 16 columns at a time: registers
          uint32_t r[16];
          tmem_ld16_nw(from + (j >> 6) * 128 + (j & 63), r);
          tmem_wait_ld(r);
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            uint32_t &x = v[j / 32][j % 32 + i];
            x = __float_as_uint(__uint_as_float(x) + __uint_as_float(r[i]));
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) f8_release<PAIR>(&acce[buf]);
    }
    const int64_t m0 = t.m0 + q * 32, n0 = t.n0 / 2, n = n0 + h * 64;
    const bool row = m0 + lane < g.M;
    bool odd_g = false, odd_u = false, odd_a = false;
    if (keeps) {
      const uint32_t mg = f8_top<64>(v[0], odd_g), mu = f8_top<64>(v[2], odd_u);
      if ((odd_g && g.gate.codes) || (odd_u && g.up.codes)) record_status(g.status, FQT_ENONFINITE);
      mine[0] = mg;
      mine[256] = mu;
      if (f8_either(q, !ok)) break;
      float ig, iu;
      const uint32_t eg = f8_scale(max(mg, other[0]), ig), eu = f8_scale(max(mu, other[256]), iu);
      if (g.gate.codes) {
        if (m0 < g.M && n < g.N)
          f8_store_codes(&maps.gate, box, spare, lane, m0, n, v[0], ig, odd_g);
        if (row && h == 0) g.gate.scales[scale_at(n0 / kF8Block, g.sp, m0 + lane)] = (uint8_t)eg;
      }
      if (g.up.codes) {
        if (m0 < g.M && n < g.N)
          f8_store_codes(&maps.up, box, spare, lane, m0, n, v[2], iu, odd_u);
        if (row && h == 0) g.up.scales[scale_at(n0 / kF8Block, g.sp, m0 + lane)] = (uint8_t)eu;
      }
    }
    if (!codes && !ok) break;
    with_act(g.act, [&](auto act) {
#pragma unroll
      for (int i = 0; i < 64; i += 2) {
        uint32_t *x = &v[i / 32][i % 32], *y = &v[2 + i / 32][i % 32];
        float p, q;
        unpack2(mul2(act2<act.value>(pack2(__uint_as_float(x[0]), __uint_as_float(x[1]))),
                     pack2(__uint_as_float(y[0]), __uint_as_float(y[1]))),
                p, q);
        x[0] = __float_as_uint(p), x[1] = __float_as_uint(q);
      }
    });
    if (g.out && ok) {
      if (!g.boxes && lane == 0) bulk_wait_read(0);  // (the box is written without asking)
      float *fp32 = static_cast<float *>(g.out);
      __nv_bfloat16 *bf16 = static_cast<__nv_bfloat16 *>(g.out);
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const int64_t np = n + 32 * p;
        if (g.boxes && g.bf16)
          f8_store_box<__nv_bfloat16>(g, &maps.out, box, lane, m0, np, v[p]);
        else if (g.boxes)
          f8_store_box<float>(g, &maps.out, box, lane, m0, np, v[p]);
        else if (g.bf16)
          f8_store_rows<__nv_bfloat16>(g, bf16, g.ldo, box, lane, m0, np, v[p]);
        else
          f8_store_rows<float>(g, fp32, g.ldo, box, lane, m0, np, v[p]);
      }
      float *const used = box;
      box = spare;
      spare = used;
    }
    if (g.q.codes) {
      const uint32_t ma = f8_top<64>(v[0], odd_a);
      if (odd_a) record_status(g.status, FQT_ENONFINITE);
      mine[512] = ma;
      if (f8_either(q, !ok)) break;
      float ia;
      const uint32_t ea = f8_scale(max(ma, other[512]), ia);
      if (m0 < g.M && n < g.N)
        f8_store_codes(&maps.q, box, spare, lane, m0, n, v[0], ia, odd_a);
      if (row && h == 0) g.q.scales[scale_at(n0 / kF8Block, g.sp, m0 + lane)] = (uint8_t)ea;
    }
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

// W consecutive codes of lane's values, whose block (the warp's) has the maximum m.
template <int W>
__device__ __forceinline__ void f8_put_codes(const F8Codes &o, const F8GatedArgs &g, int64_t token,
                                             int64_t j, const uint32_t (&v)[W], int lane) {
  static_assert(W == 4, "a block of 128 entries is a warp's");
  if (!o.codes) return;
  bool odd;
  const uint32_t m = __reduce_max_sync(0xffffffffu, f8_top<W>(v, odd));
  if (odd) record_status(g.status, FQT_ENONFINITE);
  float inv;
  const uint32_t e = f8_scale(m, inv);
  // (rows of codes are whole 16 bytes)
  if (j < g.M)
    *reinterpret_cast<uint32_t *>(o.codes + token * o.pitch + j) = f8_codes4<true>(v, inv);
  if (lane == 0) o.scales[scale_at(j / kF8Block, g.sp, token)] = (uint8_t)e;
}

// Few tokens: g and u of this CTA's hidden columns (g.part each) lie in its shared memory,
// a token's 128 sums in a row (g, then u).  The CTAs of a cluster hold the 32 W columns of
// whole blocks; a warp takes a token, a lane W columns.
template <int W>
__device__ __forceinline__ void f8_gated_join(const F8GatedArgs &g, const float *part) {
  const int parts = 32 * W / g.part, self = (int)(blockIdx.x % parts);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t j = (int64_t)(blockIdx.x / parts) * 32 * W + lane * W;
  const int cta = lane * W / g.part, at = lane * W % g.part;
  for (int64_t token = self + parts * warp; token < g.N; token += parts * (kF8Threads / 32)) {
    uint32_t a[W], u[W];
    f8_remote<W>(part + token * BM + at, cta, a);
    f8_remote<W>(part + token * BM + g.part + at, cta, u);
    if constexpr (W == 4) {
      f8_put_codes<W>(g.gate, g, token, j, a, lane);
      f8_put_codes<W>(g.up, g, token, j, u, lane);
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
        if (j + i < g.M) {
          if (g.bf16)
            static_cast<__nv_bfloat16 *>(g.out)[o + i] = __float2bfloat16_rn(__uint_as_float(a[i]));
          else
            static_cast<float *>(g.out)[o + i] = __uint_as_float(a[i]);
        }
    }
    if constexpr (W == 4) f8_put_codes<W>(g.q, g, token, j, a, lane);
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

// No two outputs in the same place.
template <int N>
inline bool all_apart(const fqt_fp8 *const (&q)[N]) {
  for (int i = 0; i < N; ++i)
    for (int j = i + 1; j < N; ++j)
      if (q[i] && q[j] && (q[i]->codes == q[j]->codes || q[i]->scales == q[j]->scales)) return false;
  return true;
}

}  // namespace fqt
