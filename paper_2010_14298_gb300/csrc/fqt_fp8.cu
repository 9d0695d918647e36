// fqt_fp8.cu -- matrix products of 8-bit floating-point codes (E4M3) with one
// scale for each block of 128 entries along the contraction, and their quantizer.
//
//   out_mn = sum_kb sa[kb][m] sb[kb][n] sum_(k in block kb) a_mk b_nk
//
// The inner sum of a block runs on the tensor cores (tcgen05 kind::f8f6f4, products
// exact, fp32 accumulators in tensor memory); the scales belong to blocks, so each
// block's sums are read back, multiplied by their two scales and added to fp32
// running sums in registers: 128 sums a thread, two accumulators in tensor memory in
// turn, so that the fold of one block overlaps the next block's products.
#include <cuda_runtime.h>
#include <math.h>

#include "fqt.h"
#include "fqt_common.cuh"
#include "fqt_gemm_core.cuh"
#include "fqt_internal.h"

namespace fqt {

constexpr int kF8Block = 128;  // entries per scale along the contraction (= bytes of a K block)
constexpr int64_t kF8MaxSize = 1 << 22;  // of any dimension (32768 blocks: a grid's y)

// ---------------------------------------------------------------------------
// Quantizer
// ---------------------------------------------------------------------------
// A block's scale 2^e: the least power of two for which amax <= 448 2^e (448 =
// 1.75 2^8, E4M3's largest value), e in [-127, 127]; e = 0 for a block of zeros.
// Division by it is exact, so a code is one rounding of the entry (to nearest, ties
// to even) in any arithmetic, and the value code 2^e is exact in fp32.  amax as
// fp32 bits; returns e.
__device__ __forceinline__ int f8_exponent(uint32_t amax) {
  if (amax == 0u) return 0;
  const int e = (int)(amax >> 23) - 127 - 8 + ((amax & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return max(e, -127);  // subnormal amax too
}
__device__ __forceinline__ float pow2(int e) {  // -127 <= e <= 127
  return __uint_as_float(e > -127 ? (uint32_t)(e + 127) << 23 : 1u << 22);
}

// Codes of two values (lo, hi in the low and high byte), |.| <= 448 or NaN.
__device__ __forceinline__ uint32_t f8_pair(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}

struct F8QuantArgs {
  const void *x;
  int64_t ldx, rows;
  int cols;
  uint8_t *c, *ct;  // codes by rows, and of the transpose (either may be null)
  int64_t pitch, pitch_t;
  float *s, *st;  // scales [column block][row], [row block][column]
  int64_t sp, spt;
  int whole;  // one scale for the 128 x 128 block
  int *status;
};

constexpr int kF8Pitch = kF8Block + 16;  // bytes of a transposed row in shared memory

// One CTA per 128 x 128 tile.  A thread holds 8 rows x 8 columns of it, so it packs
// codes along either axis without exchanging bytes: 8 bytes of each of its rows go
// straight to memory, 8 bytes of each of its columns through shared memory.  Bound by
// memory traffic: the entries are read once for both outputs.
template <typename T>
__global__ void __launch_bounds__(256) k_f8_quant(const F8QuantArgs a, const bool vec) {
  __shared__ uint32_t cmax[8][kF8Block];
  __shared__ __align__(16) uint8_t tr[kF8Block * kF8Pitch];
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  const int cg = t & 15, rg = t >> 4;  // its 8 columns and its 8 rows
  const int64_t r0 = (int64_t)blockIdx.y * kF8Block;
  const int64_t c0 = (int64_t)blockIdx.x * kF8Block;
  const int64_t row = r0 + rg * 8, col = c0 + cg * 8;
  float v[8][8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const T *p = static_cast<const T *>(a.x) + (row + i) * a.ldx + col;
    if (row + i < a.rows && vec && col + 8 <= a.cols) {
      load_oct(p, v[i]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        v[i][j] = row + i < a.rows && col + j < a.cols ? (float)p[j] : 0.0f;
    }
  }
  uint32_t top = 0u;
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(v[i][j]) & 0x7FFFFFFFu);
  // entries that are no numbers count for no scale and take the NaN code
  const bool bad = top >= 0x7F800000u;
  if (bad) {
    record_status(a.status, FQT_ENONFINITE);
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (!isfinite(v[i][j])) v[i][j] = __uint_as_float(0x7FFFFFFFu);
  }
  auto mag = [&](float x) {
    const uint32_t m = __float_as_uint(x) & 0x7FFFFFFFu;
    return m < 0x7F800000u ? m : 0u;
  };
  // row maxima: over the 16 threads of a row; column maxima: over the two row groups
  // of a warp, then over the warps
  uint32_t rm[8], cm[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) rm[i] = cm[i] = 0u;
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t m = mag(v[i][j]);
      rm[i] = max(rm[i], m);
      cm[j] = max(cm[j], m);
    }
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) rm[i] = max(rm[i], __shfl_xor_sync(0xffffffffu, rm[i], o));
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    cm[j] = max(cm[j], __shfl_xor_sync(0xffffffffu, cm[j], 16));
    if (lane < 16) cmax[warp][cg * 8 + j] = cm[j];
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < 8; ++j)
#pragma unroll
    for (int w = 0; w < 8; ++w) cm[j] = max(cm[j], cmax[w][cg * 8 + j]);
  if (a.whole) {
    uint32_t m = 0u;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, cm[j]);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
#pragma unroll
    for (int i = 0; i < 8; ++i) rm[i] = cm[i] = m;
  }
  if (a.c) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int e = f8_exponent(rm[i]);
      if (cg == 0) a.s[blockIdx.x * a.sp + row + i] = row + i < a.rows ? pow2(e) : 0.0f;
      if (row + i >= a.rows || col >= a.cols) continue;
      const float inv = pow2(-e);
      uint32_t w[2];
#pragma unroll
      for (int h = 0; h < 2; ++h)
        w[h] = f8_pair(v[i][4 * h] * inv, v[i][4 * h + 1] * inv) |
               f8_pair(v[i][4 * h + 2] * inv, v[i][4 * h + 3] * inv) << 16;
      *reinterpret_cast<uint2 *>(a.c + (row + i) * a.pitch + col) = make_uint2(w[0], w[1]);
    }
  }
  if (a.ct) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int e = f8_exponent(cm[j]);
      if (rg == 0) a.st[blockIdx.y * a.spt + col + j] = col + j < a.cols ? pow2(e) : 0.0f;
      const float inv = pow2(-e);
      uint32_t w[2];
#pragma unroll
      for (int h = 0; h < 2; ++h)
        w[h] = f8_pair(v[4 * h][j] * inv, v[4 * h + 1][j] * inv) |
               f8_pair(v[4 * h + 2][j] * inv, v[4 * h + 3][j] * inv) << 16;
      *reinterpret_cast<uint2 *>(tr + (cg * 8 + j) * kF8Pitch + rg * 8) = make_uint2(w[0], w[1]);
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int at = k * 256 + t, j = at >> 3, ch = at & 7;
      if (c0 + j < a.cols && r0 + ch * 16 < a.rows)
        *reinterpret_cast<uint4 *>(a.ct + (c0 + j) * a.pitch_t + r0 + ch * 16) =
            *reinterpret_cast<const uint4 *>(tr + j * kF8Pitch + ch * 16);
    }
  }
}

// ---------------------------------------------------------------------------
// Product
// ---------------------------------------------------------------------------
constexpr int kF8EpiWarps = 8, kF8Epi0 = 4;  // warps 0 loads, 1 products, 2 scales, 3 none
constexpr int kF8Threads = 32 * (kF8Epi0 + kF8EpiWarps);
constexpr int kF8RegsCtl = 64, kF8RegsEpi = 216;
static_assert(128 * kF8RegsCtl + 256 * kF8RegsEpi <= kF8Threads * ((65536 / kF8Threads) / 8 * 8),
              "register shares exceed the launch's");
constexpr int kF8Slots = 8;             // K blocks of scales in shared memory
constexpr size_t kF8SlotBytes = 1536;   // 128 of A, up to 256 of B
constexpr size_t kF8OffBar = kF8Slots * kF8SlotBytes;
constexpr size_t kF8Bars = 2 * kMaxStages + 4 + 2 * kF8Slots + 1;
constexpr size_t kF8Fixed = (kF8OffBar + kF8Bars * 8 + 16 + 1023) & ~(size_t)1023;

struct F8Args {
  const float *sa, *sb;  // scales, K blocks spa / spb entries apart
  int64_t spa, spb;
  int64_t M, N;  // rows of A and of B
  int nkb;       // K blocks
  int m_tiles, n_tiles, splits, kb_per;
  int64_t items;
  void *out;
  int64_t ldo;
  int bf16, swap;  // swap: out is indexed [B row][A row]
  float *part;     // splits > 1: fp32 partial outputs, one after another
  int stages;
  int b_whole;  // B's scale is one for 128 rows
  int *status;
};

__device__ __forceinline__ void bulk_load(void *dst, const void *src, uint32_t bytes,
                                          uint64_t *bar) {
  asm volatile(
      "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::
          "r"(smem_u32(dst)),
      "l"(src), "r"(bytes), "r"(smem_u32(bar))
      : "memory");
}

__device__ __forceinline__ void f8_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc,
                                       uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}

struct F8Item {
  int64_t m0, n0;
  int kb0, kb1, split;
};

template <int NT>
__device__ __forceinline__ F8Item f8_item(const F8Args &g, int64_t it) {
  F8Item t;
  const int64_t tiles = (int64_t)g.m_tiles * g.n_tiles;
  t.split = (int)(it / tiles);
  const int64_t r = it - t.split * tiles;
  const int64_t n = r / g.m_tiles;
  t.n0 = n * NT;
  t.m0 = (r - n * g.m_tiles) * BM;
  t.kb0 = t.split * g.kb_per;
  t.kb1 = min(g.nkb, t.kb0 + g.kb_per);
  return t;
}

template <typename T>
__device__ __forceinline__ T f8_out(float v) {
  if constexpr (sizeof(T) == 4) return v;
  else return __float2bfloat16_rn(v);
}

// This thread's W sums: row m of the tile's rows, columns n .. n + W - 1.
template <typename T, int W>
__device__ __forceinline__ void f8_store(const F8Args &g, T *out, int64_t ld, int64_t m,
                                         int64_t n, const f32x2 (&acc)[W / 2]) {
  if (m >= g.M) return;
  if (g.swap) {
#pragma unroll
    for (int j = 0; j < W / 2; ++j) {
      float u, v;
      unpack2(acc[j], u, v);
      if (n + 2 * j < g.N) out[(n + 2 * j) * ld + m] = f8_out<T>(u);
      if (n + 2 * j + 1 < g.N) out[(n + 2 * j + 1) * ld + m] = f8_out<T>(v);
    }
    return;
  }
  T *p = out + m * ld + n;
  constexpr int E = 16 / sizeof(T);
  const bool vec = (reinterpret_cast<uintptr_t>(p) & 15) == 0;
#pragma unroll
  for (int j = 0; j < W; j += E) {
    float v[E];
#pragma unroll
    for (int i = 0; i < E; i += 2) unpack2(acc[(j + i) / 2], v[i], v[i + 1]);
    if (vec && n + j + E <= g.N) {
      if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<float4 *>(p + j) = make_float4(v[0], v[1], v[2], v[3]);
      } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
          w[i] = *reinterpret_cast<const uint32_t *>(&b);
        }
        *reinterpret_cast<uint4 *>(p + j) = make_uint4(w[0], w[1], w[2], w[3]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (n + j + i < g.N) p[j + i] = f8_out<T>(v[i]);
    }
  }
}

// One CTA per 128 x NT tile (and split of the K blocks), persistent.  Warp 0 feeds
// operand stages of one K block by TMA, warp 1 issues a K block's four products into
// one of two accumulators, warp 2 feeds the blocks' scales; the eight epilogue warps
// (quadrant of rows x half of the columns) fold each K block into their sums.
template <int NT>
__global__ void __launch_bounds__(kF8Threads, 1)
    k_f8_mm(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
            const F8Args g) {
  constexpr int W = NT / 2;  // columns of an epilogue warp
  constexpr uint32_t kStage = (uint32_t)(kTileBytes + NT * kF8Block);
  constexpr uint32_t kCols = 2 * NT < 32 ? 32 : 2 * NT;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint64_t *full = reinterpret_cast<uint64_t *>(smem + kF8OffBar), *empty = full + kMaxStages;
  uint64_t *accf = empty + kMaxStages, *acce = accf + 2;
  uint64_t *sfull = acce + 2, *sempty = sfull + kF8Slots, *drain = sempty + kF8Slots;
  uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(full + kF8Bars);
  volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
  uint8_t *ops = smem + kF8Fixed;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < g.stages; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&accf[i], 1);
      mbar_init(&acce[i], kF8EpiWarps);
    }
    for (int i = 0; i < kF8Slots; ++i) {
      mbar_init(&sfull[i], 1);
      mbar_init(&sempty[i], kF8EpiWarps);
    }
    mbar_init(drain, 1);
    *abort_flag = 0;
    fence_barrier_init();
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                     smem_u32(tmem_slot)),
                 "r"(kCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  if (warp >= kF8Epi0) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kF8RegsEpi));
    const int q = warp & 3, h = (warp - kF8Epi0) >> 2;
    const uint32_t lane_base = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(h * W);
    uint32_t c = 0;  // K blocks so far
    bool ok = true;
    for (int64_t it = blockIdx.x; ok && it < g.items && !*abort_flag; it += gridDim.x) {
      const F8Item t = f8_item<NT>(g, it);
      f32x2 acc[W / 2];
#pragma unroll
      for (int j = 0; j < W / 2; ++j) acc[j] = pack2(0.0f, 0.0f);
      for (int kb = t.kb0; kb < t.kb1; ++kb, ++c) {
        const int slot = c % kF8Slots, buf = c & 1;
        if (!mbar_wait(&sfull[slot], (c / kF8Slots) & 1u, g.status) ||
            !mbar_wait(&accf[buf], (c >> 1) & 1u, g.status)) {
          *abort_flag = 1;
          ok = false;
          break;
        }
        tc_fence_after();
        const float *sc = reinterpret_cast<const float *>(smem + slot * kF8SlotBytes);
        const float sa = sc[q * 32 + lane];
        const float *sb = sc + BM + h * W;
        const float s1 = sa * sb[0];
        const f32x2 s2 = pack2(s1, s1), sa2 = pack2(sa, sa);
        constexpr int CH = W < 32 ? W : 32;
#pragma unroll
        for (int j = 0; j < W; j += CH) {
          uint32_t r[CH];
          tmem_ldw_nw<CH>(lane_base + (uint32_t)(buf * NT + j), r);
          tmem_wait_ld(r);
          if (g.b_whole) {
#pragma unroll
            for (int i = 0; i < CH; i += 2)
              acc[(j + i) / 2] = fma2(pack2(__uint_as_float(r[i]), __uint_as_float(r[i + 1])), s2,
                                      acc[(j + i) / 2]);
          } else {
#pragma unroll
            for (int i = 0; i < CH; i += 4) {
              const float4 b = *reinterpret_cast<const float4 *>(sb + j + i);
              acc[(j + i) / 2] = fma2(pack2(__uint_as_float(r[i]), __uint_as_float(r[i + 1])),
                                      mul2(sa2, pack2(b.x, b.y)), acc[(j + i) / 2]);
              acc[(j + i) / 2 + 1] =
                  fma2(pack2(__uint_as_float(r[i + 2]), __uint_as_float(r[i + 3])),
                       mul2(sa2, pack2(b.z, b.w)), acc[(j + i) / 2 + 1]);
            }
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&acce[buf]);
          mbar_arrive(&sempty[slot]);
        }
      }
      if (!ok) break;
      const int64_t m = t.m0 + q * 32 + lane, n = t.n0 + h * W;
      if (g.splits > 1) {
        f8_store<float, W>(g, g.part + t.split * g.M * g.N, g.swap ? g.M : g.N, m, n, acc);
      } else if (g.bf16) {
        f8_store<__nv_bfloat16, W>(g, static_cast<__nv_bfloat16 *>(g.out), g.ldo, m, n, acc);
      } else {
        f8_store<float, W>(g, static_cast<float *>(g.out), g.ldo, m, n, acc);
      }
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kF8RegsCtl));
    if (warp == 0 && lane == 0) {
      int s = 0;
      uint32_t ph = 0;
      bool ok = true;
      for (int64_t it = blockIdx.x; ok && it < g.items && !*abort_flag; it += gridDim.x) {
        const F8Item t = f8_item<NT>(g, it);
        for (int kb = t.kb0; kb < t.kb1; ++kb) {
          if (!mbar_wait(&empty[s], ph ^ 1u, g.status)) {
            *abort_flag = 1;
            ok = false;
            break;
          }
          mbar_expect_tx(&full[s], kStage);
          uint8_t *st = ops + (size_t)s * kStage;
          tma_load_2d(st, &tmA, kb * kF8Block, (int32_t)t.m0, &full[s]);
          tma_load_2d(st + kTileBytes, &tmB, kb * kF8Block, (int32_t)t.n0, &full[s]);
          if (++s == g.stages) { s = 0; ph ^= 1u; }
        }
      }
      // every load has landed before the CTA exits
      if (*abort_flag) {
        sleep_ns(200000);
      } else {
        for (int i = 0; i < g.stages; ++i) {
          if (!mbar_wait(&empty[s], ph ^ 1u, g.status)) break;
          if (++s == g.stages) { s = 0; ph ^= 1u; }
        }
      }
    } else if (warp == 1 && lane == 0) {
      int s = 0;
      uint32_t ph = 0, c = 0;
      bool ok = true;
      // D fp32; A, B E4M3 (format 0), both K-major
      constexpr uint32_t idesc =
          (1u << 4) | ((uint32_t)(NT >> 3) << 17) | ((uint32_t)(BM >> 4) << 24);
      for (int64_t it = blockIdx.x; ok && it < g.items && !*abort_flag; it += gridDim.x) {
        const F8Item t = f8_item<NT>(g, it);
        for (int kb = t.kb0; kb < t.kb1; ++kb, ++c) {
          const int buf = c & 1;
          if (!mbar_wait(&acce[buf], ((c >> 1) & 1u) ^ 1u, g.status) ||
              !mbar_wait(&full[s], ph, g.status)) {
            *abort_flag = 1;
            ok = false;
            break;
          }
          tc_fence_after();
          const uint32_t a_addr = smem_u32(ops + (size_t)s * kStage);
          const uint64_t da = sw128_desc(a_addr), db = sw128_desc(a_addr + (uint32_t)kTileBytes);
#pragma unroll
          for (int k = 0; k < 4; ++k)  // 32 entries each
            f8_mma(tmem + (uint32_t)(buf * NT), da + 2 * k, db + 2 * k, idesc, k > 0 ? 1u : 0u);
          umma_commit(&empty[s]);
          umma_commit(&accf[buf]);
          if (++s == g.stages) { s = 0; ph ^= 1u; }
        }
      }
      // every product has completed before tensor memory is released
      umma_commit(drain);
      mbar_wait(drain, 0, g.status);
    } else if (warp == 2 && lane == 0) {
      uint32_t c = 0;
      bool ok = true;
      for (int64_t it = blockIdx.x; ok && it < g.items && !*abort_flag; it += gridDim.x) {
        const F8Item t = f8_item<NT>(g, it);
        const int64_t left = g.spb - t.n0;
        const uint32_t nb = (uint32_t)(left < NT ? left : NT) * 4u;
        for (int kb = t.kb0; kb < t.kb1; ++kb, ++c) {
          const int slot = c % kF8Slots;
          if (!mbar_wait(&sempty[slot], ((c / kF8Slots) & 1u) ^ 1u, g.status)) {
            *abort_flag = 1;
            ok = false;
            break;
          }
          uint8_t *dst = smem + slot * kF8SlotBytes;
          mbar_expect_tx(&sfull[slot], BM * 4u + nb);
          bulk_load(dst, g.sa + kb * g.spa + t.m0, BM * 4u, &sfull[slot]);
          bulk_load(dst + BM * 4, g.sb + kb * g.spb + t.n0, nb, &sfull[slot]);
        }
      }
      if (*abort_flag) {
        sleep_ns(200000);
      } else {
        for (int i = 0; i < kF8Slots; ++i, ++c)
          if (!mbar_wait(&sempty[c % kF8Slots], ((c / kF8Slots) & 1u) ^ 1u, g.status)) break;
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kCols)
                 : "memory");
  }
}

// The sum of the splits' partial outputs, in their order.
template <typename T>
__global__ void __launch_bounds__(256)
    k_f8_join(const float *part, int splits, int64_t rows, int64_t cols, T *out, int64_t ldo) {
  const int64_t n = rows * cols;
  for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n;
       i += (int64_t)gridDim.x * blockDim.x) {
    float s = 0.0f;
    for (int k = 0; k < splits; ++k) s += __ldg(part + k * n + i);
    const int64_t r = i / cols;
    out[r * ldo + (i - r * cols)] = f8_out<T>(s);
  }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
static bool make_map_codes(CUtensorMap *m, const fqt_fp8 *q, uint32_t box_rows) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[2] = {(cuuint64_t)q->cols, (cuuint64_t)q->rows};
  cuuint64_t strides[1] = {(cuuint64_t)q->pitch};
  cuuint32_t box[2] = {kF8Block, box_rows};
  cuuint32_t es[2] = {1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, q->codes, dims, strides, box, es,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// How a product of M x N outputs over nkb K blocks is cut into tiles.
struct F8Plan {
  bool swap;  // A is the right operand, out is written transposed
  int nt, m_tiles, n_tiles, splits, kb_per;
};

static F8Plan f8_plan(int64_t M, int64_t N, int64_t nkb, int nsm) {
  F8Plan p;
  // few rows: they become the narrow side, and the other operand fills the 128 rows
  p.swap = M <= 64;
  const int64_t a = p.swap ? N : M, b = p.swap ? M : N;
  p.m_tiles = (int)((a + BM - 1) / BM);
  if (p.swap) {
    p.nt = b <= 32 ? 32 : 64;
  } else {
    // 256 columns where the tiles fill the SMs, else 128
    p.nt = (int64_t)p.m_tiles * ((b + 255) / 256) >= nsm ? 256 : 128;
  }
  p.n_tiles = (int)((b + p.nt - 1) / p.nt);
  const int64_t tiles = (int64_t)p.m_tiles * p.n_tiles;
  // fewer tiles than SMs: the contraction is split, at least 4 K blocks each
  int64_t splits = tiles < nsm ? nsm / tiles : 1;
  if (splits > nkb / 4) splits = nkb / 4;
  if (splits > 16) splits = 16;
  if (splits < 1) splits = 1;
  p.kb_per = (int)((nkb + splits - 1) / splits);
  p.splits = (int)((nkb + p.kb_per - 1) / p.kb_per);
  return p;
}

size_t fp8_matmul_ws_bytes(int64_t M, int64_t N, int64_t K) {
  if (M <= 0 || N <= 0 || K <= 0) return kHeaderBytes;
  const F8Plan p = f8_plan(M, N, (K + kF8Block - 1) / kF8Block, device_sm_count());
  return kHeaderBytes + (p.splits > 1 ? (size_t)p.splits * M * N * sizeof(float) : 0);
}

template <int NT>
static fqt_status launch_f8(const CUtensorMap &ta, const CUtensorMap &tb, F8Args &g, int nsm,
                            cudaStream_t st) {
  constexpr size_t stage = kTileBytes + NT * kF8Block;
  constexpr size_t room = 227 * 1024 - 1024 - kF8Fixed;
  constexpr int stages = room / stage < kMaxStages ? (int)(room / stage) : kMaxStages;
  constexpr size_t smem = 1024 + kF8Fixed + stages * stage;
  g.stages = stages;
  cudaError_t e = cudaFuncSetAttribute(k_f8_mm<NT>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       (int)smem);
  if (e != cudaSuccess) return cuda_fail(e, "FP8 product attribute");
  const int grid = (int)(g.items < nsm ? g.items : nsm);
  k_f8_mm<NT><<<grid, kF8Threads, smem, st>>>(ta, tb, g);
  return cuda_fail(cudaGetLastError(), "FP8 product launch");
}

static bool f8_aligned(const void *p, size_t n) {
  return reinterpret_cast<uintptr_t>(p) % n == 0;
}

static int64_t scale_pitch(int64_t rows) { return (rows + kF8Block - 1) / kF8Block * kF8Block; }

// a code matrix whose rows and pitch stay inside 32-bit coordinates and 64-bit offsets
static bool f8_good(const fqt_fp8 *q) {
  return q->codes && q->scales && f8_aligned(q->codes, 16) && f8_aligned(q->scales, 16) &&
         q->pitch % 16 == 0 && q->pitch >= q->cols;
}

fqt_status quantize_fp8(const void *X, int64_t ldx, bool bf16, int64_t rows, int64_t cols,
                        int block_rows, fqt_fp8 *q, fqt_fp8 *qt, int *status, cudaStream_t st) {
  F8QuantArgs a = {};
  a.x = X;
  a.ldx = rows > 1 ? ldx : 0;
  a.rows = rows;
  a.cols = (int)cols;
  a.whole = block_rows == kF8Block;
  a.status = status;
  if (q) {
    a.c = q->codes;
    a.pitch = q->pitch;
    a.s = q->scales;
    a.sp = scale_pitch(rows);
  }
  if (qt) {
    a.ct = qt->codes;
    a.pitch_t = qt->pitch;
    a.st = qt->scales;
    a.spt = scale_pitch(cols);
  }
  const bool vec = f8_aligned(X, 16) && a.ldx * (bf16 ? 2 : 4) % 16 == 0;
  const dim3 grid((unsigned)((cols + kF8Block - 1) / kF8Block),
                  (unsigned)((rows + kF8Block - 1) / kF8Block));
  if (bf16) k_f8_quant<__nv_bfloat16><<<grid, 256, 0, st>>>(a, vec);
  else k_f8_quant<float><<<grid, 256, 0, st>>>(a, vec);
  return cuda_fail(cudaGetLastError(), "FP8 quantizer launch");
}

fqt_status fp8_matmul(const fqt_fp8 *A, const fqt_fp8 *B, bool bf16, void *out, int64_t ldo,
                      void *ws, cudaStream_t st) {
  const int64_t M = A->rows, N = B->rows, K = A->cols;
  const int nsm = device_sm_count();
  const F8Plan p = f8_plan(M, N, (K + kF8Block - 1) / kF8Block, nsm);
  const fqt_fp8 *a = p.swap ? B : A, *b = p.swap ? A : B;
  CUtensorMap ta, tb;
  if (!make_map_codes(&ta, a, BM) || !make_map_codes(&tb, b, (uint32_t)p.nt))
    return cuda_fail(cudaErrorUnknown, "FP8 tensor map");
  F8Args g = {};
  g.sa = a->scales;
  g.sb = b->scales;
  g.spa = scale_pitch(a->rows);
  g.spb = scale_pitch(b->rows);
  g.M = a->rows;
  g.N = b->rows;
  g.nkb = (int)((K + kF8Block - 1) / kF8Block);
  g.m_tiles = p.m_tiles;
  g.n_tiles = p.n_tiles;
  g.splits = p.splits;
  g.kb_per = p.kb_per;
  g.items = (int64_t)p.m_tiles * p.n_tiles * p.splits;
  g.out = out;
  g.ldo = M > 1 ? ldo : 0;
  g.bf16 = bf16;
  g.swap = p.swap;
  g.part = reinterpret_cast<float *>(static_cast<char *>(ws) + kHeaderBytes);
  g.b_whole = b->block_rows == kF8Block;
  g.status = static_cast<int *>(ws);
  fqt_status s = p.nt == 256   ? launch_f8<256>(ta, tb, g, nsm, st)
                 : p.nt == 128 ? launch_f8<128>(ta, tb, g, nsm, st)
                 : p.nt == 64  ? launch_f8<64>(ta, tb, g, nsm, st)
                               : launch_f8<32>(ta, tb, g, nsm, st);
  if (s != FQT_OK || p.splits == 1) return s;
  const int64_t blocks = (M * N + 255) / 256;
  const int grid = (int)(blocks < 8 * nsm ? blocks : 8 * nsm);
  if (bf16)
    k_f8_join<__nv_bfloat16><<<grid, 256, 0, st>>>(g.part, p.splits, M, N,
                                                   static_cast<__nv_bfloat16 *>(out), g.ldo);
  else
    k_f8_join<float><<<grid, 256, 0, st>>>(g.part, p.splits, M, N, static_cast<float *>(out),
                                           g.ldo);
  return cuda_fail(cudaGetLastError(), "FP8 join launch");
}

}  // namespace fqt

using namespace fqt;

extern "C" {

fqt_status fqt_quantize_fp8(const void *X, int64_t ldx, fqt_dtype dtype, int64_t rows,
                            int64_t cols, int block_rows, fqt_fp8 *q, fqt_fp8 *qt,
                            void *workspace, size_t ws_bytes, void *stream) {
  if (rows < 0 || cols <= 0 || rows > kF8MaxSize || cols > kF8MaxSize) return FQT_EINVAL;
  if (block_rows != 1 && block_rows != kF8Block) return FQT_EINVAL;
  if (dtype != FQT_F32 && dtype != FQT_BF16) return FQT_EINVAL;
  if (!q && !qt) return FQT_EINVAL;
  if (rows > 1 && (ldx < cols || ldx > ((int64_t)1 << 40))) return FQT_EINVAL;
  if (rows > 0 && (!X || !f8_aligned(X, dtype == FQT_BF16 ? 2 : 4))) return FQT_EINVAL;
  for (int i = 0; i < 2; ++i) {
    fqt_fp8 *o = i ? qt : q;
    if (!o) continue;
    fqt_fp8 v = *o;
    v.rows = i ? cols : rows;
    v.cols = i ? rows : cols;
    if (rows > 0 && !f8_good(&v)) return FQT_EINVAL;
  }
  if (!workspace || !f8_aligned(workspace, 256) || ws_bytes < kHeaderBytes) return FQT_EWORKSPACE;
  for (int i = 0; i < 2; ++i) {
    fqt_fp8 *o = i ? qt : q;
    if (!o) continue;
    o->rows = i ? cols : rows;
    o->cols = i ? rows : cols;
    o->block_rows = block_rows;
  }
  if (rows == 0) return FQT_OK;
  return quantize_fp8(X, ldx, dtype == FQT_BF16, rows, cols, block_rows, q, qt,
                      static_cast<int *>(workspace), reinterpret_cast<cudaStream_t>(stream));
}

size_t fqt_fp8_matmul_workspace_size(int64_t M, int64_t N, int64_t K) {
  return fp8_matmul_ws_bytes(M, N, K);
}

fqt_status fqt_fp8_matmul(const fqt_fp8 *A, const fqt_fp8 *B, fqt_dtype dtype, void *out,
                          int64_t ldo, void *workspace, size_t ws_bytes, void *stream) {
  if (!A || !B || (dtype != FQT_F32 && dtype != FQT_BF16)) return FQT_EINVAL;
  if (A->rows < 0 || B->rows < 0 || A->cols < 0 || A->cols != B->cols) return FQT_EINVAL;
  const int64_t M = A->rows, N = B->rows, K = A->cols;
  if (M > kF8MaxSize || N > kF8MaxSize || K > kF8MaxSize) return FQT_EINVAL;
  for (const fqt_fp8 *q : {A, B})
    if (q->block_rows != 1 && q->block_rows != kF8Block) return FQT_EINVAL;
  if (M == 0 || N == 0) return FQT_OK;
  const size_t es = dtype == FQT_BF16 ? 2 : 4;
  if (!out || !f8_aligned(out, es) || (M > 1 && (ldo < N || ldo > ((int64_t)1 << 40))))
    return FQT_EINVAL;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  if (K == 0) {  // an empty sum
    const cudaError_t e = cudaMemset2DAsync(out, (M > 1 ? ldo : N) * es, 0, N * es, M, st);
    return cuda_fail(e, "FP8 product clear");
  }
  if (!f8_good(A) || !f8_good(B)) return FQT_EINVAL;
  if (!workspace || !f8_aligned(workspace, 256) || ws_bytes < fp8_matmul_ws_bytes(M, N, K))
    return FQT_EWORKSPACE;
  return fp8_matmul(A, B, dtype == FQT_BF16, out, ldo, workspace, st);
}

}  // extern "C"
