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
constexpr int kF8EpiWarps = 8, kF8Epi0 = 4;  // warps 0 loads, 1 products, 2 and 3 none
constexpr int kF8Threads = 32 * (kF8Epi0 + kF8EpiWarps);
constexpr int kF8RegsCtl = 64, kF8RegsEpi = 216;
static_assert(128 * kF8RegsCtl + 256 * kF8RegsEpi <= kF8Threads * ((65536 / kF8Threads) / 8 * 8),
              "register shares exceed the launch's");
constexpr int kF8Band = 8;  // row tiles of a band of tiles
// Scales: an epilogue warp keeps those of four K blocks (32 of A's rows, then up to 128
// of B's) in shared memory and the next four on their way in registers; a read from L2
// takes as long as two or three K blocks of products.
constexpr int kF8Ahead = 4;
constexpr size_t kF8ScaleBytes = 640;
constexpr size_t kF8OffBar = kF8Ahead * kF8EpiWarps * kF8ScaleBytes;
constexpr size_t kF8Bars = 2 * kMaxStages + 5;
constexpr size_t kF8Fixed = (kF8OffBar + kF8Bars * 8 + 16 + 1023) & ~(size_t)1023;
constexpr size_t kF8BoxBytes = 4096;    // an epilogue warp's 32 rows x 128 bytes of output

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
  int boxes;       // out is written in boxes by TMA
  float *part;     // splits > 1: fp32 partial outputs, one after another
  int stages;
  int b_whole;  // B's scale is one for 128 rows
  int *status;
};

// mbar_wait without its read of the timer at the first miss, which takes longer than a
// K block's products: the timer is read after a few tries that sleep.
__device__ __forceinline__ bool f8_wait(uint64_t *bar, uint32_t parity, int *status) {
#pragma unroll 1
  for (int i = 0; i < 4; ++i)
    if (mbar_try_wait_sleep(bar, parity, 20000u)) return true;
  return mbar_wait(bar, parity, status);
}

// The accumulator's reader is done with it (the pair's leader counts both CTAs).  What
// it read is ordered by tcgen05.wait and tcgen05.fence; a releasing arrival would also
// wait for the scales on their way.
template <bool PAIR>
__device__ __forceinline__ void f8_release(uint64_t *bar) {
  if constexpr (PAIR)
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(
                     leader_addr(bar))
                 : "memory");
  else
    asm volatile("mbarrier.arrive.relaxed.cta.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar))
                 : "memory");
}

template <bool PAIR>
__device__ __forceinline__ void f8_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc,
                                       uint32_t accumulate) {
  if constexpr (PAIR)
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
}

// An item: this CTA's 128 rows of A against NT rows of B over some K blocks.  The
// two CTAs of a pair take the same item, each its 128 of the super tile's 256 rows.
struct F8Item {
  int64_t m0, n0;
  int kb0, kb1, split;
};

template <int NT, bool PAIR>
__device__ __forceinline__ F8Item f8_item(const F8Args &g, int64_t it) {
  F8Item t;
  const int64_t tiles = (int64_t)g.m_tiles * g.n_tiles;
  t.split = (int)(it / tiles);
  const int64_t r = it - t.split * tiles;
  // bands of kF8Band row tiles, so that the tiles in flight share rows of both operands
  const int64_t band = r / ((int64_t)kF8Band * g.n_tiles);
  const int64_t in = r - band * kF8Band * g.n_tiles;
  const int high = (int)min((int64_t)kF8Band, g.m_tiles - band * kF8Band);
  const int64_t n = in / high;
  t.n0 = n * NT;
  t.m0 = (band * kF8Band + in - n * high) * (PAIR ? 2 * BM : BM) +
         (PAIR ? (blockIdx.x & 1) * BM : 0);
  t.kb0 = t.split * g.kb_per;
  t.kb1 = min(g.nkb, t.kb0 + g.kb_per);
  return t;
}

template <typename T>
__device__ __forceinline__ T f8_out(float v) {
  if constexpr (sizeof(T) == 4) return v;
  else return __float2bfloat16_rn(v);
}

// 16 bytes of output from the sums at acc.
template <typename T>
__device__ __forceinline__ uint4 f8_pack(const f32x2 *acc) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float u, v;
    if constexpr (sizeof(T) == 4) {
      unpack2(acc[i / 2], u, v);
      w[i] = __float_as_uint(i & 1 ? v : u);
    } else {
      unpack2(acc[i], u, v);
      const __nv_bfloat162 b = __floats2bfloat162_rn(u, v);
      w[i] = *reinterpret_cast<const uint32_t *>(&b);
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
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
    if (vec && n + j + E <= g.N) {
      *reinterpret_cast<uint4 *>(p + j) = f8_pack<T>(&acc[j / 2]);
    } else {
#pragma unroll
      for (int i = 0; i < E; ++i) {
        float u, v;
        unpack2(acc[(j + i) / 2], u, v);
        if (n + j + i < g.N) p[j + i] = f8_out<T>(i & 1 ? v : u);
      }
    }
  }
}

// The same through boxes of 32 rows x 128 bytes: a warp lays its rows' 128 bytes in
// shared memory (128-byte swizzle) and TMA writes them, leaving out what lies past
// the output's ends.  (Stored from registers, a warp's 16-byte pieces of 32 rows
// take half a sector each.)
template <typename T, int W>
__device__ __forceinline__ void f8_store_boxes(const F8Args &g, const CUtensorMap *map,
                                               uint8_t *box, int lane, int64_t m0, int64_t n,
                                               const f32x2 (&acc)[W / 2]) {
  constexpr int E = 16 / sizeof(T), C = 8 * E;  // columns of a box
  if (m0 >= g.M) return;
#pragma unroll
  for (int j = 0; j < W; j += C) {
    if (n + j >= g.N) break;
    if (lane == 0) bulk_wait_read(0);
    __syncwarp();
#pragma unroll
    for (int k = 0; k < 8; ++k)
      *reinterpret_cast<uint4 *>(box + sw128_off(lane, k)) = f8_pack<T>(&acc[(j + k * E) / 2]);
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) {
      tma_store_2d(map, (int32_t)(n + j), (int32_t)m0, box);
      bulk_commit();
    }
  }
}

// The scales of kF8Ahead K blocks on their way: this lane's row of A, and four of B's
// columns a lane (or, with one scale for 128 of B's rows, the one of the first column).
// Entries past the ends of the scales are others' and belong to no output.
template <int W>
struct F8Ahead {
  float a[kF8Ahead];
  float4 b[kF8Ahead];
  __device__ __forceinline__ void get(const F8Args &g, int64_t m, int64_t n, int kb, int kb1,
                                      int lane) {
    const float *pa = g.sa + min(m + lane, g.spa - 1);
    const float *pb = g.sb + (g.b_whole ? min(n, g.spb - 1) : min(n + 4 * lane, g.spb - 4));
#pragma unroll
    for (int i = 0; i < kF8Ahead; ++i) {
      if (kb + i >= kb1) break;
      a[i] = __ldg(pa + (kb + i) * g.spa);
      if (g.b_whole) b[i].x = __ldg(pb + (kb + i) * g.spb);
      else if (4 * lane < W) b[i] = __ldg(reinterpret_cast<const float4 *>(pb + (kb + i) * g.spb));
    }
  }
  __device__ __forceinline__ void put(float *sc, int lane, bool whole) const {
#pragma unroll
    for (int i = 0; i < kF8Ahead; ++i) {
      float *to = sc + i * (int)(kF8ScaleBytes / 4);
      to[lane] = a[i];
      if (whole) to[32] = b[i].x;
      else if (4 * lane < W) reinterpret_cast<float4 *>(to + 32)[lane] = b[i];
    }
  }
};

// Adds one accumulator's W columns, scaled, to the sums.  The columns come in pieces
// of 16, the next one on its way while this one is added.
template <int W>
__device__ __forceinline__ void f8_fold(uint32_t taddr, float sa, const float *sb, bool whole,
                                        f32x2 (&acc)[W / 2]) {
  constexpr int CH = 16;
  const float s1 = sa * sb[0];
  const f32x2 s2 = pack2(s1, s1), sa2 = pack2(sa, sa);
  uint32_t r[2][CH];
  tmem_ldw_nw<CH>(taddr, r[0]);
  tmem_wait_ld(r[0]);
#pragma unroll
  for (int j = 0; j < W; j += CH) {
    const uint32_t(&v)[CH] = r[(j / CH) & 1];
    if (j + CH < W) tmem_ldw_nw<CH>(taddr + (uint32_t)(j + CH), r[(j / CH + 1) & 1]);
    if (whole) {
#pragma unroll
      for (int i = 0; i < CH; i += 2)
        acc[(j + i) / 2] =
            fma2(pack2(__uint_as_float(v[i]), __uint_as_float(v[i + 1])), s2, acc[(j + i) / 2]);
    } else {
#pragma unroll
      for (int i = 0; i < CH; i += 4) {
        const float4 b = *reinterpret_cast<const float4 *>(sb + j + i);
        acc[(j + i) / 2] = fma2(pack2(__uint_as_float(v[i]), __uint_as_float(v[i + 1])),
                                mul2(sa2, pack2(b.x, b.y)), acc[(j + i) / 2]);
        acc[(j + i) / 2 + 1] = fma2(pack2(__uint_as_float(v[i + 2]), __uint_as_float(v[i + 3])),
                                    mul2(sa2, pack2(b.z, b.w)), acc[(j + i) / 2 + 1]);
      }
    }
    if (j + CH < W) tmem_wait_ld(r[(j / CH + 1) & 1]);
  }
}

// One CTA per 128 x NT tile (and split of the K blocks), persistent, or a pair of CTAs
// per 256 x 256 super tile: each loads its 128 rows of A and 128 of B's 256 rows, and
// the leader issues products over both (cta_group::2), so an operand byte is loaded
// for twice the products.  Warp 0 feeds operand stages of one K block by TMA, warp 1
// issues a K block's four products into one of two accumulators; the eight epilogue
// warps (quadrant of rows x half of the columns) read the blocks' scales ahead and
// fold each K block into their sums.
template <int NT, bool PAIR>
__global__ void __launch_bounds__(kF8Threads, 1)
    k_f8_mm(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
            const __grid_constant__ CUtensorMap tmOut, const F8Args g) {
  static_assert(!PAIR || NT == 256, "a pair's super tile has 256 columns");
  constexpr int W = NT / 2;                 // columns of an epilogue warp
  constexpr int NB = PAIR ? NT / 2 : NT;    // rows of B that this CTA loads
  constexpr uint32_t kStage = (uint32_t)(kTileBytes + NB * kF8Block);
  constexpr uint32_t kCols = 2 * NT < 32 ? 32 : 2 * NT;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint64_t *full = reinterpret_cast<uint64_t *>(smem + kF8OffBar), *empty = full + kMaxStages;
  uint64_t *accf = empty + kMaxStages, *acce = accf + 2;
  uint64_t *drain = acce + 2;
  uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(full + kF8Bars);
  volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
  uint8_t *ops = smem + kF8Fixed;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = PAIR ? (int)(blockIdx.x & 1) : 0;
  const int64_t first = PAIR ? blockIdx.x >> 1 : blockIdx.x;
  const int64_t step = PAIR ? gridDim.x >> 1 : gridDim.x;
  if (threadIdx.x == 0) {
    for (int i = 0; i < g.stages; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&accf[i], 1);
      mbar_init(&acce[i], (PAIR ? 2 : 1) * kF8EpiWarps);
    }
    mbar_init(drain, 1);
    *abort_flag = 0;
    fence_barrier_init();
  }
  if (warp == 1) {
    if constexpr (PAIR) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                       smem_u32(tmem_slot)),
                   "r"(kCols)
                   : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                       smem_u32(tmem_slot)),
                   "r"(kCols)
                   : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  tc_fence_before();
  __syncthreads();
  if constexpr (PAIR) cluster_sync();  // the peer's barriers exist
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  if (warp >= kF8Epi0) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kF8RegsEpi));
    const int q = warp & 3, h = (warp - kF8Epi0) >> 2;
    const uint32_t lane_base = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(h * W);
    uint8_t *box = ops + (size_t)g.stages * kStage + (size_t)(warp - kF8Epi0) * kF8BoxBytes;
    float *sc = reinterpret_cast<float *>(smem + kF8Ahead * (warp - kF8Epi0) * kF8ScaleBytes);
    F8Ahead<W> ahead;
    if (first < g.items) {
      const F8Item t = f8_item<NT, PAIR>(g, first);
      ahead.get(g, t.m0 + q * 32, t.n0 + h * W, t.kb0, t.kb1, lane);
    }
    uint32_t c = 0;  // K blocks so far
    bool ok = true;
    for (int64_t it = first; ok && it < g.items && !*abort_flag; it += step) {
      const F8Item t = f8_item<NT, PAIR>(g, it);
      f32x2 acc[W / 2];
#pragma unroll
      for (int j = 0; j < W / 2; ++j) acc[j] = pack2(0.0f, 0.0f);
      const int64_t m = t.m0 + q * 32, n = t.n0 + h * W;
      for (int kb = t.kb0; kb < t.kb1; ++kb, ++c) {
        const int buf = c & 1, at = (kb - t.kb0) % kF8Ahead;
        if (at == 0) {
          __syncwarp();
          ahead.put(sc, lane, g.b_whole);
          __syncwarp();
          if (kb + kF8Ahead < t.kb1) {
            ahead.get(g, m, n, kb + kF8Ahead, t.kb1, lane);
          } else if (it + step < g.items) {
            const F8Item u = f8_item<NT, PAIR>(g, it + step);
            ahead.get(g, u.m0 + q * 32, u.n0 + h * W, u.kb0, u.kb1, lane);
          }
        }
        if (!f8_wait(&accf[buf], (c >> 1) & 1u, g.status)) {
          *abort_flag = 1;
          ok = false;
          break;
        }
        tc_fence_after();
        const float *mine = sc + at * (int)(kF8ScaleBytes / 4);
        f8_fold<W>(lane_base + (uint32_t)(buf * NT), mine[lane], mine + 32, g.b_whole, acc);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) f8_release<PAIR>(&acce[buf]);
      }
      if (!ok) break;
      if (W >= 64 && g.boxes) {
        if constexpr (W >= 64) {
          if (g.bf16) f8_store_boxes<__nv_bfloat16, W>(g, &tmOut, box, lane, m, n, acc);
          else f8_store_boxes<float, W>(g, &tmOut, box, lane, m, n, acc);
        }
      } else if (g.splits > 1) {
        f8_store<float, W>(g, g.part + t.split * g.M * g.N, g.swap ? g.M : g.N, m + lane, n, acc);
      } else if (g.bf16) {
        f8_store<__nv_bfloat16, W>(g, static_cast<__nv_bfloat16 *>(g.out), g.ldo, m + lane, n,
                                   acc);
      } else {
        f8_store<float, W>(g, static_cast<float *>(g.out), g.ldo, m + lane, n, acc);
      }
    }
    if (lane == 0) bulk_wait_all();
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kF8RegsCtl));
    if (warp == 0 && lane == 0) {
      int s = 0;
      uint32_t ph = 0;
      bool ok = true;
      for (int64_t it = first; ok && it < g.items && !*abort_flag; it += step) {
        const F8Item t = f8_item<NT, PAIR>(g, it);
        for (int kb = t.kb0; kb < t.kb1; ++kb) {
          if (!f8_wait(&empty[s], ph ^ 1u, g.status)) {
            *abort_flag = 1;
            ok = false;
            break;
          }
          uint8_t *st = ops + (size_t)s * kStage;
          if constexpr (PAIR) {  // the leader's barrier counts both CTAs' bytes
            if (rank == 0) mbar_expect_tx(&full[s], 2 * kStage);
            const uint32_t bar = leader_addr(&full[s]);
            tma_load_2d_pair(st, &tmA, kb * kF8Block, (int32_t)t.m0, bar);
            tma_load_2d_pair(st + kTileBytes, &tmB, kb * kF8Block, (int32_t)t.n0 + rank * NB, bar);
          } else {
            mbar_expect_tx(&full[s], kStage);
            tma_load_2d(st, &tmA, kb * kF8Block, (int32_t)t.m0, &full[s]);
            tma_load_2d(st + kTileBytes, &tmB, kb * kF8Block, (int32_t)t.n0, &full[s]);
          }
          if (++s == g.stages) { s = 0; ph ^= 1u; }
        }
      }
      // every load has landed before the CTA exits
      if (*abort_flag) {
        sleep_ns(200000);
      } else {
        for (int i = 0; i < g.stages; ++i) {
          if (!f8_wait(&empty[s], ph ^ 1u, g.status)) break;
          if (++s == g.stages) { s = 0; ph ^= 1u; }
        }
      }
    } else if (warp == 1 && lane == 0 && rank == 0) {
      int s = 0;
      uint32_t ph = 0, c = 0;
      bool ok = true;
      // D fp32; A, B E4M3 (format 0), both K-major
      constexpr uint32_t idesc = (1u << 4) | ((uint32_t)(NT >> 3) << 17) |
                                 ((uint32_t)((PAIR ? 2 * BM : BM) >> 4) << 24);
      for (int64_t it = first; ok && it < g.items && !*abort_flag; it += step) {
        const F8Item t = f8_item<NT, PAIR>(g, it);
        for (int kb = t.kb0; kb < t.kb1; ++kb, ++c) {
          const int buf = c & 1;
          if (!f8_wait(&acce[buf], ((c >> 1) & 1u) ^ 1u, g.status) ||
              !f8_wait(&full[s], ph, g.status)) {
            *abort_flag = 1;
            ok = false;
            break;
          }
          tc_fence_after();
          const uint32_t a_addr = smem_u32(ops + (size_t)s * kStage);
          const uint64_t da = sw128_desc(a_addr), db = sw128_desc(a_addr + (uint32_t)kTileBytes);
#pragma unroll
          for (int k = 0; k < 4; ++k)  // 32 entries each
            f8_mma<PAIR>(tmem + (uint32_t)(buf * NT), da + 2 * k, db + 2 * k, idesc,
                         k > 0 ? 1u : 0u);
          if constexpr (PAIR) {
            umma_commit_pair(&empty[s]);
            umma_commit_pair(&accf[buf]);
          } else {
            umma_commit(&empty[s]);
            umma_commit(&accf[buf]);
          }
          if (++s == g.stages) { s = 0; ph ^= 1u; }
        }
      }
      // every product has completed before tensor memory is released
      if constexpr (PAIR)
        asm volatile(
            "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(
                smem_u32(drain))
            : "memory");
      else
        umma_commit(drain);
      f8_wait(drain, 0, g.status);
    }
  }
  tc_fence_before();
  __syncthreads();
  // neither CTA of a pair leaves while the other may still reach its memory
  if constexpr (PAIR) cluster_sync();
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    if constexpr (PAIR)
      asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem),
                   "r"(kCols)
                   : "memory");
    else
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem),
                   "r"(kCols)
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

// The output as boxes of 32 rows x 128 bytes (its base and its pitch on 16 bytes).
static bool make_map_f8_out(CUtensorMap *m, void *out, bool bf16, int64_t rows, int64_t cols,
                            int64_t ldo) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t es = bf16 ? 2 : 4;
  cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  cuuint64_t strides[1] = {(cuuint64_t)ldo * es};
  cuuint32_t box[2] = {(cuuint32_t)(128 / es), 32};
  cuuint32_t one[2] = {1, 1};
  return fn(m, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 2, out,
            dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_NONE,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// How a product of M x N outputs over nkb K blocks is cut into tiles.
struct F8Plan {
  bool swap;  // A is the right operand, out is written transposed
  bool pair;  // 256 x 256 super tiles on CTA pairs
  int nt, m_tiles, n_tiles, splits, kb_per;
};

static F8Plan f8_plan(int64_t M, int64_t N, int64_t nkb, int nsm) {
  F8Plan p;
  // few rows: they become the narrow side, and the other operand fills the 128 rows
  p.swap = M <= 64;
  const int64_t a = p.swap ? N : M, b = p.swap ? M : N;
  // super tiles where they occupy three quarters of the SMs
  p.pair = !p.swap && nsm >= 2 &&
           ((a + 255) / 256) * ((b + 255) / 256) * 8 >= (int64_t)nsm * 3;
  const int rows = p.pair ? 2 * BM : BM;
  p.m_tiles = (int)((a + rows - 1) / rows);
  p.nt = p.pair ? 256 : !p.swap ? 128 : b <= 32 ? 32 : 64;
  p.n_tiles = (int)((b + p.nt - 1) / p.nt);
  if (p.pair) {
    p.splits = 1;
    p.kb_per = (int)nkb;
    return p;
  }
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

template <int NT, bool PAIR>
static fqt_status launch_f8(const CUtensorMap &ta, const CUtensorMap &tb, const CUtensorMap &to,
                            F8Args &g, int nsm, cudaStream_t st) {
  constexpr size_t stage = kTileBytes + (PAIR ? NT / 2 : NT) * kF8Block;
  constexpr size_t boxes = NT >= 128 ? kF8EpiWarps * kF8BoxBytes : 0;
  constexpr size_t room = 227 * 1024 - 1024 - kF8Fixed - boxes;
  constexpr int stages = room / stage < kMaxStages ? (int)(room / stage) : kMaxStages;
  constexpr size_t smem = 1024 + kF8Fixed + stages * stage + boxes;
  g.stages = stages;
  auto kernel = k_f8_mm<NT, PAIR>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       (int)smem);
  if (e != cudaSuccess) return cuda_fail(e, "FP8 product attribute");
  const int64_t ctas = g.items * (PAIR ? 2 : 1);
  const int most = PAIR ? nsm & ~1 : nsm;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(ctas < most ? ctas : most));
  cfg.blockDim = dim3(kF8Threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = PAIR ? 2 : 1;
  at[0].val.clusterDim.y = 1;
  at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cuda_fail(cudaLaunchKernelEx(&cfg, kernel, ta, tb, to, (const F8Args &)g),
                   "FP8 product launch");
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
  F8Args g = {};
  g.ldo = M > 1 ? ldo : N;
  g.boxes = p.nt >= 128 && p.splits == 1 && f8_aligned(out, 16) &&
            g.ldo * (bf16 ? 2 : 4) % 16 == 0;
  CUtensorMap ta, tb, to = {};
  if (!make_map_codes(&ta, a, BM) || !make_map_codes(&tb, b, p.pair ? 128u : (uint32_t)p.nt) ||
      (g.boxes && !make_map_f8_out(&to, out, bf16, M, N, g.ldo)))
    return cuda_fail(cudaErrorUnknown, "FP8 tensor map");
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
  g.bf16 = bf16;
  g.swap = p.swap;
  g.part = reinterpret_cast<float *>(static_cast<char *>(ws) + kHeaderBytes);
  g.b_whole = b->block_rows == kF8Block;
  g.status = static_cast<int *>(ws);
  fqt_status s = p.pair        ? launch_f8<256, true>(ta, tb, to, g, nsm, st)
                 : p.nt == 128 ? launch_f8<128, false>(ta, tb, to, g, nsm, st)
                 : p.nt == 64  ? launch_f8<64, false>(ta, tb, to, g, nsm, st)
                               : launch_f8<32, false>(ta, tb, to, g, nsm, st);
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
