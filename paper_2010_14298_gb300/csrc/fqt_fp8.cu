// fqt_fp8.cu -- matrix products of 8-bit floating-point codes (E4M3) with one
// power-of-two scale for each block of 128 entries along the contraction, and their
// quantizer.
//
//   out_mn = sum_kb 2^(ea[kb][m] + eb[kb][n]) sum_(k in block kb) a_mk b_nk
#include <cuda_runtime.h>
#include <math.h>

#include <algorithm>

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
// 2^e, -127 <= e <= 127
__device__ __forceinline__ float pow2(int e) {
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
  uint8_t *s, *st;  // scales, four blocks of a row side by side (fqt.h)
  int64_t sp, spt;  // rows of scales
  int whole;  // one scale for the 128 x 128 block
  int *status;
};

__device__ __forceinline__ int64_t scale_at(int64_t block, int64_t rows, int64_t row) {
  return ((block >> 2) * rows + row) * 4 + (block & 3);
}

// Entries that are no numbers, given as NaN: they count for no scale and take the NaN
// code (0x7F or 0xFF).  Magnitudes are compared as integers.
__device__ __forceinline__ uint32_t f8_mag(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

// Packed bf16: the products of both halves; a power of two in both.
__device__ __forceinline__ uint32_t bf16_mul2(uint32_t a, uint32_t b) {
  const __nv_bfloat162 p = __hmul2(*reinterpret_cast<const __nv_bfloat162 *>(&a),
                                   *reinterpret_cast<const __nv_bfloat162 *>(&b));
  return *reinterpret_cast<const uint32_t *>(&p);
}
__device__ __forceinline__ uint32_t bf16_both(float v) {
  return __byte_perm(__float_as_uint(v), 0u, 0x3232);
}

// N consecutive entries as they lie in memory: bf16 in half the registers, so that
// more of them can be on their way.
template <typename T, int N>
struct F8Raw {
  static constexpr int words = N * (int)sizeof(T) / 4;
  uint32_t w[words];
  // zeros past `left` entries
  __device__ __forceinline__ void load(const T *p, int64_t left) {
    if (left >= N) {
#pragma unroll
      for (int i = 0; i < words; i += 4) {
        const uint4 v = __ldg(reinterpret_cast<const uint4 *>(p) + i / 4);
        w[i] = v.x; w[i + 1] = v.y; w[i + 2] = v.z; w[i + 3] = v.w;
      }
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < N; ++i)
        w[i] = i < left ? __ldg(reinterpret_cast<const unsigned *>(p) + i) : 0u;
    } else {
      const unsigned short *h = reinterpret_cast<const unsigned short *>(p);
#pragma unroll
      for (int i = 0; i < words; ++i)
        w[i] = (2 * i < left ? __ldg(h + 2 * i) : 0u) |
               (uint32_t)(2 * i + 1 < left ? __ldg(h + 2 * i + 1) : 0u) << 16;
    }
  }
  // from shared memory
  __device__ __forceinline__ void take(const T *p) {
#pragma unroll
    for (int i = 0; i < words; i += 4) {
      const uint4 v = reinterpret_cast<const uint4 *>(p)[i / 4];
      w[i] = v.x; w[i + 1] = v.y; w[i + 2] = v.z; w[i + 3] = v.w;
    }
  }
  __device__ __forceinline__ float f(int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
    else return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
  }
  __device__ __forceinline__ void set_nan(int i) {
    if constexpr (sizeof(T) == 4) w[i] = 0x7FFFFFFFu;
    else w[i / 2] |= i & 1 ? 0x7FFF0000u : 0x7FFFu;
  }
  // The largest magnitude (fp32 bits).  Entries that are no numbers become NaN and
  // count for none.
  __device__ __forceinline__ uint32_t top(int *status) {
    uint32_t m = 0u;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < N; ++i) m = max(m, w[i] & 0x7FFFFFFFu);
    } else {
#pragma unroll
      for (int i = 0; i < words; ++i) m = __vmaxu2(m, w[i] & 0x7FFF7FFFu);
      m = max(m << 16, m & 0xFFFF0000u);
    }
    if (m >= 0x7F800000u) {
      record_status(status, FQT_ENONFINITE);
      m = 0u;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if (isfinite(f(i))) m = max(m, f8_mag(f(i)));
        else set_nan(i);
      }
    }
    return m;
  }
  // Codes of entries 2 i and 2 i + 1, which share a scale.  (A product with a power of
  // two is exact in bf16 down to 2^-133, far below what E4M3 holds of it.)
  __device__ __forceinline__ uint32_t pair(int i, float inv) const {
    if constexpr (sizeof(T) == 4) {
      return f8_pair(f(2 * i) * inv, f(2 * i + 1) * inv);
    } else {
      const uint32_t s = bf16_mul2(w[i], bf16_both(inv));
      return f8_pair(__uint_as_float(s << 16), __uint_as_float(s & 0xFFFF0000u));
    }
  }
};

// N consecutive entries that lie on no 16-byte boundary, read by one warp (zeros past
// `left`) entry by entry, but neighbouring lanes read neighbours, and put into shared
// memory.  (Each lane its own 8 or 16 entries took eight times the wavefronts.)
template <typename T, int N>
__device__ __forceinline__ void f8_fetch(T (&v)[N / 32], const T *p, int64_t left, int lane) {
#pragma unroll
  for (int k = 0; k < N / 32; ++k)
    v[k] = lane + 32 * k < left ? p[lane + 32 * k] : (T)0.0f;
}
template <typename T, int N>
__device__ __forceinline__ void f8_put(T *dst, const T (&v)[N / 32], int lane) {
#pragma unroll
  for (int k = 0; k < N / 32; ++k) dst[lane + 32 * k] = v[k];
}

// Codes by rows alone, one scale per 128 entries: a warp takes 512 columns of R rows,
// a lane 16 of each, so that a block's maximum is three shuffles, the codes leave in
// 16-byte stores and a row's four scales in one word.  Bound by memory traffic: 8192 x
// 4096 in bf16 19.8 us, 5.1 TB/s; in fp32 28.7 us, 5.8 TB/s.
template <typename T, int R>
__global__ void __launch_bounds__(256) k_f8_rows(const F8QuantArgs a, const bool vec) {
  __shared__ __align__(16) uint32_t stages[8][512 * sizeof(T) / 4];
  let_next_start();
  wait_for_previous();
  const int lane = threadIdx.x & 31;
  const int64_t row = ((int64_t)blockIdx.x * 8 + (threadIdx.x >> 5)) * R;
  const int64_t col = (int64_t)blockIdx.y * 512 + lane * 16;
  F8Raw<T, 16> v[R];
  uint32_t m[R];
  if (vec) {
#pragma unroll
    for (int r = 0; r < R; ++r)
      v[r].load(static_cast<const T *>(a.x) + (row + r) * a.ldx + col,
                row + r < a.rows ? a.cols - col : 0);
  } else {
    T *stage = reinterpret_cast<T *>(stages[threadIdx.x >> 5]);
    const int64_t c0 = (int64_t)blockIdx.y * 512;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      T e[512 / 32];
      f8_fetch<T, 512>(e, static_cast<const T *>(a.x) + (row + r) * a.ldx + c0,
                       row + r < a.rows ? a.cols - c0 : 0, lane);
      f8_put<T, 512>(stage, e, lane);
      __syncwarp();
      v[r].take(stage + lane * 16);
      __syncwarp();
    }
  }
#pragma unroll
  for (int r = 0; r < R; ++r) m[r] = v[r].top(a.status);
#pragma unroll
  for (int o = 4; o > 0; o >>= 1)
#pragma unroll
    for (int r = 0; r < R; ++r) m[r] = max(m[r], __shfl_xor_sync(0xffffffffu, m[r], o));
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int e = f8_exponent(m[r]);
    // the four blocks' bytes, from lanes 0, 8, 16 and 24
    uint32_t w = (uint32_t)(e + 127) << (lane >> 3) * 8;
    w |= __shfl_xor_sync(0xffffffffu, w, 8);
    w |= __shfl_xor_sync(0xffffffffu, w, 16);
    if (row + r >= a.rows) continue;
    if (lane == 0) reinterpret_cast<uint32_t *>(a.s)[blockIdx.y * a.sp + row + r] = w;
    if (col >= a.cols) continue;
    const float inv = pow2(-e);
    uint32_t c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = v[r].pair(2 * i, inv) | v[r].pair(2 * i + 1, inv) << 16;
    *reinterpret_cast<uint4 *>(a.c + (row + r) * a.pitch + col) =
        make_uint4(c[0], c[1], c[2], c[3]);
  }
}

// Codes along both axes (or blocks of 128 x 128): one CTA per 128 x 128 tile.  A thread
// holds 4 rows x 8 columns, so it packs codes along either axis without exchanging
// bytes: 8 bytes of each of its rows go straight to memory, 4 bytes of each of its
// columns through shared memory.  The entries are read once for both outputs: 8192 x 4096
// in bf16 28.8 us, 4.7 TB/s (66% of the issue slots taken), in fp32 37.8 us, 5.3 TB/s.
constexpr int kF8TileThreads = 512;

template <typename T>
__global__ void __launch_bounds__(kF8TileThreads, sizeof(T) == 4 ? 2 : 3)
    k_f8_tile(const F8QuantArgs a, const bool vec) {
  let_next_start();
  wait_for_previous();
  __shared__ __align__(16) uint32_t cmax[kF8TileThreads / 32][kF8Block];  // fp32 bits
  __shared__ __align__(16) float cinv[kF8Block];
  __shared__ uint32_t wmax[4];
  // a column's 32 words of 4 rows, word w at place w ^ 2 (column / 8): the threads of a
  // warp, 16 columns 8 apart x 2 words, write 32 banks
  __shared__ __align__(16) uint32_t tr[kF8Block * 32];
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  const int cg = t & 15, rg = t >> 4;  // its 8 columns and its 4 rows
  const int64_t r0 = (int64_t)blockIdx.x * kF8Block;
  const int64_t c0 = (int64_t)blockIdx.y * kF8Block;
  const int64_t row = r0 + rg * 4, col = c0 + cg * 8;
  F8Raw<T, 8> v[4];
  uint32_t rm[4], cm[8];
  if (vec) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      v[i].load(static_cast<const T *>(a.x) + (row + i) * a.ldx + col,
                row + i < a.rows ? a.cols - col : 0);
  } else {  // the warp's two rows i at a time, by way of 1 KB of `tr`
    T *stage = reinterpret_cast<T *>(tr + warp * 256);
    // all on their way at once: 8192 x 4095 in fp32 44 us, two at a time 55, in bf16 36 and 41
    T e[4][2][kF8Block / 32];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int64_t r = r0 + (2 * warp + h) * 4 + i;
        f8_fetch<T, kF8Block>(e[i][h], static_cast<const T *>(a.x) + r * a.ldx + c0,
                              r < a.rows ? a.cols - c0 : 0, lane);
      }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int h = 0; h < 2; ++h) f8_put<T, kF8Block>(stage + h * kF8Block, e[i][h], lane);
      __syncwarp();
      v[i].take(stage + (lane >> 4) * kF8Block + cg * 8);
      __syncwarp();
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) rm[i] = v[i].top(a.status);
  // column maxima over the thread's rows (NaN counts for none) and the warp's two row
  // groups; packed for bf16
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      cm[j] = 0u;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t m = f8_mag(v[i].f(j));
        cm[j] = max(cm[j], m < 0x7F800000u ? m : 0u);
      }
      cm[j] = max(cm[j], __shfl_xor_sync(0xffffffffu, cm[j], 16));
    }
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint32_t m = 0u;
#pragma unroll
      for (int i = 0; i < 4; ++i) m = __vmaxu2(m, v[i].w[j] & 0x7FFF7FFFu);
      if (max(m << 16, m & 0xFFFF0000u) >= 0x7F800000u) {
        m = 0u;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t x = v[i].w[j] & 0x7FFF7FFFu;
          m = __vmaxu2(m, ((x & 0xFFFFu) < 0x7F80u ? x & 0xFFFFu : 0u) |
                              (x < 0x7F800000u ? x & 0xFFFF0000u : 0u));
        }
      }
      m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, 16));
      cm[2 * j] = m << 16;
      cm[2 * j + 1] = m & 0xFFFF0000u;
    }
  }
  if (lane < 16) {
    *reinterpret_cast<uint4 *>(&cmax[warp][cg * 8]) = make_uint4(cm[0], cm[1], cm[2], cm[3]);
    *reinterpret_cast<uint4 *>(&cmax[warp][cg * 8 + 4]) = make_uint4(cm[4], cm[5], cm[6], cm[7]);
  }
#pragma unroll
  for (int o = 8; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < 4; ++i) rm[i] = max(rm[i], __shfl_xor_sync(0xffffffffu, rm[i], o));
  __syncthreads();
  int e_col = 0;
  if (t < kF8Block) {
    uint32_t m = 0u;
#pragma unroll
    for (int w = 0; w < kF8TileThreads / 32; ++w) m = max(m, cmax[w][t]);
    if (a.whole) {
      m = __reduce_max_sync(0xffffffffu, m);
      if (lane == 0) wmax[warp] = m;
    } else {
      e_col = f8_exponent(m);
      cinv[t] = pow2(-e_col);
    }
  }
  __syncthreads();
  if (a.whole) {
    const uint32_t m = max(max(wmax[0], wmax[1]), max(wmax[2], wmax[3]));
#pragma unroll
    for (int i = 0; i < 4; ++i) rm[i] = m;
    e_col = f8_exponent(m);
  }
  if (a.ct && t < kF8Block) a.st[scale_at(blockIdx.x, a.spt, c0 + t)] = (uint8_t)(e_col + 127);
  if (a.c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int e = f8_exponent(rm[i]);
      if (cg == 0) a.s[scale_at(blockIdx.y, a.sp, row + i)] = (uint8_t)(e + 127);
      if (row + i >= a.rows || col >= a.cols) continue;
      const float inv = pow2(-e);
      *reinterpret_cast<uint2 *>(a.c + (row + i) * a.pitch + col) =
          make_uint2(v[i].pair(0, inv) | v[i].pair(1, inv) << 16,
                     v[i].pair(2, inv) | v[i].pair(3, inv) << 16);
    }
  }
  if (a.ct) {
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
      float2 inv = *reinterpret_cast<const float2 *>(&cinv[cg * 8 + j]);
      if (a.whole) inv.x = inv.y = pow2(-e_col);
      uint32_t c[2];
      if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float s = h ? inv.y : inv.x;
          c[h] = f8_pair(v[0].f(j + h) * s, v[1].f(j + h) * s) |
                 f8_pair(v[2].f(j + h) * s, v[3].f(j + h) * s) << 16;
        }
      } else {
        const uint32_t s =
            __byte_perm(__float_as_uint(inv.x), __float_as_uint(inv.y), 0x7632);
        uint32_t p[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = bf16_mul2(v[i].w[j / 2], s);
        c[0] = f8_pair(__uint_as_float(p[0] << 16), __uint_as_float(p[1] << 16)) |
               f8_pair(__uint_as_float(p[2] << 16), __uint_as_float(p[3] << 16)) << 16;
        c[1] = f8_pair(__uint_as_float(p[0] & 0xFFFF0000u), __uint_as_float(p[1] & 0xFFFF0000u)) |
               f8_pair(__uint_as_float(p[2] & 0xFFFF0000u), __uint_as_float(p[3] & 0xFFFF0000u))
                   << 16;
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) tr[(cg * 8 + j + h) * 32 + (rg ^ (2 * cg))] = c[h];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int at = k * kF8TileThreads + t, j = at >> 3, ch = at & 7;
      if (c0 + j >= a.cols || r0 + ch * 16 >= a.rows) continue;
      const uint2 *pairs = reinterpret_cast<const uint2 *>(tr + j * 32);
      const uint2 lo = pairs[(2 * ch) ^ (j >> 3)], hi = pairs[(2 * ch + 1) ^ (j >> 3)];
      *reinterpret_cast<uint4 *>(a.ct + (c0 + j) * a.pitch_t + r0 + ch * 16) =
          make_uint4(lo.x, lo.y, hi.x, hi.y);
    }
  }
}

// ---------------------------------------------------------------------------
// Product
// ---------------------------------------------------------------------------
// The scales are powers of two, so the tensor cores apply them themselves: tcgen05
// kind::mxf8f6f4 multiplies the sum of 32 products by 2^(ea + eb), with ea and eb read
// from tensor memory, before it adds it to the fp32 accumulator.  Its scales belong to
// 32 entries of K; a block's four steps use the same ones.  (With unscaled products,
// each block's sums read back and folded into registers, the hand-over of an
// accumulator for every 128 entries of K bound the kernel: 172 us for 8192 x 4096 x
// 4096, with per-row scales on both sides 232.)  Now 77 us, 3.6 PFLOP/s of the tensor
// cores' nominal 4.5: a K block of a super tile takes 0.30 us, 0.28 at that rate, and
// handing its accumulator over 1.2 us.  An fp32 output takes 103 us (its accumulators are
// handed over every eight K blocks; super tiles of 224 columns, which leave room for two
// accumulators, took 101, and 38 us where 256 take 25: 4096 x 1024 x 8192 in bf16).
constexpr int kF8EpiWarps = 8, kF8Epi0 = 4;  // warps 0 loads, 1 products, 2 and 3 scales
constexpr int kF8Threads = 32 * (kF8Epi0 + kF8EpiWarps);
// K blocks of an accumulator: a step of the tensor core drops what lies below the
// accumulator's last bit, which adds up where the terms have one sign (5e-7 of the result
// after 8192 terms of equal size, 8e-6 after 65536; 3e-4 there, and 1.8e-2 after 2^21,
// where the first few terms are as large as all others together).  So after 1024 terms
// for an fp32 output, and after 8192 for a bf16 one, which rounds up to 4e-3 away, the
// sums move to fp32 registers, rounded to nearest.
constexpr int kF8Chunk = 8, kF8ChunkBf16 = 64;
constexpr int kF8Group = 4;             // K blocks whose scales share a 32-bit word
constexpr int kF8Ring = 4;              // groups of scales in shared memory
constexpr size_t kF8RingBytes = 1536;   // 128 of A's rows, up to 256 of B's
constexpr size_t kF8OffBar = kF8Ring * kF8RingBytes;
constexpr size_t kF8Bars = 2 * kMaxStages + 2 * kF8Ring + 5;
constexpr size_t kF8Fixed = (kF8OffBar + kF8Bars * 8 + 16 + 1023) & ~(size_t)1023;
constexpr size_t kF8BoxBytes = 2048;    // an epilogue warp's box of output
constexpr int kF8Parts = 8;             // CTAs that share a tile's K blocks at most
constexpr int kF8Band = 8;              // row tiles of a band of tiles

struct F8Args {
  const uint32_t *sa, *sb;  // scales of four K blocks a word, groups spa / spb words apart
  int64_t spa, spb;
  int64_t M, N;  // rows of A and of B
  int nkb;       // K blocks
  int chunk;     // of them, to an accumulator
  int m_tiles, n_tiles, splits, kb_per;
  int64_t items;
  void *out;
  int64_t ldo;
  int bf16, swap;  // swap: out is indexed [B row][A row]
  int boxes;       // out is written in boxes by TMA
  int stages;
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

// True in one lane of a converged warp, the same one every time.
__device__ __forceinline__ bool elect_one() {
  uint32_t one;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "elect.sync _|p, 0xffffffff;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(one));
  return one != 0;
}

// A wait that acquires what the pair's other CTA has written.
__device__ __forceinline__ bool f8_wait_cluster(uint64_t *bar, uint32_t parity, int *status) {
  uint64_t t0 = 0;
  for (int i = 0;; ++i) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2, %3;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(smem_u32(bar)), "r"(parity), "r"(20000u)
        : "memory");
    if (ok) return true;
    if ((i & 3) == 3) {
      const uint64_t t = global_ns();
      if (t0 == 0) t0 = t;
      if (t - t0 > kWaitLimitNs) {
        record_status(status, FQT_ETIMEOUT);
        return false;
      }
    }
  }
}

// The accumulator's reader is done with it (the pair's leader counts both CTAs).  What
// it read is ordered by tcgen05.wait and tcgen05.fence.
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

// 32 entries of K: D (+)= 2^(ea + eb) A B^T, the exponents in the bytes of the
// tensor-memory words at sa and sb that the instruction descriptor names.
template <bool PAIR>
__device__ __forceinline__ void f8_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc,
                                       uint32_t sa, uint32_t sb, uint32_t accumulate) {
  if constexpr (PAIR)
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X "
        "[%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X "
        "[%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate)
        : "memory");
}

// Scales of 128 rows from shared memory (32 rows of 16 bytes: word w of row r is that
// of row 32 w + r) to four columns of tensor memory, in every quadrant of its lanes.
template <bool PAIR>
__device__ __forceinline__ void f8_copy_scales(uint32_t taddr, uint32_t saddr) {
  // 8 x 16 byte core matrices 128 bytes apart, no swizzle, descriptor version 1
  const uint64_t desc = (uint64_t)((saddr & 0x3FFFFu) >> 4) | (uint64_t)(128 >> 4) << 32 |
                        (uint64_t)1 << 46;
  if constexpr (PAIR)
    asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc)
                 : "memory");
  else
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc)
                 : "memory");
}

// An item: this CTA's 128 rows of A against NT rows of B over some K blocks (from a
// multiple of kF8Group; a tile's parts follow one another).  The two CTAs of a pair take
// the same item, each its 128 of the super tile's 256 rows.
struct F8Item {
  int64_t m0, n0;
  int kb0, kb1;
};

template <int NT, bool PAIR>
__device__ __forceinline__ F8Item f8_item(const F8Args &g, int64_t it) {
  F8Item t;
  const int64_t r = PAIR ? it : it / g.splits;
  // bands of kF8Band row tiles, so that the tiles in flight share rows of both operands
  const int64_t band = r / ((int64_t)kF8Band * g.n_tiles);
  const int64_t in = r - band * kF8Band * g.n_tiles;
  const int high = (int)min((int64_t)kF8Band, g.m_tiles - band * kF8Band);
  const int64_t n = in / high;
  t.n0 = n * NT;
  t.m0 = (band * kF8Band + in - n * high) * (PAIR ? 2 * BM : BM) +
         (PAIR ? (blockIdx.x & 1) * BM : 0);
  t.kb0 = PAIR ? 0 : (int)(it - r * g.splits) * g.kb_per;
  t.kb1 = min(g.nkb, t.kb0 + g.kb_per);
  return t;
}

template <typename T>
__device__ __forceinline__ T f8_out(float v) {
  if constexpr (sizeof(T) == 4) return v;
  else return __float2bfloat16_rn(v);
}

// 32 columns (16 where the warp has no more) of this warp's lanes, without waiting.
template <int W>
__device__ __forceinline__ void f8_read(uint32_t taddr, uint32_t (&v)[32]) {
  if constexpr (W < 32) tmem_ld16_nw(taddr, *reinterpret_cast<uint32_t(*)[16]>(v));
  else tmem_ld32_nw(taddr, v);
}

// 16 bytes of output from the sums at v (fp32 bits).
template <typename T>
__device__ __forceinline__ uint4 f8_pack(const uint32_t *v) {
  if constexpr (sizeof(T) == 4) {
    return make_uint4(v[0], v[1], v[2], v[3]);
  } else {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 b =
          __floats2bfloat162_rn(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1]));
      w[i] = *reinterpret_cast<const uint32_t *>(&b);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// Byte offset of 16-byte chunk k of row r in a box of 32 rows of 64 bytes (the 64-byte
// swizzle: no bank conflicts either way).
__device__ __forceinline__ uint32_t box_off(int r, int k) {
  return (uint32_t)(r * 64 + ((k ^ ((r >> 1) & 3)) << 4));
}

// W <= 32 columns from n on of this lane's row m of a transposed output: lanes are
// neighbours there.
template <typename T>
__device__ __forceinline__ void f8_store_swapped(const F8Args &g, T *out, int64_t ld, int64_t m,
                                                 int64_t n, const uint32_t (&v)[32], int W) {
#pragma unroll
  for (int j = 0; j < 32; ++j)
    if (m < g.M && j < W && n + j < g.N) out[(n + j) * ld + m] = f8_out<T>(__uint_as_float(v[j]));
}

// A warp's 32 rows (this lane's is m0 + lane) x 32 columns from n on, entry by entry, by
// way of the box, so that a row's columns are neighbours.  (The loop over rows stays a
// loop: unrolled into every piece and type, the kernel waited for its instructions.)
template <typename T>
__device__ __forceinline__ void f8_store_rows(const F8Args &g, T *out, int64_t ld, float *box,
                                              int lane, int64_t m0, int64_t n,
                                              const uint32_t (&v)[32]) {
  if (m0 >= g.M || n >= g.N) return;
  const int rows = (int)min((int64_t)32, g.M - m0);
  const int col = lane & 15, up = lane >> 4;
#pragma unroll
  for (int h = 0; h < 32; h += 16) {  // 16 columns of 32 rows at a time, two rows a store
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *reinterpret_cast<uint4 *>(box + box_off(lane, j) / 4) =
          make_uint4(v[h + 4 * j], v[h + 4 * j + 1], v[h + 4 * j + 2], v[h + 4 * j + 3]);
    __syncwarp();
    if (n + h + col >= g.N) continue;
    T *p = out + (m0 + up) * ld + n + h + col;
#pragma unroll 2
    for (int r = up; r < rows; r += 2, p += 2 * ld)
      *p = f8_out<T>(box[box_off(r, col >> 2) / 4 + (col & 3)]);
  }
}

// The same through a box that TMA writes (it leaves out what lies past the output's
// ends): rows of 64 bytes, 16 columns of fp32 or 32 of bf16.  Stored from registers, a
// warp's pieces of 32 rows would take a part of a sector each.
template <typename T>
__device__ __forceinline__ void f8_store_box(const F8Args &g, const CUtensorMap *map, float *box,
                                             int lane, int64_t m0, int64_t n,
                                             const uint32_t (&v)[32]) {
  constexpr int E = 16 / sizeof(T);
  if (m0 >= g.M) return;
#pragma unroll
  for (int h = 0; h < 32; h += 4 * E) {
    if (n + h >= g.N) return;
    if (lane == 0) bulk_wait_read(0);
    __syncwarp();
#pragma unroll
    for (int k = 0; k < 4; ++k)
      *reinterpret_cast<uint4 *>(box + box_off(lane, k) / 4) = f8_pack<T>(&v[h + k * E]);
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) {
      tma_store_2d(map, (int32_t)(n + h), (int32_t)m0, box);
      bulk_commit();
    }
  }
}

// The sums of a tile whose K blocks a cluster's CTAs share, the parts in their order:
// each part lies in its CTA's shared memory at the same place, in the output's order, in
// rows of NT + 4 entries or (swapped) columns of 128, and each CTA adds up its share.
template <int NT>
__device__ __forceinline__ void f8_join(const F8Args &g, int64_t it, const float *part) {
  const F8Item t = f8_item<NT, false>(g, it);
  const int parts = g.splits, self = (int)(it % parts);
  const int run = g.swap ? BM : NT, pitch = g.swap ? BM : NT + 4;  // of outputs in a row
  // rows and entries of a row that the output has
  const int64_t r0 = g.swap ? t.n0 : t.m0, c0 = g.swap ? t.m0 : t.n0;
  const int rows = (int)min((int64_t)(g.swap ? NT : BM), (g.swap ? g.N : g.M) - r0);
  const int cols = (int)min((int64_t)run, (g.swap ? g.M : g.N) - c0);
  for (int e = (self * kF8Threads + (int)threadIdx.x) * 4; e < rows * run;
       e += parts * kF8Threads * 4) {
    const int r = e / run, c = e % run;
    if (c >= cols) continue;
    float v[kF8Parts][4];
#pragma unroll
    for (int k = 0; k < kF8Parts; ++k)
      if (k < parts)
        asm volatile(
            "{\n\t.reg .b32 a;\n\t"
            "mapa.shared::cluster.u32 a, %4, %5;\n\t"
            "ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [a];\n\t}"
            : "=f"(v[k][0]), "=f"(v[k][1]), "=f"(v[k][2]), "=f"(v[k][3])
            : "r"(smem_u32(part + r * pitch + c)), "r"(k)
            : "memory");
#pragma unroll
    for (int k = 1; k < kF8Parts; ++k)
      if (k < parts)
#pragma unroll
        for (int i = 0; i < 4; ++i) v[0][i] += v[k][i];
    const int64_t o = (r0 + r) * g.ldo + c0 + c;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (c + i < cols) {
        if (g.bf16) static_cast<__nv_bfloat16 *>(g.out)[o + i] = __float2bfloat16_rn(v[0][i]);
        else static_cast<float *>(g.out)[o + i] = v[0][i];
      }
  }
}

// One CTA per 128 x NT tile (and part of the K blocks), persistent, or a pair of CTAs
// per 256 x NT super tile: each loads its 128 rows of A and half of B's NT rows, and
// the leader issues products over both (cta_group::2), so an operand byte is loaded
// for twice the products.  Warp 0 feeds operand stages of one K block by TMA, warps 2
// and 3 in turn the scales of four K blocks, warp 1 issues a K block's four products;
// the eight epilogue warps (quadrant of rows x half of the columns) take an accumulator
// into registers, hand it back and store it.  ACCS accumulators of NT columns: with two
// the products go on meanwhile.  FOLD: an accumulator holds g.chunk K blocks, and the
// epilogue adds them up.
template <int NT, int ACCS, bool PAIR, bool FOLD>
__global__ void __launch_bounds__(kF8Threads, 1)
    k_f8_mm(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
            const __grid_constant__ CUtensorMap tmOut, const F8Args g) {
  // columns of an epilogue warp: a multiple of 32 for the first half's
  constexpr int W0 = NT <= 64 ? NT / 2 : (NT / 2 + 31) / 32 * 32, W1 = NT - W0;
  constexpr int NB = PAIR ? NT / 2 : NT;    // rows of B that this CTA loads
  constexpr uint32_t kStage = (uint32_t)(kTileBytes + NB * kF8Block);
  constexpr int kSbCols = (NT + 127) / 128 * 4;       // columns of B's scales
  constexpr uint32_t kScales = ACCS * NT;             // two buffers of A's and B's scales
  constexpr uint32_t kUsed = kScales + 2 * (4 + kSbCols);
  constexpr uint32_t kCols = kUsed <= 128 ? 128 : kUsed <= 256 ? 256 : 512;
  static_assert(kUsed <= 512, "tensor memory has 512 columns");
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint64_t *full = reinterpret_cast<uint64_t *>(smem + kF8OffBar), *empty = full + kMaxStages;
  uint64_t *accf = empty + kMaxStages, *acce = accf + 2;
  uint64_t *sfull = acce + 2, *sempty = sfull + kF8Ring, *drain = sempty + kF8Ring;
  uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(full + kF8Bars);
  volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
  uint8_t *ops = smem + kF8Fixed;
  let_next_start();
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
    for (int i = 0; i < kF8Ring; ++i) {
      mbar_init(&sfull[i], PAIR ? 2 : 1);
      mbar_init(&sempty[i], 1);
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
  wait_for_previous();

  if (warp >= kF8Epi0) {
    const int q = warp & 3, h = (warp - kF8Epi0) >> 2;
    const int W = h ? W1 : W0;
    const uint32_t lane_base = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(h * W0);
    float *box = reinterpret_cast<float *>(ops + (size_t)g.stages * kStage +
                                           (size_t)(warp - kF8Epi0) * kF8BoxBytes);
    uint32_t c = 0;  // accumulators so far
    bool ok = true;
    for (int64_t it = first; ok && it < g.items && !*abort_flag; it += step) {
      const F8Item t = f8_item<NT, PAIR>(g, it);
      constexpr int P = (W0 + 31) / 32;  // pieces of up to 32 columns
      uint32_t v[P][32];
      if constexpr (FOLD)
#pragma unroll
        for (int i = 0; i < 32 * P; ++i) v[i / 32][i % 32] = 0u;
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
          for (int p = 0; p < P; ++p) f8_read<W0>(from + 32 * p, v[p]);
#pragma unroll
          for (int p = 0; p < P; ++p) tmem_wait_ld(v[p]);
        } else {
#pragma unroll
          for (int j = 0; j < W0; j += 16) {  // 16 columns at a time: registers
            uint32_t r[16];
            tmem_ld16_nw(from + (uint32_t)j, r);
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
      if (!ok) break;
      if constexpr (!PAIR) {
        if (g.splits > 1) {  // the products are done with the operand stages
          float *part = reinterpret_cast<float *>(ops);
          const int r = q * 32 + lane, j = h * W0;
#pragma unroll
          for (int i = 0; i < W0; i += 4) {
            const uint32_t *x = &v[i / 32][i % 32];
            if (!g.swap) {
              *reinterpret_cast<uint4 *>(part + r * (NT + 4) + j + i) =
                  make_uint4(x[0], x[1], x[2], x[3]);
            } else {
#pragma unroll
              for (int k = 0; k < 4; ++k) part[(j + i + k) * BM + r] = __uint_as_float(x[k]);
            }
          }
          break;
        }
      }
      const int64_t m = t.m0 + q * 32, n = t.n0 + h * W0;
      float *fp32 = g.bf16 ? nullptr : static_cast<float *>(g.out);
      __nv_bfloat16 *bf16 = static_cast<__nv_bfloat16 *>(g.out);
      const int64_t ld = g.ldo;
#pragma unroll
      for (int p = 0; p < P; ++p) {
        if (32 * p >= W) break;
        const int64_t np = n + 32 * p;
        if constexpr (NT >= 64) {
          if (!g.swap) {
            if (g.boxes && g.bf16)
              f8_store_box<__nv_bfloat16>(g, &tmOut, box, lane, m, np, v[p]);
            else if (g.boxes)
              f8_store_box<float>(g, &tmOut, box, lane, m, np, v[p]);
            else if (fp32)
              f8_store_rows<float>(g, fp32, ld, box, lane, m, np, v[p]);
            else
              f8_store_rows<__nv_bfloat16>(g, bf16, ld, box, lane, m, np, v[p]);
          }
        }
        if constexpr (NT <= 64) {
          if (g.swap && fp32)
            f8_store_swapped<float>(g, fp32, ld, m + lane, np, v[p], W);
          else if (g.swap)
            f8_store_swapped<__nv_bfloat16>(g, bf16, ld, m + lane, np, v[p], W);
        }
      }
    }
    if (lane == 0) bulk_wait_all();
  } else if (warp == 0) {
    if (lane == 0) {
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
    }
  } else if (warp == 1) {
    // The whole warp runs this loop and one lane issues: addresses and descriptors that
    // are the same in every lane live in uniform registers, where the instructions want
    // them.  (In a loop of one lane's own, an instruction took longer to issue than to
    // run: 94 us for 8192 x 4096 x 4096, now 77.)
    if (rank == 0) {
      const bool one = elect_one();
      int s = 0;
      uint32_t ph = 0, c = 0, grp = 0;
      bool ok = true;
      // D fp32; A, B E4M3 (format 0), both K-major; E8M0 scales; bits 4-5 and 29-30: the
      // byte of B's and A's scale words
      constexpr uint32_t idesc0 = ((uint32_t)(NT >> 3) << 17) | (1u << 23) |
                                  ((uint32_t)(PAIR ? 2 : 1) << 27);
      const uint64_t da0 = sw128_desc(smem_u32(ops));
      const uint64_t db0 = sw128_desc(smem_u32(ops) + (uint32_t)kTileBytes);
      for (int64_t it = first; ok && it < g.items && !*abort_flag; it += step) {
        const F8Item t = f8_item<NT, PAIR>(g, it);
        uint32_t sa = 0;
        for (int k0 = t.kb0; ok && k0 < t.kb1; k0 = FOLD ? k0 + g.chunk : t.kb1, ++c) {
          const int k1 = FOLD ? min(k0 + g.chunk, t.kb1) : t.kb1, buf = c % ACCS;
          if (!f8_wait(&acce[buf], ((c / ACCS) & 1u) ^ 1u, g.status)) {
            ok = false;
            break;
          }
          const uint32_t acc = tmem + (uint32_t)(buf * NT);
          for (int kb = k0; kb < k1; ++kb) {
            if ((kb & (kF8Group - 1)) == 0) {  // the next group's scales
              const int slot = grp % kF8Ring;
              if (!f8_wait_cluster(&sfull[slot], (grp / kF8Ring) & 1u, g.status)) {
                ok = false;
                break;
              }
              tc_fence_after();
              sa = tmem + kScales + (grp & 1u) * (4 + kSbCols);
              if (one) {
                const uint32_t src = smem_u32(smem + slot * kF8RingBytes);
                f8_copy_scales<PAIR>(sa, src);
#pragma unroll
                for (int i = 0; i < kSbCols / 4; ++i)
                  f8_copy_scales<PAIR>(sa + 4 + 4 * i, src + 512 + 512 * i);
                if constexpr (PAIR) umma_commit_pair(&sempty[slot]);
                else umma_commit(&sempty[slot]);
              }
              ++grp;
            }
            if (!f8_wait(&full[s], ph, g.status)) {
              ok = false;
              break;
            }
            tc_fence_after();
            if (one) {
              const uint64_t da = da0 + (uint64_t)(s * (int)(kStage >> 4));
              const uint64_t db = db0 + (uint64_t)(s * (int)(kStage >> 4));
              const uint32_t id = (uint32_t)kb & (kF8Group - 1);
              const uint32_t idesc = idesc0 | id << 4 | id << 29;
#pragma unroll
              for (int k = 0; k < 4; ++k)  // 32 entries each
                f8_mma<PAIR>(acc, da + 2 * k, db + 2 * k, idesc, sa, sa + 4,
                             (k > 0 || kb > k0) ? 1u : 0u);
              if constexpr (PAIR) umma_commit_pair(&empty[s]);
              else umma_commit(&empty[s]);
            }
            if (++s == g.stages) { s = 0; ph ^= 1u; }
          }
          if (!ok) break;
          if (one) {
            if constexpr (PAIR) umma_commit_pair(&accf[buf]);
            else umma_commit(&accf[buf]);
          }
        }
      }
      if (!ok) *abort_flag = 1;
      // every product has completed before tensor memory is released
      if (one) {
        if constexpr (PAIR)
          asm volatile(
              "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(
                  smem_u32(drain))
              : "memory");
        else
          umma_commit(drain);
      }
      f8_wait(drain, 0, g.status);
    }
  } else {
    // scales: words of four K blocks, warps 2 and 3 a group in turn
    uint32_t grp = 0;
    bool ok = true;
    for (int64_t it = first; ok && it < g.items && !*abort_flag; it += step) {
      const F8Item t = f8_item<NT, PAIR>(g, it);
      for (int kb = t.kb0; kb < t.kb1; kb += kF8Group, ++grp) {
        if ((grp & 1u) != (uint32_t)(warp - 2)) continue;
        const int slot = grp % kF8Ring;
        const int64_t kg = kb / kF8Group;
        uint32_t w[4 + kSbCols];
#pragma unroll
        for (int i = 0; i < 4 + kSbCols; ++i) {  // row 32 i + lane of A's, then of B's
          const bool in_a = i < 4;
          const int64_t r = in_a ? t.m0 + 32 * i + lane : t.n0 + 32 * (i - 4) + lane;
          // rows past the ends: any scale that is a number (127: one)
          w[i] = r < (in_a ? g.spa : g.spb)
                     ? __ldg((in_a ? g.sa + kg * g.spa : g.sb + kg * g.spb) + r)
                     : 0x7F7F7F7Fu;
        }
        if (!f8_wait(&sempty[slot], ((grp / kF8Ring) & 1u) ^ 1u, g.status)) {
          *abort_flag = 1;
          ok = false;
          break;
        }
        uint4 *dst = reinterpret_cast<uint4 *>(smem + slot * kF8RingBytes);
#pragma unroll
        for (int i = 0; i < (4 + kSbCols) / 4; ++i)
          dst[32 * i + lane] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          if constexpr (PAIR) mbar_arrive_cluster(leader_addr(&sfull[slot]));
          else mbar_arrive(&sfull[slot]);
        }
      }
    }
    // the last copies have been read (and, in a pair, the leader's arrivals are in)
    for (int i = 0; ok && i < kF8Ring; ++i, ++grp)
      ok = f8_wait(&sempty[grp % kF8Ring], ((grp / kF8Ring) & 1u) ^ 1u, g.status);
  }
  tc_fence_before();
  __syncthreads();
  if constexpr (!PAIR) {
    if (g.splits > 1) {
      cluster_sync();  // the tile's parts are in the shared memory of the cluster
      f8_join<NT>(g, first, reinterpret_cast<const float *>(ops));
      __syncthreads();
    }
  }
  // no CTA of a pair or a cluster leaves while another may still reach its memory
  if (PAIR || g.splits > 1) cluster_sync();
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

// The output as boxes of 32 rows x 64 bytes (its base and its pitch on 16 bytes).
static bool make_map_f8_out(CUtensorMap *m, void *out, bool bf16, int64_t rows, int64_t cols,
                            int64_t ldo) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t es = bf16 ? 2 : 4;
  cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  cuuint64_t strides[1] = {(cuuint64_t)ldo * es};
  cuuint32_t box[2] = {(cuuint32_t)(64 / es), 32};
  cuuint32_t one[2] = {1, 1};
  return fn(m, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 2, out,
            dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B,
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
  const int64_t groups = (nkb + kF8Group - 1) / kF8Group;
  auto cut = [&](int nt, int64_t splits) {  // whole groups of scales each
    p.nt = nt;
    p.n_tiles = (int)((b + nt - 1) / nt);
    p.kb_per = (int)((groups + splits - 1) / splits) * kF8Group;
    p.splits = (int)((nkb + p.kb_per - 1) / p.kb_per);
  };
  if (p.pair) {
    cut(256, 1);
    return p;
  }
  // Single CTAs: the width, and the CTAs of a cluster that share a tile's K blocks, of
  // which the estimate is least. A K block takes 0.27 us in a tile of 128 columns, 0.23 of
  // 64 and 0.2 of 32 (its operands come in at 120 GB/s a CTA), meeting in shared memory
  // 2.3: 2360 x 283 x 8179 14.7 us in tiles of 128 shared by two, 19.6 of 64 unshared;
  // 700 x 1000 x 2000 9.5 and 7.8; 1 x 1024 x 4096 5.5 us shared by eight, 6.2 by four;
  // 1 x 4096 x 1024 4.8 unshared, 5.5 by two.
  // A cluster lies within one of the GPU's groups of SMs, so not all SMs have a place in
  // one (15 clusters of eight ran at once, 36 of four, 44 of three): what does not fit
  // would wait for a second round (2048 x 128 x 4096 15.0 us by eight, 8.2 by four).
  int64_t least = INT64_MAX;
  F8Plan best = p;
  const int widest = p.swap ? (b <= 32 ? 32 : 64) : 128;
  for (int nt = widest; nt >= (p.swap ? widest : 64); nt /= 2)
    for (int64_t splits = 1; splits <= kF8Parts && (splits == 1 || splits <= groups); ++splits) {
      cut(nt, splits);
      const int64_t tiles = (int64_t)p.m_tiles * p.n_tiles;
      const int room = p.splits > 4 ? nsm * 3 / 4 : p.splits > 2 ? nsm * 7 / 8 : nsm;
      if (splits > 1 && tiles * p.splits > room) break;
      const int64_t rounds = (tiles * p.splits + nsm - 1) / nsm;
      const int64_t ns =
          rounds * std::min<int64_t>(p.kb_per, nkb) * (nt == 128 ? 270 : nt == 64 ? 230 : 200) +
          (p.splits > 1 ? 2300 : 0);
      if (ns < least) {
        least = ns;
        best = p;
      }
    }
  return best;
}

template <int NT, int ACCS, bool PAIR, bool FOLD>
static fqt_status launch_f8_as(const CUtensorMap &ta, const CUtensorMap &tb, const CUtensorMap &to,
                            F8Args &g, int nsm, cudaStream_t st) {
  constexpr size_t stage = kTileBytes + (PAIR ? NT / 2 : NT) * kF8Block;
  constexpr size_t boxes = NT >= 64 ? kF8EpiWarps * kF8BoxBytes : 0;
  constexpr size_t room = 227 * 1024 - 1024 - kF8Fixed - boxes;
  constexpr int stages = room / stage < kMaxStages ? (int)(room / stage) : kMaxStages;
  constexpr size_t smem = 1024 + kF8Fixed + stages * stage + boxes;
  g.stages = stages;
  auto kernel = k_f8_mm<NT, ACCS, PAIR, FOLD>;
  static DeviceOnce once;
  cudaError_t e = allow_smem(kernel, smem, once);
  if (e != cudaSuccess) return cuda_fail(e, "FP8 product attribute");
  const int64_t ctas = g.items * (PAIR ? 2 : 1);
  const int most = PAIR ? nsm & ~1 : nsm;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(ctas < most ? ctas : most));
  cfg.blockDim = dim3(kF8Threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = PAIR ? 2 : (unsigned)g.splits;
  at[1].val.clusterDim.y = 1;
  at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = PAIR || g.splits > 1 ? 2 : 1;
  return cuda_fail(cudaLaunchKernelEx(&cfg, kernel, ta, tb, to, (const F8Args &)g),
                   "FP8 product launch");
}

template <int NT, int ACCS, bool PAIR>
static fqt_status launch_f8(const CUtensorMap &ta, const CUtensorMap &tb, const CUtensorMap &to,
                            F8Args &g, int nsm, cudaStream_t st) {
  g.chunk = g.bf16 ? kF8ChunkBf16 : kF8Chunk;
  if (g.kb_per > g.chunk)
    return launch_f8_as<NT, ACCS, PAIR, true>(ta, tb, to, g, nsm, st);
  return launch_f8_as<NT, ACCS, PAIR, false>(ta, tb, to, g, nsm, st);
}

static bool f8_aligned(const void *p, size_t n) {
  return reinterpret_cast<uintptr_t>(p) % n == 0;
}

static int64_t scale_rows(int64_t rows) { return (rows + kF8Block - 1) / kF8Block * kF8Block; }

// a code matrix whose pitch a tensor map takes, and its offsets 64 bits
static bool f8_good(const fqt_fp8 *q) {
  return q->codes && q->scales && f8_aligned(q->codes, 16) && f8_aligned(q->scales, 16) &&
         q->pitch % 16 == 0 && q->pitch >= q->cols && q->pitch < ((int64_t)1 << 40);
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
    a.sp = scale_rows(rows);
  }
  if (qt) {
    a.ct = qt->codes;
    a.pitch_t = qt->pitch;
    a.st = qt->scales;
    a.spt = scale_rows(cols);
  }
  const bool vec = f8_aligned(X, 16) && a.ldx * (bf16 ? 2 : 4) % 16 == 0;
  if (!qt && block_rows == 1) {
    // rows of a warp: 64 entries of a thread on their way, fewer where the rows are few
    const int64_t chunks = (cols + 511) / 512;
    const int per = rows * chunks < 32 * device_sm_count() ? 1 : bf16 ? 4 : 2;
    const dim3 grid((unsigned)((rows + 8 * per - 1) / (8 * per)), (unsigned)chunks);
    auto kernel = bf16 ? (per == 4 ? k_f8_rows<__nv_bfloat16, 4> : k_f8_rows<__nv_bfloat16, 1>)
                       : (per == 2 ? k_f8_rows<float, 2> : k_f8_rows<float, 1>);
    return cuda_fail(launch_behind(kernel, grid, 256, 0, st, a, vec), "FP8 quantizer launch");
  }
  const dim3 grid((unsigned)((rows + kF8Block - 1) / kF8Block),
                  (unsigned)((cols + kF8Block - 1) / kF8Block));
  auto kernel = bf16 ? k_f8_tile<__nv_bfloat16> : k_f8_tile<float>;
  return cuda_fail(launch_behind(kernel, grid, kF8TileThreads, 0, st, a, vec),
                   "FP8 quantizer launch");
}

fqt_status fp8_matmul(const fqt_fp8 *A, const fqt_fp8 *B, bool bf16, void *out, int64_t ldo,
                      void *ws, cudaStream_t st) {
  const int64_t M = A->rows, N = B->rows, K = A->cols;
  const int nsm = device_sm_count();
  const F8Plan p = f8_plan(M, N, (K + kF8Block - 1) / kF8Block, nsm);
  const fqt_fp8 *a = p.swap ? B : A, *b = p.swap ? A : B;
  F8Args g = {};
  g.ldo = M > 1 ? ldo : N;
  // (TMA's stores end at 16 bytes, not at the last column of wider rows)
  g.boxes = !p.swap && p.splits == 1 && f8_aligned(out, 16) &&
            g.ldo * (bf16 ? 2 : 4) % 16 == 0 && N * (bf16 ? 2 : 4) % 16 == 0;
  CUtensorMap ta, tb, to = {};
  if (!make_map_codes(&ta, a, BM) || !make_map_codes(&tb, b, (uint32_t)(p.pair ? p.nt / 2 : p.nt)) ||
      (g.boxes && !make_map_f8_out(&to, out, bf16, M, N, g.ldo)))
    return cuda_fail(cudaErrorUnknown, "FP8 tensor map");
  g.sa = reinterpret_cast<const uint32_t *>(a->scales);
  g.sb = reinterpret_cast<const uint32_t *>(b->scales);
  g.spa = scale_rows(a->rows);
  g.spb = scale_rows(b->rows);
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
  g.status = static_cast<int *>(ws);
  if (p.pair) return launch_f8<256, 1, true>(ta, tb, to, g, nsm, st);
  if (p.nt == 128) return launch_f8<128, 2, false>(ta, tb, to, g, nsm, st);
  if (p.nt == 64) return launch_f8<64, 2, false>(ta, tb, to, g, nsm, st);
  return launch_f8<32, 2, false>(ta, tb, to, g, nsm, st);
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
  // the status word (tiles whose K blocks are shared meet in shared memory)
  (void)M, (void)N, (void)K;
  return kHeaderBytes;
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
  if (!workspace || !f8_aligned(workspace, 256) || ws_bytes < fqt_fp8_matmul_workspace_size(M, N, K))
    return FQT_EWORKSPACE;
  return fp8_matmul(A, B, dtype == FQT_BF16, out, ldo, workspace, st);
}

}  // extern "C"
