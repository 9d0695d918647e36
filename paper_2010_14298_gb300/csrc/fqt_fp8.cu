// fqt_fp8.cu -- matrix products of 8-bit floating-point codes (E4M3) with one
// power-of-two scale for each block of 128 entries along the contraction, and their
// quantizer.
//
//   out_mn = sum_kb 2^(ea[kb][m] + eb[kb][n]) sum_(k in block kb) a_mk b_nk
#include "fqt_fp8_core.cuh"

namespace fqt {

// ---------------------------------------------------------------------------
// Quantizer
// ---------------------------------------------------------------------------
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
    float inv;
    // the four blocks' bytes, from lanes 0, 8, 16 and 24
    uint32_t w = f8_scale(m[r], inv) << (lane >> 3) * 8;
    w |= __shfl_xor_sync(0xffffffffu, w, 8);
    w |= __shfl_xor_sync(0xffffffffu, w, 16);
    if (row + r >= a.rows) continue;
    if (lane == 0) reinterpret_cast<uint32_t *>(a.s)[blockIdx.y * a.sp + row + r] = w;
    if (col >= a.cols) continue;
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
  uint32_t e_col = 0;
  float inv_col;
  if (t < kF8Block) {
    uint32_t m = 0u;
#pragma unroll
    for (int w = 0; w < kF8TileThreads / 32; ++w) m = max(m, cmax[w][t]);
    if (a.whole) {
      m = __reduce_max_sync(0xffffffffu, m);
      if (lane == 0) wmax[warp] = m;
    } else {
      e_col = f8_scale(m, cinv[t]);
    }
  }
  __syncthreads();
  if (a.whole) {
    const uint32_t m = max(max(wmax[0], wmax[1]), max(wmax[2], wmax[3]));
#pragma unroll
    for (int i = 0; i < 4; ++i) rm[i] = m;
    e_col = f8_scale(m, inv_col);
  }
  if (a.ct && t < kF8Block) a.st[scale_at(blockIdx.x, a.spt, c0 + t)] = (uint8_t)e_col;
  if (a.c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float inv;
      const uint32_t e = f8_scale(rm[i], inv);
      if (cg == 0) a.s[scale_at(blockIdx.y, a.sp, row + i)] = (uint8_t)e;
      if (row + i >= a.rows || col >= a.cols) continue;
      *reinterpret_cast<uint2 *>(a.c + (row + i) * a.pitch + col) =
          make_uint2(v[i].pair(0, inv) | v[i].pair(1, inv) << 16,
                     v[i].pair(2, inv) | v[i].pair(3, inv) << 16);
    }
  }
  if (a.ct) {
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
      float2 inv = *reinterpret_cast<const float2 *>(&cinv[cg * 8 + j]);
      if (a.whole) inv.x = inv.y = inv_col;
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

// The launch of a plan; fills what all kinds of products have in common.
template <int KIND>
static fqt_status launch_plan(const F8Plan &p, const fqt_fp8 *A, const fqt_fp8 *B, bool bf16,
                              void *out, int64_t ldo, int nkb, typename F8Of<KIND>::Maps &maps,
                              typename F8Of<KIND>::Args &g, int nsm, void *ws, cudaStream_t st) {
  const int64_t M = A->rows, N = B->rows;
  const fqt_fp8 *a = p.swap ? B : A, *b = p.swap ? A : B;
  g.ldo = M > 1 ? ldo : N;
  // (TMA's stores end at 16 bytes, not at the last column of wider rows)
  g.boxes = !p.swap && p.splits == 1 && f8_aligned(out, 16) &&
            g.ldo * (bf16 ? 2 : 4) % 16 == 0 && N * (bf16 ? 2 : 4) % 16 == 0;
  if (!make_map_codes(&maps.a, a, BM) ||
      !make_map_codes(&maps.b, b, (uint32_t)(p.pair ? p.nt / 2 : p.nt)) ||
      (g.boxes && !make_map_f8_out(&maps.out, out, bf16, M, N, g.ldo)))
    return cuda_fail(cudaErrorUnknown, "FP8 tensor map");
  g.sa = reinterpret_cast<const uint32_t *>(a->scales);
  g.sb = reinterpret_cast<const uint32_t *>(b->scales);
  g.spa = scale_rows(a->rows);
  g.spb = scale_rows(b->rows);
  g.M = a->rows;
  g.N = b->rows;
  g.nkb = nkb;
  g.m_tiles = p.m_tiles;
  g.n_tiles = p.n_tiles;
  g.splits = p.splits;
  g.kb_per = p.kb_per;
  g.items = (int64_t)p.m_tiles * p.n_tiles * p.splits;
  g.out = out;
  g.bf16 = bf16;
  g.swap = p.swap;
  g.status = static_cast<int *>(ws);
  if (p.pair) return launch_f8<256, 1, true, KIND>(maps, g, nsm, st);
  if (p.nt == 128) return launch_f8<128, 2, false, KIND>(maps, g, nsm, st);
  if (p.nt == 64) return launch_f8<64, 2, false, KIND>(maps, g, nsm, st);
  return launch_f8<32, 2, false, KIND>(maps, g, nsm, st);
}

static int64_t k_blocks(int64_t K) { return (K + kF8Block - 1) / kF8Block; }

fqt_status fp8_matmul(const fqt_fp8 *A, const fqt_fp8 *B, bool bf16, void *out, int64_t ldo,
                      void *ws, cudaStream_t st) {
  const int nsm = device_sm_count();
  const int64_t nkb = k_blocks(A->cols);
  const F8Plan p = f8_plan(A->rows, B->rows, nkb, nsm);
  F8Of<F8_ONE>::Maps maps = {};
  F8Args g = {};
  return launch_plan<F8_ONE>(p, A, B, bf16, out, ldo, (int)nkb, maps, g, nsm, ws, st);
}

// The K blocks of both pairs in one list, the second's from a group of scales on: the sums
// stay in one accumulator, so the second product adds no pass over the output.  8192 x 1024
// with K 4096 twice: 46 us, as one product of 8192 (3.0 PFLOP/s: 128 super tiles on 76 pairs
// are two rounds); two products of 4096 take 54 and need their outputs added.
fqt_status fp8_matmul_sum(const fqt_fp8 *A1, const fqt_fp8 *B1, const fqt_fp8 *A2,
                          const fqt_fp8 *B2, bool bf16, void *out, int64_t ldo, void *ws,
                          cudaStream_t st) {
  const int nsm = device_sm_count();
  F8SumArgs g = {};
  g.first = (int)k_blocks(A1->cols);
  g.second = (g.first + kF8Group - 1) / kF8Group * kF8Group;
  const int64_t nkb = g.second + k_blocks(A2->cols);
  const F8Plan p = f8_plan(A1->rows, B1->rows, nkb, nsm);
  const fqt_fp8 *a2 = p.swap ? B2 : A2, *b2 = p.swap ? A2 : B2;
  F8Of<F8_SUM>::Maps maps = {};
  if (!make_map_codes(&maps.a2, a2, BM) ||
      !make_map_codes(&maps.b2, b2, (uint32_t)(p.pair ? p.nt / 2 : p.nt)))
    return cuda_fail(cudaErrorUnknown, "FP8 tensor map");
  g.sa2 = reinterpret_cast<const uint32_t *>(a2->scales);
  g.sb2 = reinterpret_cast<const uint32_t *>(b2->scales);
  return launch_plan<F8_SUM>(p, A1, B1, bf16, out, ldo, (int)nkb, maps, g, nsm, ws, st);
}

}  // namespace fqt

using namespace fqt;

// A (M x K) and B (N x K) of a product, their sizes and kinds of blocks.
static bool f8_pair_fits(const fqt_fp8 *A, const fqt_fp8 *B) {
  for (const fqt_fp8 *q : {A, B})
    if (q->rows < 0 || q->cols < 0 || q->rows > kF8MaxSize || q->cols > kF8MaxSize ||
        (q->block_rows != 1 && q->block_rows != kF8Block))
      return false;
  return A->cols == B->cols;
}

static bool f8_out_fits(const void *out, int64_t ldo, fqt_dtype dtype, int64_t M, int64_t N) {
  return out && f8_aligned(out, dtype == FQT_BF16 ? 2 : 4) &&
         (M <= 1 || (ldo >= N && ldo <= ((int64_t)1 << 40)));
}

// an empty sum
static fqt_status f8_no_terms(void *out, int64_t ldo, fqt_dtype dtype, int64_t M, int64_t N,
                              cudaStream_t st) {
  const size_t es = dtype == FQT_BF16 ? 2 : 4;
  return cuda_fail(cudaMemset2DAsync(out, (M > 1 ? ldo : N) * es, 0, N * es, M, st),
                   "FP8 product clear");
}

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
  if (!f8_pair_fits(A, B)) return FQT_EINVAL;
  const int64_t M = A->rows, N = B->rows, K = A->cols;
  if (M == 0 || N == 0) return FQT_OK;
  if (!f8_out_fits(out, ldo, dtype, M, N)) return FQT_EINVAL;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  if (K == 0) return f8_no_terms(out, ldo, dtype, M, N, st);
  if (!f8_good(A) || !f8_good(B)) return FQT_EINVAL;
  if (!workspace || !f8_aligned(workspace, 256) || ws_bytes < fqt_fp8_matmul_workspace_size(M, N, K))
    return FQT_EWORKSPACE;
  return fp8_matmul(A, B, dtype == FQT_BF16, out, ldo, workspace, st);
}

size_t fqt_fp8_matmul_sum_workspace_size(int64_t M, int64_t N, int64_t K1, int64_t K2) {
  (void)M, (void)N, (void)K1, (void)K2;
  return kHeaderBytes;  // as one product's
}

fqt_status fqt_fp8_matmul_sum(const fqt_fp8 *A1, const fqt_fp8 *B1, const fqt_fp8 *A2,
                              const fqt_fp8 *B2, fqt_dtype dtype, void *out, int64_t ldo,
                              void *workspace, size_t ws_bytes, void *stream) {
  if (!A1 || !B1 || !A2 || !B2 || (dtype != FQT_F32 && dtype != FQT_BF16)) return FQT_EINVAL;
  if (!f8_pair_fits(A1, B1) || !f8_pair_fits(A2, B2)) return FQT_EINVAL;
  const int64_t M = A1->rows, N = B1->rows, K1 = A1->cols, K2 = A2->cols;
  if (A2->rows != M || B2->rows != N) return FQT_EINVAL;
  if (M == 0 || N == 0) return FQT_OK;
  if (!f8_out_fits(out, ldo, dtype, M, N)) return FQT_EINVAL;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  if (K1 == 0 && K2 == 0) return f8_no_terms(out, ldo, dtype, M, N, st);
  F8Apart apart;
  apart.writes(out, M, N, dtype == FQT_BF16 ? 2 : 4, ldo);
  for (const fqt_fp8 *q : {A1, B1, A2, B2}) {
    if (q->cols == 0) continue;
    if (!f8_good(q)) return FQT_EINVAL;
    apart.reads(q);
  }
  if (!apart.ok()) return FQT_EINVAL;
  if (!workspace || !f8_aligned(workspace, 256) ||
      ws_bytes < fqt_fp8_matmul_sum_workspace_size(M, N, K1, K2))
    return FQT_EWORKSPACE;
  const bool bf16 = dtype == FQT_BF16;
  if (K2 == 0) return fp8_matmul(A1, B1, bf16, out, ldo, workspace, st);
  if (K1 == 0) return fp8_matmul(A2, B2, bf16, out, ldo, workspace, st);
  return fp8_matmul_sum(A1, B1, A2, B2, bf16, out, ldo, workspace, st);
}

}  // extern "C"
