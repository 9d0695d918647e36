// fqt_gated_back.cu -- the backward pass of a = act(g) u from g and u held in 8 bits:
// dg = da u act'(g), du = da act(g), densely or as codes along both axes, and a's codes
// along the tokens.
#include "fqt_gated.cuh"

namespace fqt {

struct F8BackArgs {
  const void *da;
  int64_t ldda, rows;
  int cols;
  F8Codes gate, up;  // read
  int64_t sp, spt;   // rows of scales, of matrices and of their transposes
  void *dgate, *dup;
  int64_t lddg, lddu;
  F8Codes q[2], qt[3];  // dg, du; their transposes and a's
  int row_tiles, tiles;  // (rows and columns pass 2^22 by no more than a tile, tiles 2^30)
  int *status;
};

// E4M3 codes 2 i and 2 i + 1 of a word as fp32, exact in fp16 on the way.
__device__ __forceinline__ f32x2 f8_two(uint32_t w, int i) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)(w >> 16 * i)));
  const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h));
  return pack2(f.x, f.y);
}
__device__ __forceinline__ float f8_scale_of(uint32_t e) { return pow2((int)e - 127); }

// Two columns: dg, du and a from da and the codes' values (before their scales).
template <int ACT>
__device__ __forceinline__ void back_two(f32x2 da, f32x2 g, f32x2 u, float sg, float su, f32x2 &dg,
                                         f32x2 &du, f32x2 &a) {
  f32x2 act, slope;
  act_and_slope2<ACT>(mul2(g, both(sg)), act, slope);
  u = mul2(u, both(su));
  dg = mul2(mul2(da, u), slope);
  du = mul2(da, act);
  a = mul2(act, u);
}

// ---------------------------------------------------------------------------
// Dense outputs alone
// ---------------------------------------------------------------------------
// 2^shift lanes take 8 neighbouring columns each of a row, a thread 4 rows (on their way at
// once).  Rows of da or of an output that lie on no 16 bytes (WIDE false) go by way of shared
// memory: entry by entry, but neighbouring lanes' are neighbours.  Bound by memory traffic:
// 8192 x 4096 in bf16 43 us, 6.2 TB/s, in fp32 77, 6.1 TB/s.  8192 x 4095, which lies on no 16
// bytes, 61 and 92 (each lane its own 8 entries 187): every entry of da, dg and du is an access
// of its own, of 2 bytes in bf16, 38 instructions an entry for 25; the issue slots and the shared
// memory's wavefronts are at 54% each, memory at 47%.
constexpr int kBackRows = 4;

template <typename T, int ACT, bool WIDE>
__global__ void __launch_bounds__(256) k_f8_gated_back_dense(const F8BackArgs a, const int shift) {
  __shared__ __align__(16) T stage[WIDE ? 8 : 256 * 8];
  let_next_start();
  wait_for_previous();
  const int lanes = WIDE ? 1 << shift : 32, lane = threadIdx.x & (lanes - 1);
  const int64_t row0 = ((int64_t)blockIdx.x * kBackRows * 256 + threadIdx.x) >> shift;
  const int first = (int)blockIdx.y * lanes * 8, c0 = first + lane * 8;
  const int step = 256 >> shift;  // rows between a thread's
  T *group = stage + (WIDE ? 0 : (threadIdx.x / 32) * 256);
  const int left = a.cols - first - lane;  // (entry by entry) columns from the lane's first on
  F8Raw<T, 8> da[kBackRows];
  uint2 cg[kBackRows], cu[kBackRows];
  uint8_t sg[kBackRows], su[kBackRows];
  const bool any = c0 < a.cols;
#pragma unroll
  for (int r = 0; r < kBackRows; ++r) {
    const int64_t row = row0 + r * step;
    const bool in = row < a.rows && any;
    const T *p = static_cast<const T *>(a.da) + row * a.ldda;
    if constexpr (WIDE) {
      da[r].load(p + c0, in ? a.cols - c0 : 0);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        da[r].set(j, row < a.rows && 32 * j < left ? p[first + lane + 32 * j] : (T)0.0f);
      }
    }
    // (codes past the last column are in the row's 16 bytes; theirs are not stored)
    cg[r] = in ? __ldg(reinterpret_cast<const uint2 *>(a.gate.codes + row * a.gate.pitch + c0))
               : make_uint2(0u, 0u);
    cu[r] = in ? __ldg(reinterpret_cast<const uint2 *>(a.up.codes + row * a.up.pitch + c0))
               : make_uint2(0u, 0u);
    const int64_t at = in ? scale_at(c0 / kF8Block, a.sp, row) : 0;
    sg[r] = __ldg(a.gate.scales + at);
    su[r] = __ldg(a.up.scales + at);
  }
#pragma unroll
  for (int r = 0; r < kBackRows; ++r) {
    const int64_t row = row0 + r * step;
    if constexpr (!WIDE) {
#pragma unroll
      for (int j = 0; j < 8; ++j) group[lane + 32 * j] = da[r].entry(j);
      __syncwarp();
      da[r].take(group + lane * 8);
      __syncwarp();
    }
    uint32_t v[2][8];
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
      f32x2 dg, du, unused;
      back_two<ACT>(pack2(da[r].f(j), da[r].f(j + 1)), f8_two(j < 4 ? cg[r].x : cg[r].y, (j >> 1) & 1),
                    f8_two(j < 4 ? cu[r].x : cu[r].y, (j >> 1) & 1), f8_scale_of(sg[r]),
                    f8_scale_of(su[r]), dg, du, unused);
      float x, y;
      unpack2(dg, x, y);
      v[0][j] = __float_as_uint(x), v[0][j + 1] = __float_as_uint(y);
      unpack2(du, x, y);
      v[1][j] = __float_as_uint(x), v[1][j + 1] = __float_as_uint(y);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      T *out = static_cast<T *>(k ? a.dup : a.dgate);
      if (!out) continue;
      out += row * (k ? a.lddu : a.lddg);
      if constexpr (WIDE) {
        if (row >= a.rows) continue;
        if (c0 + 8 <= a.cols) {
#pragma unroll
          for (int j = 0; j < 8; j += 16 / (int)sizeof(T))
            *reinterpret_cast<uint4 *>(out + c0 + j) = f8_pack<T>(&v[k][j]);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (c0 + j < a.cols) out[c0 + j] = f8_out<T>(__uint_as_float(v[k][j]));
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; j += 16 / (int)sizeof(T))
          *reinterpret_cast<uint4 *>(group + lane * 8 + j) = f8_pack<T>(&v[k][j]);
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (row < a.rows && 32 * j < left) out[first + lane + 32 * j] = group[lane + 32 * j];
        __syncwarp();
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Codes
// ---------------------------------------------------------------------------
// One persistent CTA an SM over 128 x 128 tiles.  A warp takes 8 rows, a lane 4 columns of
// them, and holds dg, du and a of its 32 entries in registers (96).  So a row's maximum is one
// reduction of the warp, a column's needs no exchange within it, and a lane packs codes along
// either axis without exchanging bytes.  What the tile reads (da, both codes and their scales:
// 65 or 97 KB) comes ahead of time into shared memory by TMA, two tiles deep for bf16, one for
// fp32, so that loads run under the arithmetic of the tile before.
//
// 8192 x 4096 in bf16 70 us, in fp32 75 (4.3 TB/s; 302 MB take 45 us).  Not the loads bound it
// (they are there when a tile begins) but a tile's steps, one after the other: its 9800 cycles
// are values 2650, maxima 1500, the columns' scales and two barriers 900, codes 2800, the
// transposes' way out 2000.  Registers hold 16 warps an SM, which issue at 46% of the rate.
// (gelu_tanh 83 us, relu 66.)
// Rows' scales worked out by every lane took 23 of 63 instructions an entry (94 us), 4 rows x 8
// columns a thread with shuffles 90 us; spilled registers cost 11 us (39 instructions an entry
// now); rows' codes before the first barrier, or the transposes' way out along with the next
// tile's values, gained nothing in bf16 and lost 5 us in fp32.  Two CTAs an SM, each with half of a tile's rows and the columns' maxima exchanged in a
// cluster: 91 us (and as long as before where no columns are asked for, so it is the warps'
// own instructions that wait, four warps to a scheduler).
constexpr int kF8BackThreads = 512, kF8BackWarps = kF8BackThreads / 32;

template <typename T>
struct F8BackShared {
  static constexpr int stages = sizeof(T) == 2 ? 2 : 1;
  struct Stage {
    T da[kF8Block * kF8Block];
    uint8_t gate[kF8Block * kF8Block], up[kF8Block * kF8Block];
    uint32_t sg[kF8Block], su[kF8Block];  // four blocks' scales of a row, one of them the tile's
  } in[stages];
  uint2 tr[3][kF8Block * 16];  // a column's codes, 8 rows (a warp's) at a time: back_at
  float top[3][kF8BackWarps][kF8Block];  // column maxima by warp
  float inv[3][kF8Block];                // and what a column's entries are multiplied by
  // of a warp's 8 rows: the scales of g, then of u; the maxima of dg, then of du, and what
  // their entries are multiplied by
  float scale[kF8BackWarps][16];
  uint32_t row_top[kF8BackWarps][16];
  float row_inv[kF8BackWarps][16];
  uint64_t full[stages];
};

// The place of a warp's 8 codes of a column: half a warp's lanes (columns 4 apart) write 32
// banks, and half a warp that reads two columns' 16-byte chunks does, too.
__device__ __forceinline__ int back_at(int col, int warp) {
  return col * 16 + (warp ^ ((col >> 2 & 15) ^ (col & 1)));
}

struct F8BackMaps {
  CUtensorMap da, gate, up;
};

__device__ __forceinline__ float half_of(f32x2 v, int i) {
  float x, y;
  unpack2(v, x, y);
  return i ? y : x;
}
// Its magnitude, 0 if it is no finite number.
__device__ __forceinline__ float finite_of(f32x2 v, int i) {
  const float x = half_of(v, i);
  return is_odd(x) ? 0.0f : fabsf(x);
}

// Bytes (a multiple of 16, both ends on 16) into shared memory, counted by a barrier.
__device__ __forceinline__ void bulk_load(void *dst, const void *src, uint32_t bytes,
                                          uint64_t *bar) {
  asm volatile(
      "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
          smem_u32(dst)),
      "l"(src), "r"(bytes), "r"(smem_u32(bar))
      : "memory");
}

template <typename T>
__device__ __forceinline__ void back_fetch(const F8BackMaps &maps, const F8BackArgs &a,
                                           F8BackShared<T> &s, int stage, int tile, bool vec) {
  const int ct = tile / a.row_tiles, rt = tile - ct * a.row_tiles;
  auto &in = s.in[stage];
  uint64_t *bar = &s.full[stage];
  mbar_expect_tx(bar, (uint32_t)((vec ? sizeof(in.da) : 0) + sizeof(in.gate) + sizeof(in.up) +
                                 sizeof(in.sg) + sizeof(in.su)));
  const int r0 = rt * kF8Block, c0 = ct * kF8Block;
  if (vec) tma_load_2d(in.da, &maps.da, c0, r0, bar);
  tma_load_2d(in.gate, &maps.gate, c0, r0, bar);
  tma_load_2d(in.up, &maps.up, c0, r0, bar);
  const int64_t at = ((int64_t)(ct >> 2) * a.sp + r0) * 4;
  bulk_load(in.sg, a.gate.scales + at, sizeof(in.sg), bar);
  bulk_load(in.su, a.up.scales + at, sizeof(in.su), bar);
}

// ALL: the five matrices of codes, and no dense output (what a training step asks for).
template <typename T, int ACT, bool ALL>
__global__ void __launch_bounds__(kF8BackThreads, 1)
    k_f8_gated_back(const __grid_constant__ F8BackMaps maps, const F8BackArgs a, const bool vec) {
  extern __shared__ __align__(1024) uint8_t raw[];
  F8BackShared<T> &s = *reinterpret_cast<F8BackShared<T> *>(raw);
  constexpr int S = F8BackShared<T>::stages;
  // which outputs there are
  auto has_q = [&](int k) { return ALL || a.q[k].codes; };
  auto has_qt = [&](int k) { return ALL || a.qt[k].codes; };
  let_next_start();
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  if (t == 0) {
    for (int i = 0; i < S; ++i) mbar_init(&s.full[i], 1);
    fence_barrier_init();
  }
  __syncthreads();
  wait_for_previous();
  if (t == 0)
    for (int i = 0; i < S; ++i)
      if ((int)(blockIdx.x + i * gridDim.x) < a.tiles)
        back_fetch(maps, a, s, i, (int)(blockIdx.x + i * gridDim.x), vec);
  int n = 0;
  bool ok = true;
  for (int tile = (int)blockIdx.x; tile < a.tiles; tile += (int)gridDim.x, ++n) {
    const int ct = tile / a.row_tiles, rt = tile - ct * a.row_tiles;
    const int r0 = rt * kF8Block, c0 = ct * kF8Block;
    const int row = r0 + warp * 8, col = c0 + lane * 4;
    const int rows = min(8, (int)a.rows - row);  // of the warp's (it may have none)
    auto &in = s.in[n % S];
    if (!vec) {  // the warp's 8 rows, entry by entry, but neighbouring lanes read neighbours
      T e[8][kF8Block / 32];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int r = row + i;
        f8_fetch<T, kF8Block>(e[i], static_cast<const T *>(a.da) + (int64_t)r * a.ldda + c0,
                              r < a.rows ? a.cols - c0 : 0, lane);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i)
        f8_put<T, kF8Block>(in.da + (warp * 8 + i) * kF8Block, e[i], lane);
      __syncwarp();
    }
    ok = f8_wait(&s.full[n % S], (n / S) & 1, a.status);
    f32x2 v[3][8][2];  // dg, du, a
    {
      // lanes 0..7 prepare the scales of the warp's rows of g, lanes 8..15 of u (1 for rows past
      // the end, which are zeros)
      if (lane < 16) {
        const uint32_t w = (lane < 8 ? in.sg : in.su)[warp * 8 + (lane & 7)];
        s.scale[warp][lane] =
            (lane & 7) < rows ? f8_scale_of(w >> 8 * (int)(ct & 3) & 255u) : 1.0f;
      }
      __syncwarp();
      float4 fs[2];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (i % 4 == 0) {
          fs[0] = *reinterpret_cast<const float4 *>(&s.scale[warp][i]);
          fs[1] = *reinterpret_cast<const float4 *>(&s.scale[warp][8 + i]);
        }
        const int r = warp * 8 + i, at = r * kF8Block + lane * 4;
        f32x2 da[2];
        if constexpr (sizeof(T) == 4) {
          const float4 x = *reinterpret_cast<const float4 *>(in.da + at);
          da[0] = pack2(x.x, x.y), da[1] = pack2(x.z, x.w);
        } else {
          const uint2 x = *reinterpret_cast<const uint2 *>(in.da + at);
          da[0] = pack2(__uint_as_float(x.x << 16), __uint_as_float(x.x & 0xFFFF0000u));
          da[1] = pack2(__uint_as_float(x.y << 16), __uint_as_float(x.y & 0xFFFF0000u));
        }
        const uint32_t g = *reinterpret_cast<const uint32_t *>(in.gate + at);
        const uint32_t u = *reinterpret_cast<const uint32_t *>(in.up + at);
        const float fg = i % 4 == 0 ? fs[0].x : i % 4 == 1 ? fs[0].y : i % 4 == 2 ? fs[0].z : fs[0].w;
        const float fu = i % 4 == 0 ? fs[1].x : i % 4 == 1 ? fs[1].y : i % 4 == 2 ? fs[1].z : fs[1].w;
#pragma unroll
        for (int j = 0; j < 2; ++j)
          back_two<ACT>(da[j], f8_two(g, j), f8_two(u, j), fg, fu, v[0][i][j], v[1][i][j],
                        v[2][i][j]);
      }
    }
    // dense outputs
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      T *out = static_cast<T *>(k ? a.dup : a.dgate);
      if (ALL || !out) continue;
      const int64_t ld = k ? a.lddu : a.lddg;
      const bool wide = f8_pitch_aligned<T>(out, ld) && col + 4 <= a.cols;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (i >= rows) break;
        float x[4];
        unpack2(v[k][i][0], x[0], x[1]);
        unpack2(v[k][i][1], x[2], x[3]);
        T *p = out + (int64_t)(row + i) * ld + col;
        if (wide && sizeof(T) == 4) {
          *reinterpret_cast<float4 *>(p) = make_float4(x[0], x[1], x[2], x[3]);
        } else if (wide) {
          const __nv_bfloat162 lo = __floats2bfloat162_rn(x[0], x[1]);
          const __nv_bfloat162 hi = __floats2bfloat162_rn(x[2], x[3]);
          *reinterpret_cast<uint2 *>(p) = make_uint2(*reinterpret_cast<const uint32_t *>(&lo),
                                                     *reinterpret_cast<const uint32_t *>(&hi));
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (col + j < a.cols) p[j] = f8_out<T>(x[j]);
        }
      }
    }
    // Column maxima.  Entries that are not finite count for none; infinities' codes are put
    // right where they are written (v changes for none of this: the copies that the compiler
    // kept for two ways through cost 80 bytes of spilled registers).
    bool odd[3] = {false, false, false};
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      if (!has_qt(k) && (k == 2 || !has_q(k < 2 ? k : 0))) continue;
      float cm[4];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float x[8], y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) unpack2(v[k][i][j], x[i], y[i]);
        cm[2 * j] = top3(top3(top3(x[0], x[1], x[2]), x[3], x[4]), top3(x[5], x[6], x[7]), 0.0f);
        cm[2 * j + 1] = top3(top3(top3(y[0], y[1], y[2]), y[3], y[4]), top3(y[5], y[6], y[7]), 0.0f);
      }
      odd[k] = is_odd(top3(top3(cm[0], cm[1], cm[2]), cm[3], 0.0f));
      if (odd[k]) {
        record_status(a.status, FQT_ENONFINITE);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          cm[j] = 0.0f;
#pragma unroll
          for (int i = 0; i < 8; ++i) cm[j] = fmaxf(cm[j], finite_of(v[k][i][j / 2], j % 2));
        }
      }
      *reinterpret_cast<float4 *>(&s.top[k][warp][lane * 4]) =
          make_float4(cm[0], cm[1], cm[2], cm[3]);
    }
    // row maxima: lane c keeps row c % 8 of tensor c / 8
    if (has_q(0) || has_q(1)) {
      uint32_t mine = 0u;
#pragma unroll
      for (int c = 0; c < 16; ++c) {
        const f32x2(&x)[2] = v[c / 8][c % 8];
        float e[4], m;
        unpack2(x[0], e[0], e[1]);
        unpack2(x[1], e[2], e[3]);
        m = top3(top3(e[0], e[1], e[2]), e[3], 0.0f);
        if (odd[c / 8])
          m = top3(top3(finite_of(x[0], 0), finite_of(x[0], 1), finite_of(x[1], 0)),
                   finite_of(x[1], 1), 0.0f);
        const uint32_t r = __reduce_max_sync(0xffffffffu, __float_as_uint(m));
        if (lane == c) mine = r;
      }
      if (lane < 16) s.row_top[warp][lane] = mine;
    }
    if (__syncthreads_or(!ok)) break;
    // the scales: three quarters of the threads a column of one tensor each, the others two
    // rows; one of the others also asks for the next tile, as everybody has read this one's
    // stage
    if (t == kF8BackThreads - 1 && tile + S * (int)gridDim.x < a.tiles)
      back_fetch(maps, a, s, n % S, tile + S * (int)gridDim.x, vec);
    if (t < 3 * kF8Block && has_qt(t / kF8Block)) {
      const int k = t / kF8Block, j = t % kF8Block;
      float m = 0.0f;
#pragma unroll
      for (int w = 0; w < kF8BackWarps; w += 2) m = top3(m, s.top[k][w][j], s.top[k][w + 1][j]);
      const uint32_t e = f8_scale(__float_as_uint(m), s.inv[k][j]);
      if (c0 + j < a.cols) a.qt[k].scales[scale_at(rt, a.spt, c0 + j)] = (uint8_t)e;
    }
    if (t >= 3 * kF8Block) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int r = t - 3 * kF8Block;  // of the tile's
        if (!has_q(k)) continue;
        const uint32_t e = f8_scale(s.row_top[r / 8][k * 8 + r % 8], s.row_inv[r / 8][k * 8 + r % 8]);
        if (r0 + r < a.rows) a.q[k].scales[scale_at(ct, a.sp, r0 + r)] = (uint8_t)e;
      }
    }
    __syncthreads();
    const bool there = col < a.cols;
#pragma unroll
    for (int kk = 0; kk < 3; ++kk) {
      const int k = 2 - kk;  // a first, which has no rows
      if (has_qt(k)) {
        const float4 f = *reinterpret_cast<const float4 *>(&s.inv[k][lane * 4]);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const f32x2 f2 = j ? pack2(f.z, f.w) : pack2(f.x, f.y);
          float x[8], y[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) unpack2(mul2(v[k][i][j], f2), x[i], y[i]);
          s.tr[k][back_at(lane * 4 + 2 * j, warp)] =
              make_uint2(f8_four(x[0], x[1], x[2], x[3]), f8_four(x[4], x[5], x[6], x[7]));
          s.tr[k][back_at(lane * 4 + 2 * j + 1, warp)] =
              make_uint2(f8_four(y[0], y[1], y[2], y[3]), f8_four(y[4], y[5], y[6], y[7]));
        }
        if (odd[k])
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i)
              if (is_odd(half_of(v[k][i][j / 2], j % 2)))
                reinterpret_cast<uint8_t *>(&s.tr[k][back_at(lane * 4 + j, warp)])[i] = 0x7Fu;
      }
      if (k < 2 && has_q(k < 2 ? k : 0)) {
        const F8Codes &q = a.q[k < 2 ? k : 0];
        uint8_t *to = q.codes + (int64_t)row * q.pitch + col;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const f32x2 f = both(s.row_inv[warp][k * 8 + i]);
          float x[4];
          unpack2(mul2(v[k][i][0], f), x[0], x[1]);
          unpack2(mul2(v[k][i][1], f), x[2], x[3]);
          uint32_t code = f8_four(x[0], x[1], x[2], x[3]);
          if (odd[k])
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (is_odd(half_of(v[k][i][j / 2], j % 2))) code |= 0x7Fu << 8 * j;
          if (there && i < rows) *reinterpret_cast<uint32_t *>(to) = code;
          to += q.pitch;
        }
      }
    }
    if (!has_qt(0) && !has_qt(1) && !has_qt(2)) continue;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      if (!has_qt(k)) continue;
      const int j = t >> 3, ch = t & 7;
      const uint2 *from[2] = {&s.tr[k][back_at(j, 2 * ch)], &s.tr[k][back_at(j, 2 * ch + 1)]};
      uint8_t *to = a.qt[k].codes + (int64_t)(c0 + j) * a.qt[k].pitch + r0 + ch * 16;
#pragma unroll
      for (int h = 0; h < 2; ++h) {  // columns j and j + 64: the same places of their words
        const uint2 lo = from[0][64 * 16 * h], hi = from[1][64 * 16 * h];
        if (c0 + j + 64 * h < a.cols && r0 + ch * 16 < a.rows)
          *reinterpret_cast<uint4 *>(to) = make_uint4(lo.x, lo.y, hi.x, hi.y);
        to += 64 * a.qt[k].pitch;
      }
    }
  }
  if (!ok) sleep_ns(200000);  // copies in flight land before the CTA exits
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
// Boxes of 128 x 128 entries (the base and the pitch on 16 bytes).
static bool make_map_dense(CUtensorMap *m, const void *x, bool bf16, int64_t rows, int64_t cols,
                           int64_t ld) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  cuuint64_t strides[1] = {(cuuint64_t)ld * (bf16 ? 2 : 4)};
  cuuint32_t box[2] = {kF8Block, kF8Block};
  cuuint32_t one[2] = {1, 1};
  return fn(m, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 2,
            const_cast<void *>(x), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int ACT>
static fqt_status launch_back(F8BackArgs &a, const fqt_fp8 *gate, const fqt_fp8 *up,
                              cudaStream_t st) {
  const bool vec = f8_pitch_aligned<T>(a.da, a.ldda);
  bool codes = false, all = !a.dgate && !a.dup;
  for (const F8Codes &c : {a.q[0], a.q[1], a.qt[0], a.qt[1], a.qt[2]}) {
    codes |= c.codes != nullptr;
    all &= c.codes != nullptr;
  }
  if (!codes) {
    const bool wide = vec && (!a.dgate || f8_pitch_aligned<T>(a.dgate, a.lddg)) &&
                      (!a.dup || f8_pitch_aligned<T>(a.dup, a.lddu));
    const int64_t chunks = ((int64_t)a.cols + 7) / 8;
    int shift = 0;
    while (shift < 5 && (!wide || ((int64_t)1 << shift) < chunks)) ++shift;
    const int64_t rows = (int64_t)kBackRows * 256 >> shift;
    const dim3 grid((unsigned)((a.rows + rows - 1) / rows),
                    (unsigned)((chunks + (1 << shift) - 1) >> shift));
    auto kernel = wide ? k_f8_gated_back_dense<T, ACT, true> : k_f8_gated_back_dense<T, ACT, false>;
    return cuda_fail(launch_behind(kernel, grid, 256, 0, st, a, shift), "gated backward launch");
  }
  // (a tensor map's pitch is below 2^40 bytes)
  const bool ahead = vec && a.ldda < ((int64_t)1 << 40) / (int64_t)sizeof(T);
  F8BackMaps maps = {};
  if (!make_map_codes(&maps.gate, gate, kF8Block, false) ||
      !make_map_codes(&maps.up, up, kF8Block, false) ||
      (ahead && !make_map_dense(&maps.da, a.da, sizeof(T) == 2, a.rows, a.cols,
                              a.rows > 1 ? a.ldda : (a.cols + 7) / 8 * 8)))
    return cuda_fail(cudaErrorUnknown, "gated backward tensor map");
  a.row_tiles = (int)((a.rows + kF8Block - 1) / kF8Block);
  a.tiles = a.row_tiles * ((a.cols + kF8Block - 1) / kF8Block);
  auto kernel = all ? k_f8_gated_back<T, ACT, true> : k_f8_gated_back<T, ACT, false>;
  static DeviceOnce once[2];
  const cudaError_t e = allow_smem(kernel, sizeof(F8BackShared<T>), once[all]);
  if (e != cudaSuccess) return cuda_fail(e, "gated backward attribute");
  const dim3 grid((unsigned)std::min(a.tiles, device_sm_count()));
  return cuda_fail(launch_behind(kernel, grid, kF8BackThreads, sizeof(F8BackShared<T>), st, maps,
                                 (const F8BackArgs &)a, ahead),
                   "gated backward launch");
}

template <typename T>
static fqt_status launch_back(F8BackArgs &a, const fqt_fp8 *gate, const fqt_fp8 *up, fqt_act act,
                              cudaStream_t st) {
  switch (act) {
    case FQT_SILU: return launch_back<T, FQT_SILU>(a, gate, up, st);
    case FQT_GELU: return launch_back<T, FQT_GELU>(a, gate, up, st);
    case FQT_GELU_TANH: return launch_back<T, FQT_GELU_TANH>(a, gate, up, st);
    case FQT_RELU: return launch_back<T, FQT_RELU>(a, gate, up, st);
    default: return launch_back<T, FQT_SIGMOID>(a, gate, up, st);
  }
}

}  // namespace fqt

using namespace fqt;

extern "C" {

size_t fqt_fp8_gated_backward_workspace_size(int64_t rows, int64_t cols) {
  (void)rows, (void)cols;
  return kHeaderBytes;  // the status word
}

fqt_status fqt_fp8_gated_backward(const void *dA, int64_t ldda, fqt_dtype dtype,
                                  const fqt_fp8 *gate, const fqt_fp8 *up, fqt_act act, void *dgate,
                                  int64_t lddg, void *dup, int64_t lddu, fqt_fp8 *qgate,
                                  fqt_fp8 *qup, fqt_fp8 *qgate_t, fqt_fp8 *qup_t,
                                  fqt_fp8 *product_t, void *workspace, size_t ws_bytes,
                                  void *stream) {
  if (!gate || !up || (dtype != FQT_F32 && dtype != FQT_BF16) || !act_known(act))
    return FQT_EINVAL;
  const int64_t rows = gate->rows, cols = gate->cols;
  if (up->rows != rows || up->cols != cols || rows < 0 || cols <= 0 || rows > kF8MaxSize ||
      cols > kF8MaxSize)
    return FQT_EINVAL;
  // (blocks of 128 x 128 have their scale in every row's place)
  for (const fqt_fp8 *x : {gate, up})
    if (x->block_rows != 1 && x->block_rows != kF8Block) return FQT_EINVAL;
  if (rows > 0) {  // (an empty tensor's address may be NULL)
    if (!dgate && !dup && !qgate && !qup && !qgate_t && !qup_t && !product_t) return FQT_EINVAL;
    const size_t es = dtype == FQT_BF16 ? 2 : 4;
    const int64_t most = (int64_t)1 << 40;
    if (!f8_good(gate) || !f8_good(up)) return FQT_EINVAL;
    if (!dA || !f8_aligned(dA, es) || (rows > 1 && (ldda < cols || ldda > most))) return FQT_EINVAL;
    if (dgate && (!f8_aligned(dgate, es) || (rows > 1 && (lddg < cols || lddg > most))))
      return FQT_EINVAL;
    if (dup && (!f8_aligned(dup, es) || (rows > 1 && (lddu < cols || lddu > most))))
      return FQT_EINVAL;
    if (!codes_fit(qgate, rows, cols) || !codes_fit(qup, rows, cols) ||
        !codes_fit(qgate_t, cols, rows) || !codes_fit(qup_t, cols, rows) ||
        !codes_fit(product_t, cols, rows))
      return FQT_EINVAL;
    F8Apart apart;
    apart.writes(dgate, rows, cols, es, lddg);
    apart.writes(dup, rows, cols, es, lddu);
    for (const fqt_fp8 *x : {qgate, qup}) apart.writes(x, rows, cols);
    for (const fqt_fp8 *x : {qgate_t, qup_t, product_t}) apart.writes(x, cols, rows);
    apart.reads(dA, rows, cols, es, ldda);
    for (const fqt_fp8 *x : {gate, up}) apart.reads(x);
    if (!apart.ok()) return FQT_EINVAL;
    if (!workspace || !f8_aligned(workspace, 256) ||
        ws_bytes < fqt_fp8_gated_backward_workspace_size(rows, cols))
      return FQT_EWORKSPACE;
  }
  for (fqt_fp8 *x : {qgate, qup}) set_codes(x, rows, cols);
  for (fqt_fp8 *x : {qgate_t, qup_t, product_t}) set_codes(x, cols, rows);
  if (rows == 0) return FQT_OK;
  F8BackArgs a = {};
  a.da = dA;
  a.ldda = rows > 1 ? ldda : 0;
  a.rows = rows;
  a.cols = (int)cols;
  a.gate = codes_of(gate);
  a.up = codes_of(up);
  a.sp = scale_rows(rows);
  a.spt = scale_rows(cols);
  a.dgate = dgate;
  a.dup = dup;
  a.lddg = rows > 1 ? lddg : 0;
  a.lddu = rows > 1 ? lddu : 0;
  a.q[0] = codes_of(qgate);
  a.q[1] = codes_of(qup);
  a.qt[0] = codes_of(qgate_t);
  a.qt[1] = codes_of(qup_t);
  a.qt[2] = codes_of(product_t);
  a.status = static_cast<int *>(workspace);
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  return dtype == FQT_BF16 ? launch_back<__nv_bfloat16>(a, gate, up, act, st)
                           : launch_back<float>(a, gate, up, act, st);
}

}  // extern "C"
