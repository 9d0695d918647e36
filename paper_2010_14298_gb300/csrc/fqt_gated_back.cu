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
  int64_t row_tiles, tiles;
  int *status;
};

// E4M3 codes 2 i and 2 i + 1 of a word as fp32, exact in fp16 on the way.
__device__ __forceinline__ f32x2 f8_two(uint32_t w, int i) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)(w >> 16 * i)));
  const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h));
  return pack2(f.x, f.y);
}
__device__ __forceinline__ f32x2 both(float v) { return pack2(v, v); }
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
// 2^shift lanes take 8 columns each of a row, a thread 4 rows (on their way at once).  VEC:
// the 8 columns are neighbours in 16-byte accesses; else a lane's columns are 2^shift apart,
// neighbouring lanes' are neighbours, and a thread takes 2 rows (registers).
template <bool VEC>
constexpr int kBackRows = VEC ? 4 : 2;

template <typename T, int ACT, bool VEC>
__global__ void __launch_bounds__(256) k_f8_gated_back_dense(const F8BackArgs a, const int shift) {
  constexpr int R = kBackRows<VEC>;
  let_next_start();
  wait_for_previous();
  const int lanes = 1 << shift, lane = threadIdx.x & (lanes - 1);
  const int64_t row0 = ((int64_t)blockIdx.x * R * 256 + threadIdx.x) >> shift;
  const int64_t c0 = ((int64_t)blockIdx.y * lanes + (VEC ? lane : 0)) * 8;
  const int step = 256 >> shift;  // rows between a thread's
  auto col = [&](int j) { return VEC ? c0 + j : c0 + lane + (int64_t)lanes * j; };
  if (col(0) >= a.cols) return;
  F8Raw<T, 8> da[R];
  uint2 cg[R], cu[R];
  uint8_t sg[R][VEC ? 1 : 8], su[R][VEC ? 1 : 8];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int64_t row = row0 + r * step;
    const bool in = row < a.rows;
    if constexpr (VEC) {
      da[r].load(static_cast<const T *>(a.da) + row * a.ldda + c0, in ? a.cols - c0 : 0);
      // (codes past the last column are in the row's 16 bytes; theirs are not stored)
      cg[r] = in ? __ldg(reinterpret_cast<const uint2 *>(a.gate.codes + row * a.gate.pitch + c0))
                 : make_uint2(0u, 0u);
      cu[r] = in ? __ldg(reinterpret_cast<const uint2 *>(a.up.codes + row * a.up.pitch + c0))
                 : make_uint2(0u, 0u);
      const int64_t at = in ? scale_at(c0 / kF8Block, a.sp, row) : 0;
      sg[r][0] = __ldg(a.gate.scales + at);
      su[r][0] = __ldg(a.up.scales + at);
    } else {
      uint32_t g[2] = {0u, 0u}, u[2] = {0u, 0u};
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const bool there = in && col(j) < a.cols;
        da[r].set(j, there ? static_cast<const T *>(a.da)[row * a.ldda + col(j)] : (T)0.0f);
        if (there) {
          g[j / 4] |= (uint32_t)__ldg(a.gate.codes + row * a.gate.pitch + col(j)) << 8 * (j % 4);
          u[j / 4] |= (uint32_t)__ldg(a.up.codes + row * a.up.pitch + col(j)) << 8 * (j % 4);
        }
        const int64_t at = there ? scale_at(col(j) / kF8Block, a.sp, row) : 0;
        sg[r][j] = __ldg(a.gate.scales + at);
        su[r][j] = __ldg(a.up.scales + at);
      }
      cg[r] = make_uint2(g[0], g[1]);
      cu[r] = make_uint2(u[0], u[1]);
    }
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int64_t row = row0 + r * step;
    if (row >= a.rows) return;
    uint32_t v[2][8];
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
      const f32x2 g = f8_two(j < 4 ? cg[r].x : cg[r].y, (j >> 1) & 1);
      const f32x2 u = f8_two(j < 4 ? cu[r].x : cu[r].y, (j >> 1) & 1);
      f32x2 dg, du, unused;
      if constexpr (VEC) {
        back_two<ACT>(pack2(da[r].f(j), da[r].f(j + 1)), g, u, f8_scale_of(sg[r][0]),
                      f8_scale_of(su[r][0]), dg, du, unused);
      } else {  // two columns of blocks of their own
        const f32x2 g2 = mul2(g, pack2(f8_scale_of(sg[r][j]), f8_scale_of(sg[r][j + 1])));
        const f32x2 u2 = mul2(u, pack2(f8_scale_of(su[r][j]), f8_scale_of(su[r][j + 1])));
        back_two<ACT>(pack2(da[r].f(j), da[r].f(j + 1)), g2, u2, 1.0f, 1.0f, dg, du, unused);
      }
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
      if (VEC && c0 + 8 <= a.cols) {
#pragma unroll
        for (int j = 0; j < 8; j += 16 / (int)sizeof(T))
          *reinterpret_cast<uint4 *>(out + c0 + j) = f8_pack<T>(&v[k][j]);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (col(j) < a.cols) out[col(j)] = f8_out<T>(__uint_as_float(v[k][j]));
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Codes
// ---------------------------------------------------------------------------
// One persistent CTA an SM over 128 x 128 tiles.  A thread holds 4 rows x 8 columns of dg, du
// and a in registers (96 of them), so it packs codes along either axis without exchanging
// bytes; what it reads (da, both codes and their scales: 65 or 97 KB a tile) comes ahead of
// time into shared memory by TMA, two tiles deep for bf16, one for fp32, so that loads run
// under the arithmetic of the tile before.
constexpr int kF8BackThreads = 512, kF8BackWarps = kF8BackThreads / 32;

template <typename T>
struct F8BackShared {
  static constexpr int stages = sizeof(T) == 2 ? 2 : 1;
  struct Stage {
    T da[kF8Block * kF8Block];
    uint8_t gate[kF8Block * kF8Block], up[kF8Block * kF8Block];
    uint32_t sg[kF8Block], su[kF8Block];  // four blocks' scales of a row, one of them the tile's
  } in[stages];
  // a column's 32 words of 4 rows' codes, word w at place w ^ 2 (column / 8): a warp's
  // threads, 16 columns 8 apart x 2 words, write 32 banks
  uint32_t tr[3][kF8Block * 32];
  uint32_t top[3][kF8BackWarps][kF8Block];  // column maxima by warp
  float inv[3][kF8Block];                   // and what a column's entries are multiplied by
  uint64_t full[stages];
};

struct F8BackMaps {
  CUtensorMap da, gate, up;
};

// The larger of m and |x|, |y| (NaN if one is).
__device__ __forceinline__ float top2(float m, f32x2 v) {
  float x, y, r;
  unpack2(v, x, y);
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(m), "f"(x), "f"(y));
  return r;
}
__device__ __forceinline__ float top3(float a, float b, float c) {
  float r;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ bool is_odd(float top) { return __float_as_uint(top) >= 0x7F800000u; }

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
                                           F8BackShared<T> &s, int stage, int64_t tile, bool vec) {
  const int64_t ct = tile / a.row_tiles, rt = tile - ct * a.row_tiles;
  auto &in = s.in[stage];
  uint64_t *bar = &s.full[stage];
  mbar_expect_tx(bar, (uint32_t)((vec ? sizeof(in.da) : 0) + sizeof(in.gate) + sizeof(in.up) +
                                 sizeof(in.sg) + sizeof(in.su)));
  const int32_t r0 = (int32_t)(rt * kF8Block), c0 = (int32_t)(ct * kF8Block);
  if (vec) tma_load_2d(in.da, &maps.da, c0, r0, bar);
  tma_load_2d(in.gate, &maps.gate, c0, r0, bar);
  tma_load_2d(in.up, &maps.up, c0, r0, bar);
  const int64_t at = ((ct >> 2) * a.sp + r0) * 4;
  bulk_load(in.sg, a.gate.scales + at, sizeof(in.sg), bar);
  bulk_load(in.su, a.up.scales + at, sizeof(in.su), bar);
}

template <typename T, int ACT>
__global__ void __launch_bounds__(kF8BackThreads, 1)
    k_f8_gated_back(const __grid_constant__ F8BackMaps maps, const F8BackArgs a, const bool vec) {
  extern __shared__ __align__(1024) uint8_t raw[];
  F8BackShared<T> &s = *reinterpret_cast<F8BackShared<T> *>(raw);
  constexpr int S = F8BackShared<T>::stages;
  let_next_start();
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  const int cg = t & 15, rg = t >> 4;  // its 8 columns and its 4 rows
  if (t == 0) {
    for (int i = 0; i < S; ++i) mbar_init(&s.full[i], 1);
    fence_barrier_init();
  }
  __syncthreads();
  wait_for_previous();
  if (t == 0)
    for (int i = 0; i < S; ++i)
      if (blockIdx.x + (int64_t)i * gridDim.x < a.tiles)
        back_fetch(maps, a, s, i, blockIdx.x + (int64_t)i * gridDim.x, vec);
  const bool by_rows = a.q[0].codes || a.q[1].codes;
  int n = 0;
  bool ok = true;
  for (int64_t tile = blockIdx.x; tile < a.tiles; tile += gridDim.x, ++n) {
    const int64_t ct = tile / a.row_tiles, rt = tile - ct * a.row_tiles;
    const int64_t r0 = rt * kF8Block, c0 = ct * kF8Block;
    const int64_t row = r0 + rg * 4, col = c0 + cg * 8;
    auto &in = s.in[n % S];
    if (!vec) {  // the warp's 8 rows, entry by entry, but neighbouring lanes read neighbours
      T e[8][kF8Block / 32];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int64_t r = r0 + warp * 8 + i;
        f8_fetch<T, kF8Block>(e[i], static_cast<const T *>(a.da) + r * a.ldda + c0,
                              r < a.rows ? a.cols - c0 : 0, lane);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i)
        f8_put<T, kF8Block>(in.da + (warp * 8 + i) * kF8Block, e[i], lane);
      __syncwarp();
    }
    ok = f8_wait(&s.full[n % S], (n / S) & 1, a.status);
    f32x2 v[3][4][4];  // dg, du, a
    {
      const uint4 wg = *reinterpret_cast<const uint4 *>(&in.sg[rg * 4]);
      const uint4 wu = *reinterpret_cast<const uint4 *>(&in.su[rg * 4]);
      const uint32_t sg[4] = {wg.x, wg.y, wg.z, wg.w}, su[4] = {wu.x, wu.y, wu.z, wu.w};
      const int byte = 8 * (int)(ct & 3);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int at = (rg * 4 + i) * kF8Block + cg * 8;
        F8Raw<T, 8> da;
        da.take(in.da + at);
        const uint2 g = *reinterpret_cast<const uint2 *>(in.gate + at);
        const uint2 u = *reinterpret_cast<const uint2 *>(in.up + at);
        // (rows past the end: zeros, whatever their scale)
        const bool there = row + i < a.rows;
        const float fg = there ? f8_scale_of(sg[i] >> byte & 255u) : 1.0f;
        const float fu = there ? f8_scale_of(su[i] >> byte & 255u) : 1.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j)
          back_two<ACT>(pack2(da.f(2 * j), da.f(2 * j + 1)), f8_two(j < 2 ? g.x : g.y, j & 1),
                        f8_two(j < 2 ? u.x : u.y, j & 1), fg, fu, v[0][i][j], v[1][i][j],
                        v[2][i][j]);
      }
    }
    // dense outputs
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      T *out = static_cast<T *>(k ? a.dup : a.dgate);
      if (!out) continue;
      const int64_t ld = k ? a.lddu : a.lddg;
      const bool wide = f8_pitch_aligned<T>(out, ld) && col + 8 <= a.cols;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (row + i >= a.rows) break;
        uint32_t x[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float lo, hi;
          unpack2(v[k][i][j], lo, hi);
          x[2 * j] = __float_as_uint(lo), x[2 * j + 1] = __float_as_uint(hi);
        }
        T *p = out + (row + i) * ld + col;
        if (wide) {
#pragma unroll
          for (int j = 0; j < 8; j += 16 / (int)sizeof(T))
            *reinterpret_cast<uint4 *>(p + j) = f8_pack<T>(&x[j]);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (col + j < a.cols) p[j] = f8_out<T>(__uint_as_float(x[j]));
        }
      }
    }
    // Maxima.  Entries that are not finite count for none and become NaN, whose code is
    // NaN's.
    float rm[8];  // of row i of dg (i) and of du (4 + i)
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      if (!a.qt[k].codes && (k == 2 || !a.q[k].codes)) {
        if (k < 2)
#pragma unroll
          for (int i = 0; i < 4; ++i) rm[4 * k + i] = 0.0f;
        continue;
      }
      float r[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        r[i] = top2(top2(top2(top2(0.0f, v[k][i][0]), v[k][i][1]), v[k][i][2]), v[k][i][3]);
      float cm[8];
      if (!is_odd(top3(top3(r[0], r[1], r[2]), r[3], 0.0f))) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float x[4], y[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) unpack2(v[k][i][j], x[i], y[i]);
          cm[2 * j] = top3(top3(x[0], x[1], x[2]), x[3], 0.0f);
          cm[2 * j + 1] = top3(top3(y[0], y[1], y[2]), y[3], 0.0f);
        }
      } else {
        record_status(a.status, FQT_ENONFINITE);
#pragma unroll
        for (int j = 0; j < 8; ++j) cm[j] = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          r[i] = 0.0f;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float x[2];
            unpack2(v[k][i][j], x[0], x[1]);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              if (is_odd(fabsf(x[h]))) {
                x[h] = __uint_as_float(0x7FFFFFFFu);
              } else {
                r[i] = fmaxf(r[i], fabsf(x[h]));
                cm[2 * j + h] = fmaxf(cm[2 * j + h], fabsf(x[h]));
              }
            }
            v[k][i][j] = pack2(x[0], x[1]);
          }
        }
      }
      if (k < 2)
#pragma unroll
        for (int i = 0; i < 4; ++i) rm[4 * k + i] = r[i];
      if (a.qt[k].codes) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          cm[j] = fmaxf(cm[j], __shfl_xor_sync(0xffffffffu, cm[j], 16));
        if (lane < 16) {
          float4 *to = reinterpret_cast<float4 *>(&s.top[k][warp][cg * 8]);
          to[0] = make_float4(cm[0], cm[1], cm[2], cm[3]);
          to[1] = make_float4(cm[4], cm[5], cm[6], cm[7]);
        }
      }
    }
    if (__syncthreads_or(!ok)) break;
    if (t == 0 && tile + (int64_t)S * gridDim.x < a.tiles)  // everybody has read the stage
      back_fetch(maps, a, s, n % S, tile + (int64_t)S * gridDim.x, vec);
    if (by_rows) {
      // The 8 maxima over the 16 lanes of a row group, halving what a lane holds: lane cg
      // ends with tensor cg / 8's row cg / 2 % 4, and hands its factor to the others.
      float m[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float keep = cg & 8 ? rm[4 + i] : rm[i], give = cg & 8 ? rm[i] : rm[4 + i];
        m[i] = fmaxf(keep, __shfl_xor_sync(0xffffffffu, give, 8));
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float keep = cg & 4 ? m[2 + i] : m[i], give = cg & 4 ? m[i] : m[2 + i];
        m[i] = fmaxf(keep, __shfl_xor_sync(0xffffffffu, give, 4));
      }
      const float keep = cg & 2 ? m[1] : m[0], give = cg & 2 ? m[0] : m[1];
      m[0] = fmaxf(keep, __shfl_xor_sync(0xffffffffu, give, 2));
      m[0] = fmaxf(m[0], __shfl_xor_sync(0xffffffffu, m[0], 1));
      const int e = f8_exponent(__float_as_uint(m[0]));
      const float inv = pow2(-e);
      const F8Codes &mine = a.q[cg >> 3];
      if (!(cg & 1) && mine.codes && row + (cg >> 1 & 3) < a.rows)
        mine.scales[scale_at(ct, a.sp, row + (cg >> 1 & 3))] = (uint8_t)(e + 127);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        uint8_t *to = a.q[k].codes + row * a.q[k].pitch + col;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f32x2 f = both(__shfl_sync(0xffffffffu, inv, (lane & 16) | k << 3 | i << 1));
          if (!a.q[k].codes || row + i >= a.rows || col >= a.cols) continue;
          uint32_t c[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float x, y;
            unpack2(mul2(v[k][i][j], f), x, y);
            c[j] = f8_pair(x, y);
          }
          *reinterpret_cast<uint2 *>(to + i * a.q[k].pitch) =
              make_uint2(c[0] | c[1] << 16, c[2] | c[3] << 16);
        }
      }
    }
    if (!a.qt[0].codes && !a.qt[1].codes && !a.qt[2].codes) continue;
    if (t < 3 * kF8Block && a.qt[t / kF8Block].codes) {
      const int k = t / kF8Block, j = t % kF8Block;
      uint32_t m = 0u;
#pragma unroll
      for (int w = 0; w < kF8BackWarps; ++w) m = max(m, s.top[k][w][j]);
      const int e = f8_exponent(m);
      s.inv[k][j] = pow2(-e);
      if (c0 + j < a.cols) a.qt[k].scales[scale_at(rt, a.spt, c0 + j)] = (uint8_t)(e + 127);
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      if (!a.qt[k].codes) continue;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 f = *reinterpret_cast<const float2 *>(&s.inv[k][cg * 8 + 2 * j]);
        float x[4], y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) unpack2(mul2(v[k][i][j], pack2(f.x, f.y)), x[i], y[i]);
        uint32_t *to = &s.tr[k][(cg * 8 + 2 * j) * 32 + (rg ^ (2 * cg))];
        to[0] = f8_pair(x[0], x[1]) | f8_pair(x[2], x[3]) << 16;
        to[32] = f8_pair(y[0], y[1]) | f8_pair(y[2], y[3]) << 16;
      }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      if (!a.qt[k].codes) continue;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int at = h * kF8BackThreads + t, j = at >> 3, ch = at & 7;
        if (c0 + j >= a.cols || r0 + ch * 16 >= a.rows) continue;
        const uint2 *pairs = reinterpret_cast<const uint2 *>(s.tr[k] + j * 32);
        const uint2 lo = pairs[(2 * ch) ^ (j >> 3)], hi = pairs[(2 * ch + 1) ^ (j >> 3)];
        *reinterpret_cast<uint4 *>(a.qt[k].codes + (c0 + j) * a.qt[k].pitch + r0 + ch * 16) =
            make_uint4(lo.x, lo.y, hi.x, hi.y);
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
  bool codes = false;
  for (const F8Codes &c : a.q) codes |= c.codes != nullptr;
  for (const F8Codes &c : a.qt) codes |= c.codes != nullptr;
  if (!codes) {
    const bool wide = vec && (!a.dgate || f8_pitch_aligned<T>(a.dgate, a.lddg)) &&
                      (!a.dup || f8_pitch_aligned<T>(a.dup, a.lddu));
    const int64_t chunks = ((int64_t)a.cols + 7) / 8;
    int shift = 0;
    while (shift < 5 && ((int64_t)1 << shift) < chunks) ++shift;
    const int64_t rows = (int64_t)(wide ? kBackRows<true> : kBackRows<false>) * 256 >> shift;
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
  a.row_tiles = (a.rows + kF8Block - 1) / kF8Block;
  a.tiles = a.row_tiles * (((int64_t)a.cols + kF8Block - 1) / kF8Block);
  auto kernel = k_f8_gated_back<T, ACT>;
  static DeviceOnce once;
  const cudaError_t e = allow_smem(kernel, sizeof(F8BackShared<T>), once);
  if (e != cudaSuccess) return cuda_fail(e, "gated backward attribute");
  const dim3 grid((unsigned)std::min<int64_t>(a.tiles, device_sm_count()));
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
    if (dgate && dgate == dup) return FQT_EINVAL;
    if (!codes_fit(qgate, rows, cols) || !codes_fit(qup, rows, cols) ||
        !codes_fit(qgate_t, cols, rows) || !codes_fit(qup_t, cols, rows) ||
        !codes_fit(product_t, cols, rows) || !all_apart({qgate, qup, qgate_t, qup_t, product_t}))
      return FQT_EINVAL;
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
