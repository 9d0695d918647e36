// fqt_norm.cu -- layer norm of the rows of a matrix, forward and backward, with
// the reductions of the scale's and the shift's gradients over all rows.
//
//   mean = sum x / n,  var = sum (x - mean)^2 / n,  rstd = (var + eps)^(-1/2)
//   y    = (x - mean) rstd gamma + beta
//   xh   = (x - mean) rstd,  g = dy gamma
//   dx   = rstd (g - sum(g) / n - xh sum(g xh) / n)
//   dgamma = sum over rows of dy xh,  dbeta = sum over rows of dy
//
// Both directions are bound by memory traffic (8 and 14 operations per entry
// against 4 and 6 bytes of bf16), so a row is read once and kept in registers by a
// group of threads wide enough to hold it: the group reduces the row's sums, and every
// thread then finishes the entries it holds.  A thread holds 16 entries of a row (the
// forward 32 where it can) and keeps its columns from row to row: fewer leave the
// reductions' shuffles and the addresses to too few entries, and with more gamma and beta
// (in the backward the column sums too) no longer fit the registers, and reading them
// again for every row took as many wavefronts of the load/store pipe as the row itself.
// Rows are fetched ahead by cp.async: a thread copies the 16 bytes that it will read
// itself, so rows are on their way without registers and without barriers.  In the
// backward the columns' sums stay in registers.
// The variance is taken about the mean (a second reduction over registers), not from
// the sum of squares, which loses it where the mean is large.  All statistics and sums
// are fp32.
#include <cuda_runtime.h>
#include <math.h>

#include <algorithm>

#include "fqt.h"
#include "fqt_common.cuh"
#include "fqt_internal.h"

namespace fqt {

constexpr int kNormThreads = 512;   // of a CTA at most
constexpr int kNormMaxGroups = 16;  // of a warp each; 8 wider ones (named barriers 1 .. 8)

struct NormArgs {
  const void *x, *dy;
  void *y;  // Y, or dX (may be null)
  int64_t ldx, lddy, ldy;
  int64_t rows;
  int cols;
  const float *gamma, *beta;
  float *mean, *rstd;  // written by the forward (may be null), read by the backward
  float eps;
  float *part;  // backward: this many partial rows of 2 x cols sums, or null
  float *dgamma, *dbeta;
};

// V consecutive entries as they lie in memory (16 bytes, or one entry).
template <typename T, int V>
struct Pack {
  static constexpr int words = V * sizeof(T) >= 4 ? V * (int)sizeof(T) / 4 : 1;
  uint32_t w[words];
  __device__ __forceinline__ void load(const T *p) {
    if constexpr (words == 4) {
      const uint4 v = __ldg(reinterpret_cast<const uint4 *>(p));
      w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    } else if constexpr (sizeof(T) == 4) {
      w[0] = __ldg(reinterpret_cast<const unsigned *>(p));
    } else {
      w[0] = __ldg(reinterpret_cast<const unsigned short *>(p));
    }
  }
  __device__ __forceinline__ void take(const uint4 &v) {
    if constexpr (words == 4) {
      w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < words; ++i) w[i] = 0u;
  }
  __device__ __forceinline__ float f(int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
    else return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
  }
};

template <typename T, int V>
__device__ __forceinline__ void store_pack(T *p, const float *v) {
  if constexpr (V == 4) {
    *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
  } else if constexpr (V == 8) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t *>(&b);
    }
    *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  } else {
    *p = (T)v[0];
  }
}

// Two entries, in bf16 rows with one instruction for both: there the conversions leave
// the arithmetic too few issue slots (with 16 entries a thread, 16384 x 768 forward 12.6 us
// and 13.1 without pairs, backward 17.6 and 19.7). fp32 rows are bound by memory (8192 x
// 8192 forward 80 us, with pairs 85).
template <bool PACKED>
struct Two {
  float a, b;
  static __device__ __forceinline__ Two of(float a, float b) { return {a, b}; }
  __device__ __forceinline__ float2 get() const { return make_float2(a, b); }
};
template <>
struct Two<true> {
  f32x2 v;
  static __device__ __forceinline__ Two of(float a, float b) { return {pack2(a, b)}; }
  __device__ __forceinline__ float2 get() const {
    float2 f;
    unpack2(v, f.x, f.y);
    return f;
  }
};
template <bool P>
__device__ __forceinline__ Two<P> operator+(Two<P> x, Two<P> y) {
  if constexpr (P) return {add2(x.v, y.v)};
  else return {x.a + y.a, x.b + y.b};
}
template <bool P>
__device__ __forceinline__ Two<P> operator*(Two<P> x, Two<P> y) {
  if constexpr (P) return {mul2(x.v, y.v)};
  else return {x.a * y.a, x.b * y.b};
}
template <bool P>
__device__ __forceinline__ Two<P> fma(Two<P> x, Two<P> y, Two<P> z) {
  if constexpr (P) return {fma2(x.v, y.v, z.v)};
  else return {fmaf(x.a, y.a, z.a), fmaf(x.b, y.b, z.b)};
}
// Sums of entries and of products (in one register where the entries are not packed).
template <bool P>
__device__ __forceinline__ void add_to(Two<P> &all, Two<P> x) {
  if constexpr (P) all.v = add2(all.v, x.v);
  else all.a = (all.a + x.a) + x.b;
}
template <bool P>
__device__ __forceinline__ void add_to(Two<P> &all, Two<P> x, Two<P> y) {
  if constexpr (P) all.v = fma2(x.v, y.v, all.v);
  else all.a = fmaf(x.b, y.b, fmaf(x.a, y.a, all.a));
}
template <bool P>
__device__ __forceinline__ float sum(Two<P> x) {
  if constexpr (!P) return x.a;
  const float2 f = x.get();
  return f.x + f.y;
}

// This thread's entries of a vector of `cols` floats: V from every column (j G + t) V
// on; `none` where the vector or the column is missing.
template <int V, int VPT>
__device__ __forceinline__ void load_columns(const float *p, int cols, int G, int t, float none,
                                             float (&v)[V * VPT]) {
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const int c = (j * G + t) * V;
    if (!p || c >= cols) {
#pragma unroll
      for (int i = 0; i < V; ++i) v[j * V + i] = none;
    } else if constexpr (V == 1) {
      v[j] = __ldg(p + c);
    } else {
#pragma unroll
      for (int i = 0; i < V; i += 4) {
        const float4 f = __ldg(reinterpret_cast<const float4 *>(p + c + i));
        v[j * V + i] = f.x; v[j * V + i + 1] = f.y; v[j * V + i + 2] = f.z; v[j * V + i + 3] = f.w;
      }
    }
  }
}

template <int V, int VPT>
__device__ __forceinline__ void load_columns(const float *p, int cols, int G, int t, float none,
                                             Two<V == 8> (&v)[V * VPT / 2]) {
  float f[V * VPT];
  load_columns<V, VPT>(p, cols, G, t, none, f);
#pragma unroll
  for (int i = 0; i < V * VPT / 2; ++i) v[i] = Two<V == 8>::of(f[2 * i], f[2 * i + 1]);
}

// Sums of a value (two values) over the threads of a group (G threads from a warp
// boundary, G a multiple of 32, at most 16 warps), in every thread, in an order that
// does not change.  slot: 32 floats of the group; a call must not follow another on the
// same slot without a barrier of the group between the reads and the writes, so callers
// alternate slots.
__device__ __forceinline__ float group_sum(float v, float *slot, int G, int gid, int gw,
                                           int lane) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if (G == 32) return v;
  if (lane == 0) slot[gw] = v;
  asm volatile("bar.sync %0, %1;" ::"r"(1 + gid), "r"(G) : "memory");
  // every warp adds the warps' sums by itself
  v = lane < (G >> 5) ? slot[lane] : 0.0f;
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return __shfl_sync(0xffffffffu, v, 0);
}

// (The first value is summed in the lower half of the lanes, the second in the upper.)
__device__ __forceinline__ float2 group_sum2(float a, float b, float *slot, int G, int gid,
                                             int gw, int lane) {
  const bool up = lane & 16;
  float v = (up ? b : a) + __shfl_xor_sync(0xffffffffu, up ? a : b, 16);
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if (G > 32) {
    if ((lane & 15) == 0) slot[(lane & 16) + gw] = v;
    asm volatile("bar.sync %0, %1;" ::"r"(1 + gid), "r"(G) : "memory");
    v = (lane & 15) < (G >> 5) ? slot[lane] : 0.0f;
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  }
  return make_float2(__shfl_sync(0xffffffffu, v, 0), __shfl_sync(0xffffffffu, v, 16));
}

template <int R>
__device__ __forceinline__ void group_sums(float (&s)[R], float *slot, int G, int gid, int gw,
                                           int lane) {
  static_assert(R == 1 || R == 2, "one or two sums");
  if constexpr (R == 1) {
    s[0] = group_sum(s[0], slot, G, gid, gw, lane);
  } else {
    const float2 v = group_sum2(s[0], s[1], slot, G, gid, gw, lane);
    s[0] = v.x;
    s[1] = v.y;
  }
}

// 16 bytes of this thread on their way to its place in shared memory.
__device__ __forceinline__ void copy16(void *dst, const void *src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(src)
               : "memory");
}
__device__ __forceinline__ void copy_commit() {
  asm volatile("cp.async.commit_group;" ::: "memory");
}
template <int N>
__device__ __forceinline__ void copy_wait() {  // all but the last N groups are there
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// Threads' 16-byte places in S stages of shared memory, `N` places of a row (or of
// two rows, X's and dY's) a stage.
template <int N>
struct NormRing {
  uint4 *base;
  __device__ __forceinline__ uint4 *at(int stage, int i) const {
    return base + (stage * N + i) * blockDim.x + threadIdx.x;
  }
};

// Forward.  S > 0: rows come through S stages of shared memory.  A group takes R rows
// at a time, whose sums share shuffles and barriers.  32768 x 4096 in bf16: 90 us, 6.0
// TB/s; in fp32 167 us, 6.4 TB/s; 8192 x 1024 in bf16 8.3 us on new rows, for a floor of
// 5, and 6.6 on rows that stay in L2 from call to call (a copy of as much takes 3.8 there).
template <typename T, int V, int VPT, int R, int S>
__global__ void __launch_bounds__(kNormThreads)
    k_norm_fwd(const NormArgs a, int G) {
  extern __shared__ __align__(16) uint4 smem[];
  __shared__ float slots[kNormMaxGroups][2][32];
  let_next_start();
  wait_for_previous();
  constexpr int E = V * VPT;
  using Pair = Two<V == 8>;
  static_assert(E % 2 == 0, "entries in pairs");
  const int gid = threadIdx.x / G, t = threadIdx.x - gid * G;
  const int lane = t & 31, gw = t >> 5, ngrp = blockDim.x / G;
  const int nvec = a.cols / V;
  const float n = (float)a.cols, inv = 1.0f / n;
  const NormRing<R * VPT> ring{smem};
  const int64_t step = (int64_t)gridDim.x * ngrp * R;
  const T *px = static_cast<const T *>(a.x) + (int64_t)t * V;
  auto fetch = [&](int stage, int64_t r0) {
#pragma unroll
    for (int k = 0; k < R; ++k)
      if (r0 + k < a.rows)
#pragma unroll
        for (int j = 0; j < VPT; ++j)
          if (j * G + t < nvec)
            copy16(ring.at(stage, k * VPT + j), px + (r0 + k) * a.ldx + (int64_t)j * G * V);
    copy_commit();
  };
  int64_t r0 = ((int64_t)blockIdx.x * ngrp + gid) * R;
  if constexpr (S > 0)
#pragma unroll
    for (int i = 0; i < S - 1; ++i) fetch(i, r0 + i * step);
  Pair ga[E / 2], be[E / 2];
  load_columns<V, VPT>(a.gamma, a.cols, G, t, 1.0f, ga);
  load_columns<V, VPT>(a.beta, a.cols, G, t, 0.0f, be);
  int stage = 0;
  for (; r0 < a.rows; r0 += step) {
    Pair d[R][E / 2];
    float mean[R];
    if constexpr (S > 0) {
      fetch(stage == 0 ? S - 1 : stage - 1, r0 + (S - 1) * step);
      copy_wait<S - 1>();
    }
    float s[R];
#pragma unroll
    for (int k = 0; k < R; ++k) {
      Pack<T, V> x[VPT];
#pragma unroll
      for (int j = 0; j < VPT; ++j) {
        if (r0 + k >= a.rows || j * G + t >= nvec) x[j].zero();
        else if constexpr (S > 0) x[j].take(*ring.at(stage, k * VPT + j));
        else x[j].load(px + (r0 + k) * a.ldx + (int64_t)j * G * V);
      }
      Pair all = Pair::of(0.0f, 0.0f);
#pragma unroll
      for (int i = 0; i < E; i += 2) {
        d[k][i / 2] = Pair::of(x[i / V].f(i % V), x[(i + 1) / V].f((i + 1) % V));
        add_to(all, d[k][i / 2]);
      }
      s[k] = sum(all);
    }
    if constexpr (S > 0) stage = stage == S - 1 ? 0 : stage + 1;
    group_sums<R>(s, slots[gid][0], G, gid, gw, lane);
#pragma unroll
    for (int k = 0; k < R; ++k) {
      // s / n: by the reciprocal, and corrected by the remainder (Markstein, IBM J. Res.
      // Dev. 34, 1990); a mean that is off, though by its last bit, shows in the variance
      // of a row of equal large entries
      const float m = s[k] * inv;
      mean[k] = fmaf(fmaf(-m, n, s[k]), inv, m);
      const Pair less = Pair::of(-mean[k], -mean[k]);
      Pair all = Pair::of(0.0f, 0.0f);
#pragma unroll
      for (int i = 0; i < E; i += 2) {
        Pair &x = d[k][i / 2];
        x = x + less;
        if constexpr (V == 1) {
          const float2 f = x.get();
          x = Pair::of(i * G + t < nvec ? f.x : 0.0f, (i + 1) * G + t < nvec ? f.y : 0.0f);
          add_to(all, x, x);
        } else if ((i / V) * G + t < nvec) {
          add_to(all, x, x);
        }
      }
      s[k] = sum(all);
    }
    group_sums<R>(s, slots[gid][1], G, gid, gw, lane);
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const float rstd = rsqrtf(fmaf(s[k], inv, a.eps));
      if (r0 + k >= a.rows) break;
      if (t == 0) {
        if (a.mean) a.mean[r0 + k] = mean[k];
        if (a.rstd) a.rstd[r0 + k] = rstd;
      }
      const Pair by = Pair::of(rstd, rstd);
      T *py = static_cast<T *>(a.y) + (r0 + k) * a.ldy + (int64_t)t * V;
#pragma unroll
      for (int j = 0; j < VPT; ++j) {
        if (j * G + t >= nvec) break;
        float y[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const int e = j * V + i;
          if (V > 1 && i % 2) continue;
          const float2 f = fma(d[k][e / 2] * by, ga[e / 2], be[e / 2]).get();
          if constexpr (V == 1) {
            y[0] = e % 2 ? f.y : f.x;
          } else {
            y[i] = f.x;
            y[i + 1] = f.y;
          }
        }
        store_pack<T, V>(py + (int64_t)j * G * V, y);
      }
    }
  }
}

// Backward.  The column sums of a group's rows stay in its registers; at the end the
// groups of a CTA add theirs in shared memory, and each CTA writes one row of partial
// sums (k_norm_cols adds those).  32768 x 4096 in bf16: 133 us with k_norm_cols, 6.0
// TB/s; in fp32 261 us, 6.2 TB/s; 8192 x 1024 in bf16 16.0 us on new rows, for a floor of
// 7.6, and 12.5 on rows that stay in L2 from call to call.
template <typename T, int V, int VPT, int S>
__global__ void __launch_bounds__(kNormThreads)
    k_norm_bwd(const NormArgs a, int G) {
  extern __shared__ __align__(16) uint4 smem[];
  __shared__ float slots[kNormMaxGroups][2][32];
  let_next_start();
  wait_for_previous();
  constexpr int E = V * VPT;
  using Pair = Two<V == 8>;
  const int gid = threadIdx.x / G, t = threadIdx.x - gid * G;
  const int lane = t & 31, gw = t >> 5, ngrp = blockDim.x / G;
  const int nvec = a.cols / V;
  const float n = (float)a.cols, inv = 1.0f / n;
  const NormRing<2 * VPT> ring{smem};
  const int64_t step = (int64_t)gridDim.x * ngrp;
  const T *px = static_cast<const T *>(a.x) + (int64_t)t * V;
  const T *pdy = static_cast<const T *>(a.dy) + (int64_t)t * V;
  auto fetch = [&](int stage, int64_t r) {
    if (r < a.rows)
#pragma unroll
      for (int j = 0; j < VPT; ++j)
        if (j * G + t < nvec) {
          copy16(ring.at(stage, 2 * j), px + r * a.ldx + (int64_t)j * G * V);
          copy16(ring.at(stage, 2 * j + 1), pdy + r * a.lddy + (int64_t)j * G * V);
        }
    copy_commit();
  };
  int64_t r = (int64_t)blockIdx.x * ngrp + gid;
  if constexpr (S > 0)
#pragma unroll
    for (int i = 0; i < S - 1; ++i) fetch(i, r + i * step);
  Pair ga[E / 2], dg[E / 2], db[E / 2];
  load_columns<V, VPT>(a.gamma, a.cols, G, t, 1.0f, ga);
#pragma unroll
  for (int i = 0; i < E / 2; ++i) dg[i] = db[i] = Pair::of(0.0f, 0.0f);
  // a row's statistics, one step ahead
  float mean_next = 0.0f, rstd_next = 0.0f;
  if (r < a.rows) {
    mean_next = __ldg(a.mean + r);
    rstd_next = __ldg(a.rstd + r);
  }
  int slot = 0, stage = 0;
  for (; r < a.rows; r += step, slot ^= 1) {
    Pack<T, V> x[VPT], dy[VPT];
    const float mean = mean_next, rstd = rstd_next;
    if constexpr (S > 0) {
      fetch(stage == 0 ? S - 1 : stage - 1, r + (S - 1) * step);
      copy_wait<S - 1>();
    }
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      if (j * G + t >= nvec) {
        x[j].zero();
        dy[j].zero();
      } else if constexpr (S > 0) {
        x[j].take(*ring.at(stage, 2 * j));
        dy[j].take(*ring.at(stage, 2 * j + 1));
      } else {
        x[j].load(px + r * a.ldx + (int64_t)j * G * V);
        dy[j].load(pdy + r * a.lddy + (int64_t)j * G * V);
      }
    }
    if constexpr (S > 0) stage = stage == S - 1 ? 0 : stage + 1;
    if (r + step < a.rows) {
      mean_next = __ldg(a.mean + r + step);
      rstd_next = __ldg(a.rstd + r + step);
    }
    // u = x - mean and g = dy gamma are kept for dx; a missing entry's dy is 0
    const Pair less = Pair::of(-mean, -mean), by = Pair::of(rstd, rstd);
    Pair u[E / 2], g[E / 2], all1 = Pair::of(0.0f, 0.0f), all2 = all1;
#pragma unroll
    for (int i = 0; i < E / 2; ++i) {
      const int j = 2 * i, k = 2 * i + 1;
      const Pair e = Pair::of(dy[j / V].f(j % V), dy[k / V].f(k % V));
      u[i] = Pair::of(x[j / V].f(j % V), x[k / V].f(k % V)) + less;
      g[i] = e * ga[i];
      add_to(all1, g[i]);
      add_to(all2, g[i], u[i]);
      dg[i] = fma(e * by, u[i], dg[i]);
      db[i] = db[i] + e;
    }
    if (!a.y) continue;
    const float2 s = group_sum2(sum(all1), sum(all2), slots[gid][slot], G, gid, gw, lane);
    // dx = rstd g - rstd sum(g) / n - (x - mean) rstd^3 sum(g (x - mean)) / n
    // (single entries divide: with the reciprocal 8192 x 1021 took 27 us, so 24)
    const float m1 = V == 1 ? s.x / n : s.x * inv, m2 = V == 1 ? s.y / n : s.y * inv;
    const float k0 = -rstd * m1, k1 = -rstd * (rstd * (rstd * m2));
    const Pair c0 = Pair::of(k0, k0), c1 = Pair::of(k1, k1);
    T *pdx = static_cast<T *>(a.y) + r * a.ldy + (int64_t)t * V;
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      if (j * G + t >= nvec) break;
      float o[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int e = j * V + i;
        if (V > 1 && i % 2) continue;
        const float2 f = fma(u[e / 2], c1, fma(g[e / 2], by, c0)).get();
        if constexpr (V == 1) {
          o[0] = e % 2 ? f.y : f.x;
        } else {
          o[i] = f.x;
          o[i + 1] = f.y;
        }
      }
      store_pack<T, V>(pdx + (int64_t)j * G * V, o);
    }
  }
  if (!a.part) return;
  // every thread's sums in shared memory, entry i of thread t of a group at i G + t;
  // then the groups' sums, from the first to the last
  float *sums = reinterpret_cast<float *>(smem);
  const int per = E * G;  // sums of a group: dgamma's, then dbeta's
  float *dst = a.part + (int64_t)blockIdx.x * 2 * a.cols;
  if (ngrp > 1 && S > 0) {
    copy_wait<0>();
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const int c = ((i / V) * G + t) * V + i % V;
    const float2 f = dg[i / 2].get(), h = db[i / 2].get();
    if (ngrp > 1) {
      sums[(2 * gid) * per + i * G + t] = i & 1 ? f.y : f.x;
      sums[(2 * gid + 1) * per + i * G + t] = i & 1 ? h.y : h.x;
    } else if (c < a.cols) {
      dst[c] = i & 1 ? f.y : f.x;
      dst[a.cols + c] = i & 1 ? h.y : h.x;
    }
  }
  if (ngrp == 1) return;
  __syncthreads();
  for (int k = threadIdx.x; k < per; k += blockDim.x) {
    const int i = k / G, v = k - i * G, c = ((i / V) * G + v) * V + i % V;
    if (c >= a.cols) continue;
    float p = 0.0f, q = 0.0f;
    for (int j = 0; j < ngrp; ++j) {
      p += sums[(2 * j) * per + k];
      q += sums[(2 * j + 1) * per + k];
    }
    dst[c] = p;
    dst[a.cols + c] = q;
  }
}

// Rows wider than a CTA's registers (over 8192 entries, in the forward of aligned rows
// 16384), one CTA a row: X is read three times in the forward (the second and third time
// from L1 or L2; 2000 x 20000 in fp32 71 us, 4.5 TB/s) ...
template <typename T, int V>
__global__ void __launch_bounds__(kNormThreads)
    k_norm_fwd_wide(const NormArgs a) {
  __shared__ float slots[2][32];
  let_next_start();
  wait_for_previous();
  const int t = threadIdx.x, lane = t & 31, gw = t >> 5;
  const int nvec = a.cols / V;
  const float n = (float)a.cols;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T *px = static_cast<const T *>(a.x) + r * a.ldx;
    T *py = static_cast<T *>(a.y) + r * a.ldy;
    Pack<T, V> x;
    float s = 0.0f;
#pragma unroll 4
    for (int v = t; v < nvec; v += kNormThreads) {
      x.load(px + (int64_t)v * V);
#pragma unroll
      for (int i = 0; i < V; ++i) s += x.f(i);
    }
    const float mean = group_sum(s, slots[0], kNormThreads, 0, gw, lane) / n;
    s = 0.0f;
#pragma unroll 4
    for (int v = t; v < nvec; v += kNormThreads) {
      x.load(px + (int64_t)v * V);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float d = x.f(i) - mean;
        s = fmaf(d, d, s);
      }
    }
    const float var = group_sum(s, slots[1], kNormThreads, 0, gw, lane) / n;
    const float rstd = 1.0f / sqrtf(var + a.eps);
    if (t == 0) {
      if (a.mean) a.mean[r] = mean;
      if (a.rstd) a.rstd[r] = rstd;
    }
#pragma unroll 2
    for (int v = t; v < nvec; v += kNormThreads) {
      x.load(px + (int64_t)v * V);
      float ga[V], be[V], y[V];
      load_columns<V, 1>(a.gamma, a.cols, 0, v, 1.0f, ga);
      load_columns<V, 1>(a.beta, a.cols, 0, v, 0.0f, be);
#pragma unroll
      for (int i = 0; i < V; ++i) y[i] = fmaf((x.f(i) - mean) * rstd, ga[i], be[i]);
      store_pack<T, V>(py + (int64_t)v * V, y);
    }
  }
}

// ... and, in the backward, X and dY twice for dX by rows, and once for the column sums
// by columns.
template <typename T, int V>
__global__ void __launch_bounds__(kNormThreads)
    k_norm_bwd_wide(const NormArgs a) {
  __shared__ float slots[2][32];
  let_next_start();
  wait_for_previous();
  const int t = threadIdx.x, lane = t & 31, gw = t >> 5;
  const int nvec = a.cols / V;
  const float n = (float)a.cols;
  int slot = 0;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x, slot ^= 1) {
    const T *px = static_cast<const T *>(a.x) + r * a.ldx;
    const T *pdy = static_cast<const T *>(a.dy) + r * a.lddy;
    T *pdx = static_cast<T *>(a.y) + r * a.ldy;
    const float mean = a.mean[r], rstd = a.rstd[r];
    Pack<T, V> x, dy;
    float ga[V], s1 = 0.0f, s2 = 0.0f;
#pragma unroll 2
    for (int v = t; v < nvec; v += kNormThreads) {
      x.load(px + (int64_t)v * V);
      dy.load(pdy + (int64_t)v * V);
      load_columns<V, 1>(a.gamma, a.cols, 0, v, 1.0f, ga);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float g = dy.f(i) * ga[i];
        s1 += g;
        s2 = fmaf(g, x.f(i) - mean, s2);
      }
    }
    const float2 s = group_sum2(s1, s2, slots[slot], kNormThreads, 0, gw, lane);
    const float k0 = -rstd * (s.x / n), k1 = -rstd * (rstd * (rstd * (s.y / n)));
#pragma unroll 2
    for (int v = t; v < nvec; v += kNormThreads) {
      x.load(px + (int64_t)v * V);
      dy.load(pdy + (int64_t)v * V);
      load_columns<V, 1>(a.gamma, a.cols, 0, v, 1.0f, ga);
      float o[V];
#pragma unroll
      for (int i = 0; i < V; ++i)
        o[i] = fmaf(x.f(i) - mean, k1, fmaf(dy.f(i) * ga[i], rstd, k0));
      store_pack<T, V>(pdx + (int64_t)v * V, o);
    }
  }
}

constexpr int kNormColRows = 32;  // partial rows of the wide columns' sums

template <typename T, int V>
__global__ void __launch_bounds__(128) k_norm_cols_wide(const NormArgs a, int64_t rows_per) {
  let_next_start();
  wait_for_previous();
  const int v = blockIdx.x * blockDim.x + threadIdx.x;
  if (v >= a.cols / V) return;
  const int64_t r0 = (int64_t)blockIdx.y * rows_per, r1 = min(a.rows, r0 + rows_per);
  const T *px = static_cast<const T *>(a.x) + (int64_t)v * V;
  const T *pdy = static_cast<const T *>(a.dy) + (int64_t)v * V;
  float dg[V] = {}, db[V] = {};
#pragma unroll 4
  for (int64_t r = r0; r < r1; ++r) {
    Pack<T, V> x, dy;
    x.load(px + r * a.ldx);
    dy.load(pdy + r * a.lddy);
    const float mean = __ldg(a.mean + r), rstd = __ldg(a.rstd + r);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      dg[i] = fmaf(dy.f(i) * rstd, x.f(i) - mean, dg[i]);
      db[i] += dy.f(i);
    }
  }
  float *dst = a.part + (int64_t)blockIdx.y * 2 * a.cols + (int64_t)v * V;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    dst[i] = dg[i];
    dst[a.cols + i] = db[i];
  }
}

// dgamma and dbeta: the sums of n partial rows, 8 columns a CTA, 64 rows side by side:
// a few loads a thread on many CTAs (with 32 columns a CTA and 8 rows it took 12 us).
constexpr int kNormColThreads = 512;

__global__ void __launch_bounds__(kNormColThreads)
    k_norm_cols(const float *part, int n, int cols, float *dgamma, float *dbeta) {
  __shared__ float sums[2][kNormColThreads / 32][8];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int64_t c = (int64_t)blockIdx.x * 8 + (lane & 7);
  let_next_start();
  wait_for_previous();
  float u = 0.0f, v = 0.0f;
  if (c < cols) {
#pragma unroll 4
    for (int i = threadIdx.x >> 3; i < n; i += kNormColThreads / 8) {
      u += __ldcg(part + (int64_t)i * 2 * cols + c);
      v += __ldcg(part + (int64_t)i * 2 * cols + cols + c);
    }
  }
#pragma unroll
  for (int o = 16; o > 4; o >>= 1) {
    u += __shfl_xor_sync(0xffffffffu, u, o);
    v += __shfl_xor_sync(0xffffffffu, v, o);
  }
  if (lane < 8) {
    sums[0][w][lane] = u;
    sums[1][w][lane] = v;
  }
  __syncthreads();
  if (threadIdx.x < 16 && c < cols) {
    const int which = threadIdx.x >> 3;
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < kNormColThreads / 32; ++i) s += sums[which][i][lane & 7];
    float *out = which ? dbeta : dgamma;
    if (out) out[c] = s;
  }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
// Threads per row, groups per CTA and CTAs of the kernels that hold a row.
struct NormPlan {
  bool wide;   // rows wider than a CTA's registers
  bool ahead;  // rows fetched ahead through shared memory
  bool thin;   // 16 bytes a thread: few rows, where their latency counts
  int v, G, groups, grid;
  int entries;  // of a row, a thread: 16, or 32 of them and half as many threads
};

static NormPlan norm_plan(int64_t rows, int64_t cols, bool bf16, bool vec, bool bwd, int nsm) {
  NormPlan p = {};
  p.v = vec ? (bf16 ? 8 : 4) : 1;
  const int64_t nvec = cols / p.v;
  // a row a CTA: 16 bytes a thread (one row of 1024: 1.8 us, with 16 entries a thread 2.3)
  p.thin = vec && rows <= nsm && nvec <= kNormThreads;
  // Forward: 32 entries a thread need half the shuffles and smaller barriers (8192 x 1024
  // in bf16 8.3 us, with 16 entries 8.9, and 6.6 and 8.3 on rows in L2; 32768 x 4096 90 and
  // 98, in fp32 167 and 184), if
  // they do not leave a third of the threads idle (21276 x 1088 24.3 us and 22.8), and in
  // fp32 if a CTA holds more than two rows at a time or 16 entries would not hold the row
  // (10000 x 8192 110 us and 98; 20000 x 5120 132 and 144; 5000 x 12288 90, read three
  // times 112).  Single entries and the backward have not the registers for it.
  p.entries = 16;
  if (!bwd && vec && !p.thin) {
    const int64_t pad = (cols + 1023) / 1024 * 1024, groups = kNormThreads * 32 / pad;
    if ((pad <= (cols + 511) / 512 * 512 || cols * 3 >= pad * 2) && (bf16 || groups != 2))
      p.entries = 32;
  }
  const int vpt = p.thin ? 1 : p.entries / p.v;
  p.wide = nvec > (int64_t)vpt * kNormThreads;
  if (p.wide) {
    p.G = kNormThreads;
    p.groups = 1;
    p.grid = (int)(rows < 4 * nsm ? rows : 4 * nsm);
    return p;
  }
  const int64_t need = (nvec + vpt - 1) / vpt;
  p.G = (int)((need + 31) / 32 * 32);
  p.groups = kNormThreads / p.G;
  if (p.G > 32 && p.groups > 8) p.groups = 8;  // their named barriers
  const int64_t slots = (int64_t)nsm * p.groups;
  // rows fetched ahead where there is a next one; few rows go to SMs of their own
  p.ahead = vec && rows > slots;
  if (!p.ahead) {
    const int64_t each = (rows + nsm - 1) / nsm;
    if (each < p.groups) p.groups = (int)each;
  }
  // (the forward of 16 entries takes two rows at a time where it fetches ahead)
  const int64_t each = p.groups * (p.ahead && !bwd && p.entries == 16 ? 2 : 1);
  const int64_t want = (rows + each - 1) / each;
  p.grid = (int)(want < nsm ? want : nsm);
  return p;
}

// The most partial rows of column sums that any plan writes: a CTA each.
static int norm_parts(int nsm) { return nsm > kNormColRows ? nsm : kNormColRows; }

size_t layer_norm_ws_bytes(int64_t rows, int64_t cols) {
  (void)rows;
  if (cols <= 0) return kHeaderBytes;
  return kHeaderBytes + (size_t)norm_parts(device_sm_count()) * 2 * (size_t)cols * sizeof(float);
}

template <typename T, bool BWD, int V, int VPT, int S>
static cudaError_t launch_rows(const NormArgs &a, const NormPlan &p, cudaStream_t st) {
  const int nth = p.G * p.groups;
  constexpr int R = !BWD && S > 0 && V * VPT == 16 ? 2 : 1;
  size_t smem = (size_t)S * VPT * (BWD ? 2 : R) * 16 * nth;  // the rows on their way
  const size_t sums = BWD && p.groups > 1 && a.part ? 2 * sizeof(float) * VPT * V * nth : 0;
  smem = std::max(smem, sums);
  void (*kernel)(NormArgs, int);
  if constexpr (BWD) kernel = k_norm_bwd<T, V, VPT, S>;
  else kernel = k_norm_fwd<T, V, VPT, R, S>;
  if (smem > 40 * 1024) {  // with the static arrays past 48 KB
    static DeviceOnce once;
    const cudaError_t e = allow_smem(kernel, 200 * 1024, once);
    if (e != cudaSuccess) return e;
  }
  return launch_behind(kernel, dim3((unsigned)p.grid), nth, smem, st, a, p.G);
}

template <typename T, bool BWD, int V, int E>
static cudaError_t launch_held(const NormArgs &a, const NormPlan &p, cudaStream_t st) {
  constexpr int VPT = E / V;
  // stages: 128 KB of rows in bf16 (four) and 192 KB in fp32 (three)
  if constexpr (V == 1) return launch_rows<T, BWD, 1, VPT, 0>(a, p, st);
  else if (p.ahead) return launch_rows<T, BWD, V, VPT, V == 8 ? 4 : 3>(a, p, st);
  else return launch_rows<T, BWD, V, VPT, 0>(a, p, st);
}

template <typename T, bool BWD, int V>
static cudaError_t launch_held(const NormArgs &a, const NormPlan &p, cudaStream_t st) {
  if constexpr (V > 1)
    if (p.thin) return launch_rows<T, BWD, V, 1, 0>(a, p, st);
  if constexpr (!BWD && V > 1)
    if (p.entries == 32) return launch_held<T, BWD, V, 32>(a, p, st);
  return launch_held<T, BWD, V, 16>(a, p, st);
}

template <bool BWD>
static cudaError_t launch_norm(const NormArgs &a, const NormPlan &p, bool bf16, cudaStream_t st) {
  if (bf16)
    return p.v > 1 ? launch_held<__nv_bfloat16, BWD, 8>(a, p, st)
                   : launch_held<__nv_bfloat16, BWD, 1>(a, p, st);
  return p.v > 1 ? launch_held<float, BWD, 4>(a, p, st) : launch_held<float, BWD, 1>(a, p, st);
}

template <typename T, int V>
static cudaError_t launch_wide_rows(const NormArgs &a, const NormPlan &p, bool bwd,
                                    int64_t rows_per, int nparts, cudaStream_t st) {
  const dim3 rows((unsigned)p.grid);
  cudaError_t e = cudaSuccess;
  if (!bwd) e = launch_behind(k_norm_fwd_wide<T, V>, rows, kNormThreads, 0, st, a);
  if (bwd && a.y) e = launch_behind(k_norm_bwd_wide<T, V>, rows, kNormThreads, 0, st, a);
  if (e == cudaSuccess && nparts > 0)
    e = launch_behind(k_norm_cols_wide<T, V>,
                      dim3((unsigned)((a.cols / V + 127) / 128), (unsigned)nparts), 128, 0, st, a,
                      rows_per);
  return e;
}

static cudaError_t launch_wide(const NormArgs &a, const NormPlan &p, bool bf16, bool bwd,
                               int64_t rows_per, int nparts, cudaStream_t st) {
  if (bf16)
    return p.v > 1 ? launch_wide_rows<__nv_bfloat16, 8>(a, p, bwd, rows_per, nparts, st)
                   : launch_wide_rows<__nv_bfloat16, 1>(a, p, bwd, rows_per, nparts, st);
  return p.v > 1 ? launch_wide_rows<float, 4>(a, p, bwd, rows_per, nparts, st)
                 : launch_wide_rows<float, 1>(a, p, bwd, rows_per, nparts, st);
}

static bool ptr_aligned(const void *p, size_t n) {
  return reinterpret_cast<uintptr_t>(p) % n == 0;
}

static bool rows_aligned(const void *p, int64_t ld, int64_t esize) {
  return !p || (reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld * esize % 16 == 0);
}

fqt_status layer_norm(const NormArgs &in, bool bf16, bool bwd, cudaStream_t st) {
  NormArgs a = in;
  const int64_t es = bf16 ? 2 : 4;
  const int nsm = device_sm_count();
  const bool vec = a.cols % (bf16 ? 8 : 4) == 0 && ptr_aligned(a.gamma, 16) &&
                   ptr_aligned(a.beta, 16) && rows_aligned(a.x, a.ldx, es) &&
                   rows_aligned(a.dy, a.lddy, es) && rows_aligned(a.y, a.ldy, es);
  NormPlan p = norm_plan(a.rows, a.cols, bf16, vec, bwd, nsm);
  int nparts = p.grid;
  cudaError_t e;
  if (p.wide) {
    int64_t per = 0;
    nparts = 0;
    if (bwd && a.part) {
      nparts = (int)(a.rows < kNormColRows ? a.rows : kNormColRows);
      per = (a.rows + nparts - 1) / nparts;
      nparts = (int)((a.rows + per - 1) / per);
    }
    e = launch_wide(a, p, bf16, bwd, per, nparts, st);
  } else {
    e = bwd ? launch_norm<true>(a, p, bf16, st) : launch_norm<false>(a, p, bf16, st);
  }
  if (e != cudaSuccess) return cuda_fail(e, "layer norm launch");
  if (bwd && a.part) {
    e = launch_behind(k_norm_cols, dim3((unsigned)((a.cols + 7) / 8)), kNormColThreads, 0, st,
                      (const float *)a.part, nparts, a.cols, a.dgamma, a.dbeta);
    return cuda_fail(e, "layer norm column sums launch");
  }
  return FQT_OK;
}

// rows x cols entries at a row pitch of ld: sizes that stay inside 64 bits
static bool good_rows(int64_t rows, int64_t cols, int64_t ld) {
  return rows <= 1 || (ld >= cols && ld <= INT64_MAX / 8 / rows);
}

}  // namespace fqt

using namespace fqt;

extern "C" {

size_t fqt_layer_norm_workspace_size(int64_t rows, int64_t cols) {
  return layer_norm_ws_bytes(rows, cols);
}

fqt_status fqt_layer_norm_forward(const void *X, int64_t ldx, fqt_dtype dtype, int64_t rows,
                                  int64_t cols, const float *gamma, const float *beta, float eps,
                                  void *Y, int64_t ldy, float *mean, float *rstd,
                                  void *stream) {
  if (rows < 0 || cols <= 0 || cols > (1 << 30) || !(eps >= 0.0f) || isinf(eps))
    return FQT_EINVAL;
  if (dtype != FQT_F32 && dtype != FQT_BF16) return FQT_EINVAL;
  if (!good_rows(rows, cols, ldx) || !good_rows(rows, cols, ldy)) return FQT_EINVAL;
  if (rows == 0) return FQT_OK;
  const size_t es = dtype == FQT_BF16 ? 2 : 4;
  if (!X || !Y || !ptr_aligned(X, es) || !ptr_aligned(Y, es) || !ptr_aligned(gamma, 4) ||
      !ptr_aligned(beta, 4) || !ptr_aligned(mean, 4) || !ptr_aligned(rstd, 4))
    return FQT_EINVAL;
  NormArgs a = {};
  a.x = X;
  a.y = Y;
  a.ldx = rows > 1 ? ldx : 0;
  a.ldy = rows > 1 ? ldy : 0;
  a.rows = rows;
  a.cols = (int)cols;
  a.gamma = gamma;
  a.beta = beta;
  a.eps = eps;
  a.mean = mean;
  a.rstd = rstd;
  return layer_norm(a, dtype == FQT_BF16, false, reinterpret_cast<cudaStream_t>(stream));
}

fqt_status fqt_layer_norm_backward(const void *dY, int64_t lddy, const void *X, int64_t ldx,
                                   fqt_dtype dtype, int64_t rows, int64_t cols,
                                   const float *mean, const float *rstd, const float *gamma,
                                   void *dX, int64_t lddx, float *dgamma, float *dbeta,
                                   void *workspace, size_t ws_bytes, void *stream) {
  if (rows < 0 || cols <= 0 || cols > (1 << 30)) return FQT_EINVAL;
  if (dtype != FQT_F32 && dtype != FQT_BF16) return FQT_EINVAL;
  if (!good_rows(rows, cols, ldx) || !good_rows(rows, cols, lddy) ||
      (dX && !good_rows(rows, cols, lddx)))
    return FQT_EINVAL;
  if (!ptr_aligned(dgamma, 4) || !ptr_aligned(dbeta, 4)) return FQT_EINVAL;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  if (rows == 0) {  // sums over no rows
    for (float *o : {dgamma, dbeta})
      if (o) {
        const cudaError_t e = cudaMemsetAsync(o, 0, (size_t)cols * sizeof(float), st);
        if (e != cudaSuccess) return cuda_fail(e, "layer norm clear");
      }
    return FQT_OK;
  }
  const size_t es = dtype == FQT_BF16 ? 2 : 4;
  if (!X || !dY || !mean || !rstd || !ptr_aligned(X, es) || !ptr_aligned(dY, es) ||
      !ptr_aligned(dX, es) || !ptr_aligned(mean, 4) || !ptr_aligned(rstd, 4) ||
      !ptr_aligned(gamma, 4))
    return FQT_EINVAL;
  if (!dX && !dgamma && !dbeta) return FQT_EINVAL;
  const bool sums = dgamma || dbeta;
  if (sums && (!workspace || !ptr_aligned(workspace, 256) ||
               ws_bytes < layer_norm_ws_bytes(rows, cols)))
    return FQT_EWORKSPACE;
  NormArgs a = {};
  a.x = X;
  a.dy = dY;
  a.y = dX;
  a.ldx = rows > 1 ? ldx : 0;
  a.lddy = rows > 1 ? lddy : 0;
  a.ldy = rows > 1 ? lddx : 0;
  a.rows = rows;
  a.cols = (int)cols;
  a.gamma = gamma;
  a.mean = const_cast<float *>(mean);
  a.rstd = const_cast<float *>(rstd);
  a.part = sums ? reinterpret_cast<float *>(static_cast<char *>(workspace) + kHeaderBytes)
                : nullptr;
  a.dgamma = dgamma;
  a.dbeta = dbeta;
  return layer_norm(a, dtype == FQT_BF16, true, st);
}

}  // extern "C"
