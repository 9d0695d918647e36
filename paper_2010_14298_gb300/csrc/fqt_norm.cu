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
// against 4 and 6 bytes of bf16), so a row is read once and kept in registers, as
// it was read, by a group of threads wide enough to hold it: the group reduces the
// row's sums, and every thread then finishes the entries it holds.  A group keeps
// its columns from row to row, so gamma, beta and the partial sums of the column
// reductions stay in registers too.  The variance is taken about the mean (a second
// reduction over registers), not from the sum of squares, which loses it where the
// mean is large.  All statistics and sums are fp32.
#include <cuda_runtime.h>
#include <math.h>

#include "fqt.h"
#include "fqt_common.cuh"
#include "fqt_internal.h"

namespace fqt {

constexpr int kNormCtaThreads = 512;  // groups share a CTA up to this many threads
constexpr int kNormMaxGroups = 8;     // named barriers 1 .. 8
constexpr int kNormMaxThreads = 1024;

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
__device__ __forceinline__ void store_pack(T *p, const float (&v)[V]) {
  if constexpr (sizeof(T) == 4) {
    if constexpr (V == 4) *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
    else *p = v[0];
  } else if constexpr (V == 8) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t *>(&b);
    }
    *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  } else {
    *p = __float2bfloat16_rn(v[0]);
  }
}

// Sums of NV values over the threads of a group (G threads from a warp boundary,
// G a multiple of 32), in every thread, in an order that does not change.  slot:
// the group's NV x 32 floats of shared memory; a call must not follow another on the
// same slot without a barrier of the group between the reads and the writes, so
// callers alternate slots.
template <int NV>
__device__ __forceinline__ void group_sum(float (&v)[NV], float *slot, int G, int gid, int gw,
                                          int lane) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
#pragma unroll
    for (int k = 0; k < NV; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
  if (G == 32) return;
  if (lane == 0)
#pragma unroll
    for (int k = 0; k < NV; ++k) slot[k * 32 + gw] = v[k];
  asm volatile("bar.sync %0, %1;" ::"r"(1 + gid), "r"(G) : "memory");
  const int nw = G >> 5;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    float s = 0.0f;
    for (int i = 0; i < nw; ++i) s += slot[k * 32 + i];
    v[k] = s;
  }
}

// Forward.  A group takes R rows at a time (two where there are rows enough: twice
// the loads in flight, and half the barriers per row).
template <typename T, int V, int VPT, int R>
__global__ void __launch_bounds__(kNormMaxThreads)
    k_norm_fwd(const NormArgs a, int G) {
  __shared__ float slots[kNormMaxGroups][2][R * 32];
  const int gid = threadIdx.x / G, t = threadIdx.x - gid * G;
  const int lane = t & 31, gw = t >> 5, ngrp = blockDim.x / G;
  const int nvec = a.cols / V;
  const float n = (float)a.cols;
  float ga[VPT * V], be[VPT * V];
#pragma unroll
  for (int j = 0; j < VPT; ++j)
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int c = (j * G + t) * V + i;
      ga[j * V + i] = a.gamma && c < a.cols ? __ldg(a.gamma + c) : 1.0f;
      be[j * V + i] = a.beta && c < a.cols ? __ldg(a.beta + c) : 0.0f;
    }
  const int64_t step = (int64_t)gridDim.x * ngrp * R;
  for (int64_t r0 = ((int64_t)blockIdx.x * ngrp + gid) * R; r0 < a.rows; r0 += step) {
    Pack<T, V> x[R][VPT];
    float s[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      s[r] = 0.0f;
#pragma unroll
      for (int j = 0; j < VPT; ++j) {
        const int v = j * G + t;
        if (r0 + r < a.rows && v < nvec)
          x[r][j].load(static_cast<const T *>(a.x) + (r0 + r) * a.ldx + (int64_t)v * V);
        else
          x[r][j].zero();
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int j = 0; j < VPT; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) s[r] += x[r][j].f(i);
    group_sum<R>(s, slots[gid][0], G, gid, gw, lane);
    float mean[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      mean[r] = s[r] / n;
      s[r] = 0.0f;
#pragma unroll
      for (int j = 0; j < VPT; ++j)
        if (j * G + t < nvec)
#pragma unroll
          for (int i = 0; i < V; ++i) {
            const float d = x[r][j].f(i) - mean[r];
            s[r] = fmaf(d, d, s[r]);
          }
    }
    group_sum<R>(s, slots[gid][1], G, gid, gw, lane);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (r0 + r >= a.rows) break;
      const float rstd = 1.0f / sqrtf(s[r] / n + a.eps);
      if (t == 0) {
        if (a.mean) a.mean[r0 + r] = mean[r];
        if (a.rstd) a.rstd[r0 + r] = rstd;
      }
#pragma unroll
      for (int j = 0; j < VPT; ++j) {
        const int v = j * G + t;
        if (v >= nvec) continue;
        float y[V];
#pragma unroll
        for (int i = 0; i < V; ++i)
          y[i] = fmaf((x[r][j].f(i) - mean[r]) * rstd, ga[j * V + i], be[j * V + i]);
        store_pack<T, V>(static_cast<T *>(a.y) + (r0 + r) * a.ldy + (int64_t)v * V, y);
      }
    }
  }
}

// Backward.  The column sums of a group's rows stay in its registers; at the end
// the groups of a CTA are added in shared memory, and each CTA writes one row of
// partial sums (k_norm_cols adds those).
template <typename T, int V, int VPT, int R>
__global__ void __launch_bounds__(kNormMaxThreads)
    k_norm_bwd(const NormArgs a, int G) {
  extern __shared__ float colsum[];  // 2 x cols, where the CTA has several groups
  __shared__ float slots[kNormMaxGroups][2][2 * R * 32];
  const int gid = threadIdx.x / G, t = threadIdx.x - gid * G;
  const int lane = t & 31, gw = t >> 5, ngrp = blockDim.x / G;
  const int nvec = a.cols / V;
  const float n = (float)a.cols;
  float ga[VPT * V], dg[VPT * V], db[VPT * V];
#pragma unroll
  for (int j = 0; j < VPT; ++j)
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int c = (j * G + t) * V + i;
      ga[j * V + i] = a.gamma && c < a.cols ? __ldg(a.gamma + c) : 1.0f;
      dg[j * V + i] = db[j * V + i] = 0.0f;
    }
  const int64_t step = (int64_t)gridDim.x * ngrp * R;
  int slot = 0;
  for (int64_t r0 = ((int64_t)blockIdx.x * ngrp + gid) * R; r0 < a.rows; r0 += step, slot ^= 1) {
    Pack<T, V> x[R][VPT], dy[R][VPT];
    float mean[R], rstd[R], s[2 * R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const bool in = r0 + r < a.rows;
      mean[r] = in ? __ldg(a.mean + r0 + r) : 0.0f;
      rstd[r] = in ? __ldg(a.rstd + r0 + r) : 0.0f;
#pragma unroll
      for (int j = 0; j < VPT; ++j) {
        const int v = j * G + t;
        if (in && v < nvec) {
          x[r][j].load(static_cast<const T *>(a.x) + (r0 + r) * a.ldx + (int64_t)v * V);
          dy[r][j].load(static_cast<const T *>(a.dy) + (r0 + r) * a.lddy + (int64_t)v * V);
        } else {
          x[r][j].zero();
          dy[r][j].zero();
        }
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      s[2 * r] = s[2 * r + 1] = 0.0f;
#pragma unroll
      for (int j = 0; j < VPT; ++j) {
        if (r0 + r >= a.rows || j * G + t >= nvec) continue;
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float xh = (x[r][j].f(i) - mean[r]) * rstd[r], d = dy[r][j].f(i);
          const float g = d * ga[j * V + i];
          s[2 * r] += g;
          s[2 * r + 1] = fmaf(g, xh, s[2 * r + 1]);
          dg[j * V + i] = fmaf(d, xh, dg[j * V + i]);
          db[j * V + i] += d;
        }
      }
    }
    if (!a.y) continue;
    group_sum<2 * R>(s, slots[gid][slot], G, gid, gw, lane);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (r0 + r >= a.rows) break;
      const float m1 = s[2 * r] / n, m2 = s[2 * r + 1] / n;
#pragma unroll
      for (int j = 0; j < VPT; ++j) {
        const int v = j * G + t;
        if (v >= nvec) continue;
        float o[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float xh = (x[r][j].f(i) - mean[r]) * rstd[r];
          const float g = dy[r][j].f(i) * ga[j * V + i];
          o[i] = rstd[r] * (g - m1 - xh * m2);
        }
        store_pack<T, V>(static_cast<T *>(a.y) + (r0 + r) * a.ldy + (int64_t)v * V, o);
      }
    }
  }
  if (!a.part) return;
  float *dst = a.part + (int64_t)blockIdx.x * 2 * a.cols;
  for (int q = ngrp - 1; q >= 0; --q) {  // groups add up from the last to the first
    if (gid == q)
#pragma unroll
      for (int j = 0; j < VPT; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const int c = (j * G + t) * V + i;
          if (c >= a.cols) continue;
          float u = dg[j * V + i], w = db[j * V + i];
          if (q < ngrp - 1) {
            u += colsum[c];
            w += colsum[a.cols + c];
          }
          if (q > 0) {
            colsum[c] = u;
            colsum[a.cols + c] = w;
          } else {
            dst[c] = u;
            dst[a.cols + c] = w;
          }
        }
    if (q > 0) __syncthreads();
  }
}

// Rows wider than a CTA's registers: three reads of X in the forward ...
template <typename T>
__global__ void __launch_bounds__(kNormMaxThreads)
    k_norm_fwd_wide(const NormArgs a) {
  __shared__ float slots[2][32];
  const int t = threadIdx.x, lane = t & 31, gw = t >> 5;
  const float n = (float)a.cols;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T *x = static_cast<const T *>(a.x) + r * a.ldx;
    T *y = static_cast<T *>(a.y) + r * a.ldy;
    float s[1] = {0.0f};
    for (int c = t; c < a.cols; c += blockDim.x) s[0] += (float)x[c];
    group_sum<1>(s, slots[0], blockDim.x, 0, gw, lane);
    const float mean = s[0] / n;
    s[0] = 0.0f;
    for (int c = t; c < a.cols; c += blockDim.x) {
      const float d = (float)x[c] - mean;
      s[0] = fmaf(d, d, s[0]);
    }
    group_sum<1>(s, slots[1], blockDim.x, 0, gw, lane);
    const float rstd = 1.0f / sqrtf(s[0] / n + a.eps);
    if (t == 0) {
      if (a.mean) a.mean[r] = mean;
      if (a.rstd) a.rstd[r] = rstd;
    }
    for (int c = t; c < a.cols; c += blockDim.x) {
      const float g = a.gamma ? __ldg(a.gamma + c) : 1.0f, b = a.beta ? __ldg(a.beta + c) : 0.0f;
      y[c] = (T)fmaf(((float)x[c] - mean) * rstd, g, b);
    }
  }
}

// ... and, in the backward, dX by rows and the column sums by columns.
template <typename T>
__global__ void __launch_bounds__(kNormMaxThreads)
    k_norm_bwd_wide(const NormArgs a) {
  __shared__ float slots[2][64];
  const int t = threadIdx.x, lane = t & 31, gw = t >> 5;
  const float n = (float)a.cols;
  int slot = 0;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x, slot ^= 1) {
    const T *x = static_cast<const T *>(a.x) + r * a.ldx;
    const T *dy = static_cast<const T *>(a.dy) + r * a.lddy;
    T *dx = static_cast<T *>(a.y) + r * a.ldy;
    const float mean = a.mean[r], rstd = a.rstd[r];
    float s[2] = {0.0f, 0.0f};
    for (int c = t; c < a.cols; c += blockDim.x) {
      const float g = (float)dy[c] * (a.gamma ? __ldg(a.gamma + c) : 1.0f);
      s[0] += g;
      s[1] = fmaf(g, ((float)x[c] - mean) * rstd, s[1]);
    }
    group_sum<2>(s, slots[slot], blockDim.x, 0, gw, lane);
    const float m1 = s[0] / n, m2 = s[1] / n;
    for (int c = t; c < a.cols; c += blockDim.x) {
      const float g = (float)dy[c] * (a.gamma ? __ldg(a.gamma + c) : 1.0f);
      const float xh = ((float)x[c] - mean) * rstd;
      dx[c] = (T)(rstd * (g - m1 - xh * m2));
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(256) k_norm_cols_wide(const NormArgs a, int64_t rows_per) {
  const int c = blockIdx.x * blockDim.x + threadIdx.x;
  if (c >= a.cols) return;
  const int64_t r0 = (int64_t)blockIdx.y * rows_per, r1 = min(a.rows, r0 + rows_per);
  float dg = 0.0f, db = 0.0f;
  for (int64_t r = r0; r < r1; ++r) {
    const float d = (float)static_cast<const T *>(a.dy)[r * a.lddy + c];
    const float x = (float)static_cast<const T *>(a.x)[r * a.ldx + c];
    dg = fmaf(d, (x - a.mean[r]) * a.rstd[r], dg);
    db += d;
  }
  float *dst = a.part + (int64_t)blockIdx.y * 2 * a.cols;
  dst[c] = dg;
  dst[a.cols + c] = db;
}

// dgamma and dbeta: the sums of n partial rows, 32 columns a CTA, warp w taking
// rows w, w + 8, ...
__global__ void __launch_bounds__(256)
    k_norm_cols(const float *part, int n, int cols, float *dgamma, float *dbeta) {
  __shared__ float sums[2][8][33];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  float u = 0.0f, v = 0.0f;
  if (c < cols)
    for (int i = w; i < n; i += 8) {
      u += part[(int64_t)i * 2 * cols + c];
      v += part[(int64_t)i * 2 * cols + cols + c];
    }
  sums[0][w][lane] = u;
  sums[1][w][lane] = v;
  __syncthreads();
  if (w < 2 && c < cols) {
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s += sums[w][i][lane];
    float *out = w ? dbeta : dgamma;
    if (out) out[c] = s;
  }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
// Threads per row, groups per CTA and CTAs of the kernels that hold a row.
struct NormPlan {
  bool wide;  // rows wider than a CTA's registers
  int v, vpt, G, groups, grid;
  bool two;   // two rows at a time
};

static NormPlan norm_plan(int64_t rows, int64_t cols, bool bf16, bool vec, int nsm) {
  NormPlan p = {};
  const int vmax = bf16 ? 8 : 4;
  p.v = vec ? vmax : 1;
  const int64_t nvec = cols / p.v;
  // entries per thread: 16 bytes, or 4 single entries; twice that where a CTA's
  // threads do not cover the row
  p.vpt = vec ? 1 : 4;
  if (nvec > (int64_t)p.vpt * kNormMaxThreads) p.vpt *= 2;
  p.wide = nvec > (int64_t)p.vpt * kNormMaxThreads;
  if (p.wide) {
    p.G = kNormMaxThreads;
    p.groups = 1;
    p.grid = (int)(rows < 2 * nsm ? rows : 2 * nsm);
    return p;
  }
  const int64_t need = (nvec + p.vpt - 1) / p.vpt;
  p.G = (int)((need + 31) / 32 * 32);
  p.groups = kNormCtaThreads / p.G;
  if (p.groups < 1) p.groups = 1;
  if (p.groups > kNormMaxGroups) p.groups = kNormMaxGroups;
  // 64 registers a thread: 1024 threads an SM
  const int per_sm = kNormMaxThreads / (p.G * p.groups);
  const int64_t slots = (int64_t)nsm * per_sm * p.groups;
  p.two = rows >= 2 * slots && p.vpt == (vec ? 1 : 4);
  // few rows: one group a CTA, so that they spread over the SMs
  if (rows <= nsm) p.groups = 1;
  const int64_t each = (int64_t)p.groups * (p.two ? 2 : 1);
  const int64_t want = (rows + each - 1) / each;
  p.grid = (int)(want < nsm * per_sm ? want : nsm * per_sm);
  return p;
}

// The most partial rows of column sums that any plan writes (CTAs of 8 groups of
// a warp: four an SM).
static int norm_parts(int nsm) { return kNormMaxThreads / (32 * kNormMaxGroups) * nsm; }

size_t layer_norm_ws_bytes(int64_t rows, int64_t cols) {
  (void)rows;
  if (cols <= 0) return kHeaderBytes;
  return kHeaderBytes + (size_t)norm_parts(device_sm_count()) * 2 * (size_t)cols * sizeof(float);
}

template <typename T, int V, int VPT, int R>
static void launch_rows(const NormArgs &a, const NormPlan &p, bool bwd, cudaStream_t st) {
  const int nth = p.G * p.groups;
  // several groups only where G <= 256: at most 2 x 2048 columns, 16 KB
  const size_t smem = p.groups > 1 && a.part ? 2 * sizeof(float) * a.cols : 0;
  if (bwd) k_norm_bwd<T, V, VPT, R><<<p.grid, nth, smem, st>>>(a, p.G);
  else k_norm_fwd<T, V, VPT, R><<<p.grid, nth, 0, st>>>(a, p.G);
}

template <typename T, int V>
static void launch_held(const NormArgs &a, const NormPlan &p, bool bwd, cudaStream_t st) {
  constexpr int v1 = V == 1 ? 4 : 1;
  if (p.vpt > v1) launch_rows<T, V, 2 * v1, 1>(a, p, bwd, st);
  else if (p.two) launch_rows<T, V, v1, 2>(a, p, bwd, st);
  else launch_rows<T, V, v1, 1>(a, p, bwd, st);
}

static bool rows_aligned(const void *p, int64_t ld, int64_t esize) {
  return !p || (reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld * esize % 16 == 0);
}

fqt_status layer_norm(const NormArgs &in, bool bf16, bool bwd, cudaStream_t st) {
  NormArgs a = in;
  const int64_t es = bf16 ? 2 : 4;
  const int nsm = device_sm_count();
  const bool vec = a.cols % (bf16 ? 8 : 4) == 0 && rows_aligned(a.x, a.ldx, es) &&
                   rows_aligned(a.dy, a.lddy, es) && rows_aligned(a.y, a.ldy, es);
  NormPlan p = norm_plan(a.rows, a.cols, bf16, vec, nsm);
  int nparts = p.grid;
  if (p.wide) {
    if (!bwd) {
      if (bf16) k_norm_fwd_wide<__nv_bfloat16><<<p.grid, p.G, 0, st>>>(a);
      else k_norm_fwd_wide<float><<<p.grid, p.G, 0, st>>>(a);
    } else {
      if (a.y) {
        if (bf16) k_norm_bwd_wide<__nv_bfloat16><<<p.grid, p.G, 0, st>>>(a);
        else k_norm_bwd_wide<float><<<p.grid, p.G, 0, st>>>(a);
      }
      if (a.part) {
        nparts = (int)(a.rows < 32 ? a.rows : 32);
        const int64_t per = (a.rows + nparts - 1) / nparts;
        nparts = (int)((a.rows + per - 1) / per);
        const dim3 grid((unsigned)((a.cols + 255) / 256), (unsigned)nparts);
        if (bf16) k_norm_cols_wide<__nv_bfloat16><<<grid, 256, 0, st>>>(a, per);
        else k_norm_cols_wide<float><<<grid, 256, 0, st>>>(a, per);
      }
    }
  } else if (bf16) {
    if (vec) launch_held<__nv_bfloat16, 8>(a, p, bwd, st);
    else launch_held<__nv_bfloat16, 1>(a, p, bwd, st);
  } else {
    if (vec) launch_held<float, 4>(a, p, bwd, st);
    else launch_held<float, 1>(a, p, bwd, st);
  }
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return cuda_fail(e, "layer norm launch");
  if (bwd && a.part) {
    k_norm_cols<<<(a.cols + 31) / 32, 256, 0, st>>>(a.part, nparts, a.cols, a.dgamma, a.dbeta);
    return cuda_fail(cudaGetLastError(), "layer norm column sums launch");
  }
  return FQT_OK;
}

static bool ptr_aligned(const void *p, size_t n) {
  return reinterpret_cast<uintptr_t>(p) % n == 0;
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
