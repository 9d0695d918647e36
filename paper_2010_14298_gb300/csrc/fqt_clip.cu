// fqt_clip.cu -- the global norm of a list of gradients, and the gradients scaled to
// a largest norm.
//
//   norm = sqrt(sum over tensors and entries of g^2)
//   out  = g max_norm / norm where norm > max_norm, else g
//
// Two passes over the gradients, bound by memory traffic: one adds the squares, one
// scales.  The tensors are cut into units of 32 KB, which CTAs take in a fixed order
// whatever tensor they lie in, so that hundreds of small tensors cost one launch and
// a few large ones still fill the GPU.  The second pass runs through the units
// backwards: what the first one read last is still in L2.
#include <cuda_runtime.h>
#include <math.h>

#include "fqt.h"
#include "fqt_common.cuh"
#include "fqt_internal.h"

namespace fqt {

constexpr int kClipThreads = 256;
constexpr int kClipVecs = 8;  // 16-byte loads of a thread per unit
constexpr int kClipUnitBytes = kClipThreads * kClipVecs * 16;

struct ClipEntry {
  const void *in;
  void *out;
  int64_t count;
  uint32_t unit0;  // units of the entries before it
  uint32_t bf16;
};

// The list travels as a launch parameter: the calls copy nothing and can be
// captured, and the tensors may change from call to call.
template <int CAP>
struct ClipTable {
  ClipEntry e[CAP];
  int n;
  uint32_t units;
};

constexpr int kClipSmall = 40, kClipMid = 250, kClipLarge = 1020;  // 1.3, 8 and 32.6 KB
static_assert(sizeof(ClipTable<kClipLarge>) <= 32764 - 64, "launch parameters end at 32764 bytes");

template <int CAP>
__device__ __forceinline__ int clip_entry(const ClipTable<CAP> &t, uint32_t unit) {
  int lo = 0, hi = t.n - 1;  // the last entry with unit0 <= unit
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.e[mid].unit0 <= unit) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// A unit of an entry: `count` entries at `in` (and `out`).
struct ClipUnit {
  const char *in;
  char *out;
  int count;
  bool bf16;
};

template <int CAP>
__device__ __forceinline__ ClipUnit clip_unit(const ClipTable<CAP> &t, uint32_t unit) {
  const ClipEntry &e = t.e[clip_entry(t, unit)];
  const int per = kClipUnitBytes / (e.bf16 ? 2 : 4);
  const int64_t at = (int64_t)(unit - e.unit0) * per;
  ClipUnit u;
  u.in = static_cast<const char *>(e.in) + at * (e.bf16 ? 2 : 4);
  u.out = static_cast<char *>(e.out) + at * (e.bf16 ? 2 : 4);
  u.count = (int)min((int64_t)per, e.count - at);
  u.bf16 = e.bf16;
  return u;
}

// Squares of fp32 entries leave fp32's range for entries outside 2^-63 .. 2^64, so
// the sum of a vector's squares says which of three sums it belongs to: as it is,
// or of the entries times 2^96 or 2^-96.  (An entry that is no number is in the last
// one.)  The sums that count in practice are float-float per thread.
struct Squares {
  ff mid;
  float small, big;
};

__device__ __forceinline__ void add_squares(Squares &s, float &unit, const float *x, int n) {
  float q = 0.0f;
  for (int i = 0; i < n; ++i) q = fmaf(x[i], x[i], q);
  if (q >= 0x1p-100f && q <= 0x1p100f) {
    unit += q;
    return;
  }
  const float f = q < 1.0f ? 0x1p96f : 0x1p-96f;
  float r = 0.0f;
  for (int i = 0; i < n; ++i) {
    const float y = x[i] * f;
    r = fmaf(y, y, r);
  }
  if (q < 1.0f) s.small += r;
  else s.big += r;
}

__device__ __forceinline__ void widen(const uint4 &v, bool bf16, float (&x)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (bf16) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    } else {
      x[i] = __uint_as_float(w[i]);
    }
  }
}

__device__ __forceinline__ float one_entry(const char *p, int i, bool bf16) {
  if (bf16) return __uint_as_float((uint32_t) reinterpret_cast<const unsigned short *>(p)[i] << 16);
  return reinterpret_cast<const float *>(p)[i];
}

// Entries before the first 16-byte boundary, at most the unit's.
__device__ __forceinline__ int unit_head(const ClipUnit &u) {
  const int off = (int)(reinterpret_cast<uintptr_t>(u.in) & 15);
  return min(u.count, off ? (16 - off) / (u.bf16 ? 2 : 4) : 0);
}

// part[CTA]: the sum of its units' squares.
template <int CAP>
__global__ void __launch_bounds__(kClipThreads)
    k_clip_squares(const __grid_constant__ ClipTable<CAP> t, double *part) {
  __shared__ double sums[kClipThreads / 32];
  Squares s = {{0.0f, 0.0f}, 0.0f, 0.0f};
  for (uint32_t unit = blockIdx.x; unit < t.units; unit += gridDim.x) {
    const ClipUnit u = clip_unit(t, unit);
    const int head = unit_head(u), per = u.bf16 ? 8 : 4;
    const int nvec = (u.count - head) / per;
    const uint4 *body =
        reinterpret_cast<const uint4 *>(u.in + (size_t)head * (u.bf16 ? 2 : 4));
    uint4 v[kClipVecs];
#pragma unroll
    for (int k = 0; k < kClipVecs; ++k) {
      const int i = k * kClipThreads + threadIdx.x;
      v[k] = i < nvec ? body[i] : make_uint4(0u, 0u, 0u, 0u);
    }
    float sum = 0.0f;
#pragma unroll
    for (int k = 0; k < kClipVecs; ++k) {
      float x[8];
      widen(v[k], u.bf16, x);
      if (u.bf16) add_squares(s, sum, x, 8);
      else add_squares(s, sum, x, 4);
    }
    // what lies outside the 16-byte vectors: under 8 entries at either end
    const int tail = u.count - head - nvec * per;
    if (threadIdx.x < head + tail) {
      const int i = (int)threadIdx.x < head ? threadIdx.x : head + nvec * per + threadIdx.x - head;
      const float x = one_entry(u.in, i, u.bf16);
      add_squares(s, sum, &x, 1);
    }
    s.mid = ff_add(s.mid, {sum, 0.0f});
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const ff m = {__shfl_xor_sync(0xffffffffu, s.mid.h, o),
                  __shfl_xor_sync(0xffffffffu, s.mid.l, o)};
    s.mid = ff_add(s.mid, m);
    s.small += __shfl_xor_sync(0xffffffffu, s.small, o);
    s.big += __shfl_xor_sync(0xffffffffu, s.big, o);
  }
  if ((threadIdx.x & 31) == 0)
    sums[threadIdx.x >> 5] = (double)s.mid.h + (double)s.mid.l + (double)s.small * 0x1p-192 +
                             (double)s.big * 0x1p192;
  __syncthreads();
  if (threadIdx.x == 0) {
    double total = 0.0;
    for (int w = 0; w < kClipThreads / 32; ++w) total += sums[w];
    part[blockIdx.x] = total;
  }
}

// The factor, from the partial sums (every CTA adds them in the same order); CTA 0
// writes the norm.
__device__ __forceinline__ float clip_factor(const double *part, int nparts, float max_norm,
                                             float *norm_out, int *status) {
  __shared__ double sums[kClipThreads / 32];
  __shared__ float factor;
  double s = 0.0;
  for (int i = threadIdx.x; i < nparts; i += kClipThreads) s += part[i];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    double total = 0.0;
    for (int w = 0; w < kClipThreads / 32; ++w) total += sums[w];
    const double norm = sqrt(total);
    const bool good = isfinite(norm);
    factor = good && norm > (double)max_norm ? (float)((double)max_norm / norm) : 1.0f;
    if (blockIdx.x == 0) {
      if (norm_out) *norm_out = (float)norm;
      if (!good) record_status(status, FQT_ENONFINITE);
    }
  }
  __syncthreads();
  return factor;
}

template <int CAP>
__global__ void __launch_bounds__(kClipThreads)
    k_clip_scale(const __grid_constant__ ClipTable<CAP> t, const double *part, int nparts,
                 float max_norm, float *norm_out, int *status) {
  const float f = clip_factor(part, nparts, max_norm, norm_out, status);
  for (uint32_t k = blockIdx.x; k < t.units; k += gridDim.x) {
    const ClipUnit u = clip_unit(t, t.units - 1 - k);
    if (f == 1.0f && u.in == u.out) continue;  // nothing to change in place
    const int es = u.bf16 ? 2 : 4, per = 16 / es;
    // vectors where the output lies on the same bytes of 16 as the input
    const bool vec = ((reinterpret_cast<uintptr_t>(u.in) ^ reinterpret_cast<uintptr_t>(u.out)) &
                      15) == 0;
    const int head = vec ? unit_head(u) : 0;
    const int nvec = vec ? (u.count - head) / per : 0;
    const uint4 *in = reinterpret_cast<const uint4 *>(u.in + (size_t)head * es);
    uint4 *out = reinterpret_cast<uint4 *>(u.out + (size_t)head * es);
    uint4 v[kClipVecs];
#pragma unroll
    for (int i = 0; i < kClipVecs; ++i) {
      const int at = i * kClipThreads + threadIdx.x;
      if (at < nvec) v[i] = in[at];
    }
#pragma unroll
    for (int i = 0; i < kClipVecs; ++i) {
      const int at = i * kClipThreads + threadIdx.x;
      if (at >= nvec) continue;
      float x[8];
      widen(v[i], u.bf16, x);
      uint32_t w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (u.bf16) {
          const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * j] * f, x[2 * j + 1] * f);
          w[j] = *reinterpret_cast<const uint32_t *>(&b);
        } else {
          w[j] = __float_as_uint(x[j] * f);
        }
      }
      out[at] = f == 1.0f ? v[i] : make_uint4(w[0], w[1], w[2], w[3]);
    }
    // the ends, or a unit without vectors
    const int rest = u.count - nvec * per;
    for (int j = threadIdx.x; j < rest; j += kClipThreads) {
      const int i = j < head ? j : j + nvec * per;
      const float x = one_entry(u.in, i, u.bf16) * f;
      if (u.bf16) reinterpret_cast<__nv_bfloat16 *>(u.out)[i] = __float2bfloat16_rn(x);
      else reinterpret_cast<float *>(u.out)[i] = x;
    }
  }
}

// The norm alone.
__global__ void __launch_bounds__(kClipThreads)
    k_clip_norm(const double *part, int nparts, float *norm_out, int *status) {
  clip_factor(part, nparts, INFINITY, norm_out, status);
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
static int clip_grid(int nsm) { return 3 * nsm; }

size_t clip_ws_bytes(int64_t n) {
  const int64_t launches = n > 0 ? (n + kClipLarge - 1) / kClipLarge : 1;
  return kHeaderBytes + (size_t)launches * clip_grid(device_sm_count()) * sizeof(double);
}

// Entries first .. of the lists, as many as a table holds; returns the next one.
template <int CAP>
static int64_t fill_table(ClipTable<CAP> &t, const fqt_tensor *in, const fqt_tensor *out,
                          int64_t first, int64_t n) {
  t.n = 0;
  t.units = 0;
  int64_t i = first;
  for (; i < n && t.n < CAP; ++i) {
    if (in[i].count == 0) continue;
    const int64_t per = kClipUnitBytes / (in[i].dtype == FQT_BF16 ? 2 : 4);
    t.e[t.n++] = {in[i].data, out ? out[i].data : nullptr, in[i].count, t.units,
                  in[i].dtype == FQT_BF16 ? 1u : 0u};
    t.units += (uint32_t)((in[i].count + per - 1) / per);
  }
  return i;
}

template <int CAP>
static fqt_status clip_lists(const fqt_tensor *in, const fqt_tensor *out, int64_t n,
                             float max_norm, float *norm, void *ws, cudaStream_t st) {
  const int most = clip_grid(device_sm_count());
  double *part = reinterpret_cast<double *>(static_cast<char *>(ws) + kHeaderBytes);
  int *status = static_cast<int *>(ws);
  ClipTable<CAP> t;
  int nparts = 0;
  for (int64_t i = 0; i < n;) {
    i = fill_table(t, in, out, i, n);
    if (t.units == 0) continue;
    const int grid = t.units < (uint32_t)most ? (int)t.units : most;
    k_clip_squares<CAP><<<grid, kClipThreads, 0, st>>>(t, part + nparts);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return cuda_fail(e, "gradient norm launch");
    nparts += grid;
  }
  if (!out || nparts == 0) {
    k_clip_norm<<<1, kClipThreads, 0, st>>>(part, nparts, norm, status);
    return cuda_fail(cudaGetLastError(), "gradient norm launch");
  }
  bool first = true;
  for (int64_t i = 0; i < n;) {
    if (n > CAP) i = fill_table(t, in, out, i, n);
    else i = n;  // the table is still there
    if (t.units == 0) continue;
    const int grid = t.units < (uint32_t)most ? (int)t.units : most;
    k_clip_scale<CAP><<<grid, kClipThreads, 0, st>>>(t, part, nparts, max_norm,
                                                     first ? norm : nullptr, status);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return cuda_fail(e, "gradient clipping launch");
    first = false;
  }
  return FQT_OK;
}

}  // namespace fqt

using namespace fqt;

extern "C" {

size_t fqt_clip_grad_norm_workspace_size(int64_t n) { return clip_ws_bytes(n); }

fqt_status fqt_clip_grad_norm(const fqt_tensor *grads, const fqt_tensor *out, int64_t n,
                              float max_norm, float *norm, void *workspace, size_t ws_bytes,
                              void *stream) {
  if (n < 0 || n > (1 << 24) || (n > 0 && !grads)) return FQT_EINVAL;
  if (out ? !(max_norm >= 0.0f) : !norm) return FQT_EINVAL;
  if (reinterpret_cast<uintptr_t>(norm) % 4) return FQT_EINVAL;
  int64_t total = 0;
  for (int64_t i = 0; i < n; ++i)
    for (const fqt_tensor *l : {grads, out}) {
      if (!l) continue;
      const fqt_tensor &g = l[i];
      if (g.dtype != FQT_F32 && g.dtype != FQT_BF16) return FQT_EINVAL;
      if (g.count < 0 || g.count > ((int64_t)1 << 40)) return FQT_EINVAL;
      if (g.count != grads[i].count || g.dtype != grads[i].dtype) return FQT_EINVAL;
      if (g.count > 0 &&
          (!g.data || reinterpret_cast<uintptr_t>(g.data) % (g.dtype == FQT_BF16 ? 2 : 4)))
        return FQT_EINVAL;
      if ((total += g.count) > ((int64_t)1 << 44)) return FQT_EINVAL;
    }
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256 || ws_bytes < clip_ws_bytes(n))
    return FQT_EWORKSPACE;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  if (n <= kClipSmall) return clip_lists<kClipSmall>(grads, out, n, max_norm, norm, workspace, st);
  if (n <= kClipMid) return clip_lists<kClipMid>(grads, out, n, max_norm, norm, workspace, st);
  return clip_lists<kClipLarge>(grads, out, n, max_norm, norm, workspace, st);
}

}  // extern "C"
