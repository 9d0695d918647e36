// fqt_clip.cu -- the global norm of a list of gradients, and the gradients scaled to
// a largest norm.
//
//   norm = sqrt(sum over tensors and entries of g^2)
//   out  = g max_norm / norm where norm > max_norm, else g
//
// Two passes over the gradients, bound by memory traffic: one adds the squares, one
// scales.  The tensors are cut into units of 32 KB, which CTAs take in turn whatever
// tensor they lie in, so that hundreds of small tensors cost one launch and a few large
// ones fill the GPU.  (A run of its own for every CTA balances better, but the second
// pass then took 42 us instead of 31 for the 102 MB of a ResNet-50.)  The second pass
// goes through the units backwards: what the first one read last is still in L2.  The
// 161 tensors of a ResNet-50 in fp32, 102 MB: 50 us on new gradients, 45.5 where the same
// ones are clipped again, of them the norm 19.1 (5.3 TB/s).  The second pass reads the
// part of the list from memory again that L2 did not keep, and writes as much.  Calls on
// four lists of 40 tensors in turn: 17 MB 13.4 us into other tensors and 11.7 in place,
// 102 MB 46.6 and 49.3, 400 MB 182 and 192.
#include <cuda_runtime.h>
#include <math.h>

#include "fqt.h"
#include "fqt_common.cuh"
#include "fqt_internal.h"

namespace fqt {

constexpr int kClipThreads = 256;
constexpr int kClipCtas = 3;  // of an SM
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
  uint32_t keep;  // the first unit of those that are to stay in L2
};

constexpr int kClipSmall = 40, kClipMid = 250, kClipLarge = 1020;  // 1.3, 8 and 32.6 KB
static_assert(sizeof(ClipTable<kClipLarge>) <= 32764 - 64, "launch parameters end at 32764 bytes");

// The entry of a unit: the last one in lo .. hi with unit0 <= unit.
template <int CAP>
__device__ __forceinline__ int clip_entry(const ClipTable<CAP> &t, int lo, int hi,
                                          uint32_t unit) {
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.e[mid].unit0 <= unit) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// A unit: `count` entries at `in` (and `out`): `head` entries before the first 16-byte
// boundary, whole vectors, and what is left.
struct ClipUnit {
  const char *in;
  char *out;
  int count, head, nvec;
  bool bf16;
};

__device__ __forceinline__ ClipUnit clip_unit(const ClipEntry &e, uint32_t unit) {
  const int es = e.bf16 ? 2 : 4, per = kClipUnitBytes / es;
  const int64_t first = (int64_t)(unit - e.unit0) * per;
  ClipUnit u;
  u.in = static_cast<const char *>(e.in) + first * es;
  u.out = static_cast<char *>(e.out) + first * es;
  u.count = (int)min((int64_t)per, e.count - first);
  u.bf16 = e.bf16;
  const int off = (int)(reinterpret_cast<uintptr_t>(u.in) & 15);
  u.head = min(u.count, off ? (16 - off) / es : 0);
  u.nvec = (u.count - u.head) / (16 / es);
  return u;
}

// Squares of fp32 entries leave fp32's range for entries outside 2^-63 .. 2^64, so
// the sum of a vector's squares says which of three sums it belongs to: as it is,
// or of the entries times 2^96 or 2^-96.  A thread adds the squares of a unit (at most
// 64, and one of the ends) in fp32, and all three sums of units are float-float: plain
// fp32 ones had lost 4e-5 of the norm after 2^32 equal entries.  An infinity would be NaN
// in them, so the entries that are no numbers are added up apart.  (No 64-bit
// arithmetic: this GPU's FP64 pipe made the sum of the CTAs' sums, in every CTA of the
// second pass, take 4 us.)
// The limits: a list has up to 2^39 vectors (2^41 entries, four of fp32 or more a
// vector), so a sum of vectors of at most 2^80 stays under 2^119; one of scaled vectors
// of less than 2^(192 - 110) under 2^121, and one of entries of up to 2^(128 - 96) under
// 2^107.  Within a vector that is scaled, what an entry loses lies 2^-37 below the sum.
constexpr float kMidLeast = 0x1p-110f, kMidMost = 0x1p80f;

struct alignas(16) Squares {
  ff mid;
  float others;  // 0 where the sums below are
  float none;    // 0, or no number
  ff small, big;
};
static_assert(sizeof(Squares) == 32, "two 16-byte words");

// A thread's sums of a unit.
struct UnitSquares {
  float mid, small, big, none;
};
__device__ __forceinline__ void add(Squares &s, const UnitSquares &u) {
  s.mid = ff_add(s.mid, {u.mid, 0.0f});
  if (u.small + u.big + u.none == 0.0f) return;
  s.others = 1.0f;
  s.small = ff_add(s.small, {u.small, 0.0f});
  s.big = ff_add(s.big, {u.big, 0.0f});
  s.none += u.none;
}

// The sum over the lanes that differ in the bits under 2 FIRST, in a fixed order.
template <int FIRST>
__device__ __forceinline__ ff warp_sum(ff x) {
#pragma unroll
  for (int o = FIRST; o > 0; o >>= 1)
    x = ff_add(x, {__shfl_xor_sync(0xffffffffu, x.h, o), __shfl_xor_sync(0xffffffffu, x.l, o)});
  return x;
}
// (Few lists hold others than the middle sum: adding up all took 1 us of a call.)
template <int FIRST>
__device__ __forceinline__ Squares warp_sum(Squares s) {
  const bool all = __any_sync(0xffffffffu, s.others != 0.0f);
  s.mid = warp_sum<FIRST>(s.mid);
  if (!all) return s;
  s.others = 1.0f;
  s.small = warp_sum<FIRST>(s.small);
  s.big = warp_sum<FIRST>(s.big);
#pragma unroll
  for (int o = FIRST; o > 0; o >>= 1) s.none += __shfl_xor_sync(0xffffffffu, s.none, o);
  return s;
}

// The sum over the CTA's threads, in thread 0, in a fixed order.
__device__ __forceinline__ Squares cta_sum(Squares s) {
  __shared__ Squares sums[kClipThreads / 32];
  s = warp_sum<16>(s);
  if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x < 32) s = warp_sum<kClipThreads / 64>(sums[threadIdx.x % (kClipThreads / 32)]);
  return s;
}

// sqrt of the sum as norm = root 2^k, root in [1, 2): the sums in units of 2^192, 1 or
// 2^-192, whichever is the largest that holds any (what is then lost is under 2^-24 of
// it).  Returns whether it is finite; a sum of 0 gives root 0.
__device__ __forceinline__ bool norm_of(const Squares &s, float *root, int *k) {
  float t = ff_round(s.mid);
  int unit = 0;
  if (s.big.h != 0.0f) {
    t = ff_round(s.big) + t * 0x1p-96f * 0x1p-96f;
    unit = 96;
  } else if (t > 0.0f) {
    t += ff_round(s.small) * 0x1p-96f * 0x1p-96f;
  } else {
    t = ff_round(s.small);
    unit = -96;
  }
  *k = 0;
  *root = 0.0f;
  if (!(s.none == 0.0f)) {  // NaN too
    *root = s.none;
    return false;
  }
  if (t == 0.0f) return true;
  int e;
  float m = frexpf(t, &e);  // m in [1/2, 1)
  e -= 1;                   // 2 m in [1, 2)
  *root = sqrtf(e & 1 ? 4.0f * m : 2.0f * m);
  *k = ((e - (e & 1)) >> 1) + unit;
  return true;
}

__device__ __forceinline__ void add_squares(UnitSquares &s, const float *x, int n) {
  float q = 0.0f;
  for (int i = 0; i < n; ++i) q = fmaf(x[i], x[i], q);
  if (q >= kMidLeast && q <= kMidMost) {
    s.mid += q;
    return;
  }
  const float f = q < 1.0f ? 0x1p96f : 0x1p-96f;
  float r = 0.0f;
  for (int i = 0; i < n; ++i) {
    const float y = x[i] * f;
    r = fmaf(y, y, r);
  }
  if (q < 1.0f) s.small += r;
  else if (isfinite(r)) s.big += r;
  else s.none += r;
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

// Cache policies: the entries that the first pass reads last, and the second pass first,
// are to stay in L2, what either reads or writes besides is not.  Four lists of fp32
// tensors in turn, with 56 MB kept, with nothing kept and with no policies: 17 MB 13.4,
// 13.8 and 14.1 us, 67 MB 32.2, 33.8 and 34.8, 102 MB 46.6, 48.9 and 50.1, 200 MB 91.0,
// 95.5 and 96.5, 400 MB 182, 191 and 192 (keeping 20 or 100 MB gains half of that or
// nothing).  Only where the output lies apart: in place there may be no second reading,
// and the entries would stay for nobody.
constexpr uint32_t kClipKeep = (56u << 20) / kClipUnitBytes;  // units

__device__ __forceinline__ uint64_t keep_policy() {
  uint64_t p;
  asm("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(p));
  return p;
}
__device__ __forceinline__ uint64_t pass_policy() {
  uint64_t p;
  asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(p));
  return p;
}
__device__ __forceinline__ uint4 load_as(const uint4 *p, uint64_t policy) {
  uint4 v;
  asm volatile("ld.global.L2::cache_hint.v4.u32 {%0, %1, %2, %3}, [%4], %5;"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p), "l"(policy)
               : "memory");
  return v;
}
__device__ __forceinline__ void store_as(uint4 *p, const uint4 &v, uint64_t policy) {
  asm volatile("st.global.L2::cache_hint.v4.u32 [%0], {%1, %2, %3, %4}, %5;" ::"l"(p), "r"(v.x),
               "r"(v.y), "r"(v.z), "r"(v.w), "l"(policy)
               : "memory");
}

template <int PER, bool APART>
__device__ __forceinline__ void add_unit(Squares &s, const ClipUnit &u, bool keep) {
  const bool bf16 = PER == 8;
  const uint64_t policy = keep ? keep_policy() : pass_policy();
  const uint4 *body = reinterpret_cast<const uint4 *>(u.in + u.head * (16 / PER));
  uint4 v[kClipVecs];
#pragma unroll
  for (int k = 0; k < kClipVecs; ++k) {
    const int i = k * kClipThreads + threadIdx.x;
    v[k] = make_uint4(0u, 0u, 0u, 0u);
    if (i < u.nvec) v[k] = APART ? load_as(body + i, policy) : __ldg(body + i);
  }
  UnitSquares sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int k = 0; k < kClipVecs; ++k) {
    float x[8];
    widen(v[k], bf16, x);
    add_squares(sum, x, PER);
  }
  // what lies outside the 16-byte vectors: under PER entries at either end
  if ((int)threadIdx.x < u.count - u.nvec * PER) {
    const int i = (int)threadIdx.x < u.head ? threadIdx.x : threadIdx.x + u.nvec * PER;
    const float x = one_entry(u.in, i, bf16);
    add_squares(sum, &x, 1);
  }
  add(s, sum);
}

// part[CTA]: the sum of its units' squares.
template <int CAP, bool APART>
__global__ void __launch_bounds__(kClipThreads, kClipCtas)
    k_clip_squares(const __grid_constant__ ClipTable<CAP> t, Squares *part) {
  let_next_start();
  wait_for_previous();
  Squares s = {};
  int e = 0;
  for (uint32_t unit = blockIdx.x; unit < t.units; unit += gridDim.x) {
    if (e + 1 < t.n && t.e[e + 1].unit0 <= unit) e = clip_entry(t, e + 1, t.n - 1, unit);
    const ClipUnit u = clip_unit(t.e[e], unit);
    const bool keep = unit >= t.keep;
    if (u.bf16) add_unit<8, APART>(s, u, keep);
    else add_unit<4, APART>(s, u, keep);
  }
  s = cta_sum(s);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

// The factor f times a power of two p.  p is 1 unless the factor is below 2^-100, where
// f alone would leave fp32's normal numbers and the products, no smaller for it than
// the largest norm asked for, would have as few bits as f.  Then f is 1/4 to 1/2 (p is
// not below 2^-148), so x f does not overflow and x f p is rounded once.
struct Factor {
  float f, p;
  __device__ __forceinline__ bool one() const { return f == 1.0f; }
  __device__ __forceinline__ float of(float x) const { return x * f * p; }
};

// quotient 2^-k, the quotient in fp32
__device__ __forceinline__ Factor make_factor(float quotient, int k) {
  int e;
  const float m = frexpf(quotient, &e);  // m in [1/2, 1), or 0
  if (e - k >= -100) return {ldexpf(quotient, -k), 1.0f};
  const int down = min(k - e - 1, 148);
  return {ldexpf(m, e - k + down), ldexpf(1.0f, -down)};
}

// The factor, from the partial sums (every CTA adds them in the same order); CTA 0
// writes the norm.
__device__ __forceinline__ Factor clip_factor(const Squares *part, int nparts, float max_norm,
                                             float *norm_out, int *status) {
  __shared__ Factor factor;
  Squares s = {};
  for (int i = threadIdx.x; i < nparts; i += kClipThreads) {
    const float4 v = __ldcg(reinterpret_cast<const float4 *>(part + i));
    s.mid = ff_add(s.mid, {v.x, v.y});
    s.others += v.z;
    s.none += v.w;
  }
  if (s.others != 0.0f) {
    for (int i = threadIdx.x; i < nparts; i += kClipThreads) {
      const float4 v = __ldcg(reinterpret_cast<const float4 *>(part + i) + 1);
      s.small = ff_add(s.small, {v.x, v.y});
      s.big = ff_add(s.big, {v.z, v.w});
    }
  }
  s = cta_sum(s);
  if (threadIdx.x == 0) {
    float root;
    int k;
    const bool good = norm_of(s, &root, &k);
    const float norm = ldexpf(root, k);  // infinite where it passes fp32
    // max_norm / norm, the quotient of numbers in fp32's middle first
    factor = good && norm > max_norm ? make_factor(max_norm / root, k) : Factor{1.0f, 1.0f};
    if (blockIdx.x == 0) {
      if (norm_out) *norm_out = norm;
      if (!good) record_status(status, FQT_ENONFINITE);
    }
  }
  __syncthreads();
  return factor;
}

template <int PER, bool APART>
__device__ __forceinline__ void scale_unit(const ClipUnit &u, const Factor f) {
  const bool bf16 = PER == 8;
  // vectors where the output lies on the same bytes of 16 as the input
  const bool vec = ((reinterpret_cast<uintptr_t>(u.in) ^ reinterpret_cast<uintptr_t>(u.out)) &
                    15) == 0;
  const int head = vec ? u.head : 0, nvec = vec ? u.nvec : 0;
  const uint4 *in = reinterpret_cast<const uint4 *>(u.in + head * (16 / PER));
  uint4 *out = reinterpret_cast<uint4 *>(u.out + head * (16 / PER));
  const uint64_t policy = pass_policy();
  uint4 v[kClipVecs];
#pragma unroll
  for (int k = 0; k < kClipVecs; ++k) {
    const int i = k * kClipThreads + threadIdx.x;
    if (i < nvec) v[k] = APART ? load_as(in + i, policy) : in[i];
  }
#pragma unroll
  for (int k = 0; k < kClipVecs; ++k) {
    const int i = k * kClipThreads + threadIdx.x;
    if (i >= nvec) continue;
    float x[8];
    widen(v[k], bf16, x);
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (bf16) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(f.of(x[2 * j]), f.of(x[2 * j + 1]));
        w[j] = *reinterpret_cast<const uint32_t *>(&b);
      } else {
        w[j] = __float_as_uint(f.of(x[j]));
      }
    }
    const uint4 y = f.one() ? v[k] : make_uint4(w[0], w[1], w[2], w[3]);
    if constexpr (APART) store_as(out + i, y, policy);
    else out[i] = y;
  }
  // the ends, or a unit without vectors
  const int rest = u.count - nvec * PER;
  for (int j = threadIdx.x; j < rest; j += kClipThreads) {
    const int i = j < head ? j : j + nvec * PER;
    if (bf16) {
      const unsigned short raw = reinterpret_cast<const unsigned short *>(u.in)[i];
      const __nv_bfloat16 y = __float2bfloat16_rn(f.of(one_entry(u.in, i, true)));
      reinterpret_cast<unsigned short *>(u.out)[i] = f.one() ? raw : __bfloat16_as_ushort(y);
    } else {
      const uint32_t raw = reinterpret_cast<const uint32_t *>(u.in)[i];
      reinterpret_cast<uint32_t *>(u.out)[i] =
          f.one() ? raw : __float_as_uint(f.of(__uint_as_float(raw)));
    }
  }
}

template <int CAP, bool APART>
__global__ void __launch_bounds__(kClipThreads, kClipCtas)
    k_clip_scale(const __grid_constant__ ClipTable<CAP> t, const Squares *part, int nparts,
                 float max_norm, float *norm_out, int *status) {
  let_next_start();
  wait_for_previous();
  const Factor f = clip_factor(part, nparts, max_norm, norm_out, status);
  int e = t.n - 1;
  // the units of the CTA of this number in the first pass, from the last to the first
  const uint32_t mine = (t.units - 1 - blockIdx.x) / gridDim.x;
  for (uint32_t k = 0; k <= mine; ++k) {
    const uint32_t unit = blockIdx.x + (mine - k) * gridDim.x;
    if (t.e[e].unit0 > unit) e = clip_entry(t, 0, e - 1, unit);
    if (f.one() && t.e[e].in == t.e[e].out) continue;  // nothing to change in place
    const ClipUnit u = clip_unit(t.e[e], unit);
    if (u.bf16) scale_unit<8, APART>(u, f);
    else scale_unit<4, APART>(u, f);
  }
}

// The norm alone.
__global__ void __launch_bounds__(kClipThreads)
    k_clip_norm(const Squares *part, int nparts, float *norm_out, int *status) {
  let_next_start();
  wait_for_previous();
  clip_factor(part, nparts, INFINITY, norm_out, status);
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
static int clip_grid(int nsm) { return kClipCtas * nsm; }

size_t clip_ws_bytes(int64_t n) {
  const int64_t launches = n > 0 ? (n + kClipLarge - 1) / kClipLarge : 1;
  return kHeaderBytes + (size_t)launches * clip_grid(device_sm_count()) * sizeof(Squares);
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
  t.keep = t.units > kClipKeep ? t.units - kClipKeep : 0;
  return i;
}

template <int CAP, bool APART>
static fqt_status clip_lists(const fqt_tensor *in, const fqt_tensor *out, int64_t n,
                             float max_norm, float *norm, void *ws, cudaStream_t st) {
  const int most = clip_grid(device_sm_count());
  Squares *part = reinterpret_cast<Squares *>(static_cast<char *>(ws) + kHeaderBytes);
  int *status = static_cast<int *>(ws);
  ClipTable<CAP> t;
  int nparts = 0;
  for (int64_t i = 0; i < n;) {
    i = fill_table(t, in, out, i, n);
    if (t.units == 0) continue;
    const int grid = t.units < (uint32_t)most ? (int)t.units : most;
    const cudaError_t e = launch_behind(k_clip_squares<CAP, APART>, dim3((unsigned)grid),
                                        kClipThreads, 0, st, t, part + nparts);
    if (e != cudaSuccess) return cuda_fail(e, "gradient norm launch");
    nparts += grid;
  }
  if (!out || nparts == 0) {
    const cudaError_t e =
        launch_behind(k_clip_norm, dim3(1), kClipThreads, 0, st, (const Squares *)part, nparts,
                      norm, status);
    return cuda_fail(e, "gradient norm launch");
  }
  bool first = true;
  for (int64_t i = 0; i < n;) {
    if (n > CAP) i = fill_table(t, in, out, i, n);
    else i = n;  // the table is still there
    if (t.units == 0) continue;
    const int grid = t.units < (uint32_t)most ? (int)t.units : most;
    const cudaError_t e =
        launch_behind(k_clip_scale<CAP, APART>, dim3((unsigned)grid), kClipThreads, 0, st, t,
                      (const Squares *)part, nparts, max_norm, first ? norm : nullptr, status);
    if (e != cudaSuccess) return cuda_fail(e, "gradient clipping launch");
    first = false;
  }
  return FQT_OK;
}

template <bool APART>
static fqt_status clip_as(const fqt_tensor *in, const fqt_tensor *out, int64_t n, float max_norm,
                          float *norm, void *ws, cudaStream_t st) {
  if (n <= kClipSmall) return clip_lists<kClipSmall, APART>(in, out, n, max_norm, norm, ws, st);
  if (n <= kClipMid) return clip_lists<kClipMid, APART>(in, out, n, max_norm, norm, ws, st);
  return clip_lists<kClipLarge, APART>(in, out, n, max_norm, norm, ws, st);
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
      if ((total += g.count) > ((int64_t)1 << 41)) return FQT_EINVAL;
    }
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256 || ws_bytes < clip_ws_bytes(n))
    return FQT_EWORKSPACE;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  bool apart = false;
  for (int64_t i = 0; out && i < n; ++i) apart |= out[i].data != grads[i].data;
  return apart ? clip_as<true>(grads, out, n, max_norm, norm, workspace, st)
               : clip_as<false>(grads, out, n, max_norm, norm, workspace, st);
}

}  // extern "C"
