// fqt_gated.cu -- a gated feed-forward block in 8-bit floating point:
//
//   g = A Bg^T, u = A Bu^T, a = act(g) u       (one kernel)
//   dg = da u act'(g), du = da act(g)          from g and u held in 8 bits
#include "fqt_gated.cuh"

namespace fqt {

// ---------------------------------------------------------------------------
// Forward
// ---------------------------------------------------------------------------
static bool make_map_f8_codes_out(CUtensorMap *m, const fqt_fp8 *q) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[2] = {(cuuint64_t)q->cols, (cuuint64_t)q->rows};
  cuuint64_t strides[1] = {(cuuint64_t)q->pitch};
  cuuint32_t box[2] = {64, 32};
  cuuint32_t one[2] = {1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, q->codes, dims, strides, box, one,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B,
            CU_TENSOR_MAP_L2_PROMOTION_NONE,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

static F8Codes codes_of(const fqt_fp8 *q) {
  return q ? F8Codes{q->codes, q->scales, q->pitch} : F8Codes{nullptr, nullptr, 0};
}

static fqt_status fp8_gated_matmul(const fqt_fp8 *A, const fqt_fp8 *Bg, const fqt_fp8 *Bu,
                                   fqt_act act, bool bf16, void *out, int64_t ldo,
                                   const fqt_fp8 *q, const fqt_fp8 *gate, const fqt_fp8 *up,
                                   void *ws, cudaStream_t st) {
  const int nsm = device_sm_count();
  const int64_t M = A->rows, N = Bg->rows;
  F8GatedArgs g = {};
  g.nkb = g.kb_per = (int)((A->cols + kF8Block - 1) / kF8Block);
  g.status = static_cast<int *>(ws);
  g.out = out;
  g.ldo = M > 1 ? ldo : N;
  // (without a dense output the sums are rounded to fewer digits than bf16's)
  g.bf16 = bf16 || !out;
  g.act = act;
  g.q = codes_of(q);
  g.gate = codes_of(gate);
  g.up = codes_of(up);
  g.sp = scale_rows(M);
  g.splits = 1;
  const fqt_fp8 *w = Bg;
  g.s2 = reinterpret_cast<const uint32_t *>(Bu->scales);
  F8Of<F8_GATED>::Maps maps = {};
  if (M <= 64) {  // few tokens: the weights' rows fill the 128 rows of a tile
    const int nt = M <= 32 ? 32 : 64;
    // 32 columns of each projection to a CTA, 64 where that would be more CTAs than SMs
    g.part = (N + 31) / 32 <= nsm ? 32 : 64;
    // CTAs that hold blocks of 128 columns together
    if (q || gate || up) g.splits = kF8Block / g.part;
    const int64_t run = (int64_t)g.part * g.splits;
    g.items = (N + run - 1) / run * g.splits;
    g.swap = 1;
    g.sa = reinterpret_cast<const uint32_t *>(w->scales);
    g.sb = reinterpret_cast<const uint32_t *>(A->scales);
    g.spa = scale_rows(N);
    g.spb = scale_rows(M);
    g.M = N;
    g.N = M;
    if (!make_map_codes(&maps.a, Bg, (uint32_t)g.part) ||
        !make_map_codes(&maps.b2, Bu, (uint32_t)g.part) ||
        !make_map_codes(&maps.b, A, (uint32_t)nt))
      return cuda_fail(cudaErrorUnknown, "FP8 tensor map");
    if (nt == 32) return launch_f8<32, 2, false, F8_GATED>(maps, g, nsm, st);
    return launch_f8<64, 2, false, F8_GATED>(maps, g, nsm, st);
  }
  // super tiles of 256 tokens x 128 columns of both where they occupy three quarters of
  // the SMs, else 128 tokens to a CTA
  const int64_t n_tiles = (N + kF8Block - 1) / kF8Block;
  const bool pair = nsm >= 2 && (M + 255) / 256 * n_tiles * 8 >= (int64_t)nsm * 3;
  const int rows = pair ? 2 * BM : BM;
  g.m_tiles = (int)((M + rows - 1) / rows);
  g.n_tiles = (int)n_tiles;
  g.items = (int64_t)g.m_tiles * g.n_tiles;
  g.sa = reinterpret_cast<const uint32_t *>(A->scales);
  g.sb = reinterpret_cast<const uint32_t *>(w->scales);
  g.spa = scale_rows(M);
  g.spb = scale_rows(N);
  g.M = M;
  g.N = N;
  const int es = bf16 ? 2 : 4;
  g.boxes = out && f8_aligned(out, 16) && g.ldo * es % 16 == 0 && N * es % 16 == 0;
  if (!make_map_codes(&maps.a, A, BM) || !make_map_codes(&maps.b, Bg, BM) ||
      !make_map_codes(&maps.b2, Bu, BM) ||
      (g.boxes && !make_map_f8_out(&maps.out, out, bf16, M, N, g.ldo)) ||
      (q && !make_map_f8_codes_out(&maps.q, q)) ||
      (gate && !make_map_f8_codes_out(&maps.gate, gate)) ||
      (up && !make_map_f8_codes_out(&maps.up, up)))
    return cuda_fail(cudaErrorUnknown, "FP8 tensor map");
  if (pair) return launch_f8<256, 1, true, F8_GATED>(maps, g, nsm, st);
  return launch_f8<256, 1, false, F8_GATED>(maps, g, nsm, st);
}

// ---------------------------------------------------------------------------
// Backward
// ---------------------------------------------------------------------------
struct F8GatedBackArgs {
  const void *da;
  int64_t ldda, rows;
  int cols;
  F8Codes gate, up;  // read
  int64_t sp, spt;   // rows of scales, of matrices and of their transposes
  void *dgate, *dup;
  int64_t lddg, lddu;
  F8Codes q[2], qt[3];  // dg, du; their transposes and a's
  int *status;
};

// E4M3 codes 2 i and 2 i + 1 of a word, as fp32 (exact in fp16 on the way).
__device__ __forceinline__ float2 f8_two(uint32_t w, int i) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)(w >> 16 * i)));
  return __half22float2(*reinterpret_cast<const __half2 *>(&h));
}

// Eight codes of a row, zeros past `left`.
__device__ __forceinline__ uint2 f8_eight(const uint8_t *p, int64_t left) {
  if (left <= 0) return make_uint2(0u, 0u);
  uint2 w = __ldg(reinterpret_cast<const uint2 *>(p));
  if (left < 8) {
    if (left <= 4) w.y = 0u;
    uint32_t &last = left <= 4 ? w.x : w.y;
    const int keep = (int)(left - 1) % 4 + 1;
    if (keep < 4) last &= (1u << 8 * keep) - 1u;
  }
  return w;
}

__device__ __forceinline__ float f8_scale_of(uint8_t e) { return pow2((int)e - 127); }

constexpr int kF8BackThreads = 512, kF8BackWarps = kF8BackThreads / 32;
// a tensor's column maxima by warp, its columns' reciprocal scales, and its transposed codes
struct F8BackShared {
  uint32_t top[3][kF8BackWarps][kF8Block];
  float inv[3][kF8Block];
  uint32_t tr[3][kF8Block * 32];
};

// One CTA per 128 x 128 tile; a thread holds 4 rows x 8 columns of dg, du and a, so it
// packs codes along either axis without exchanging bytes (as the quantizer of both axes).
template <typename T, int ACT>
__global__ void __launch_bounds__(kF8BackThreads, 1) k_f8_gated_back(const F8GatedBackArgs a,
                                                                     const bool vec) {
  extern __shared__ __align__(16) uint8_t raw[];
  F8BackShared &s = *reinterpret_cast<F8BackShared *>(raw);
  let_next_start();
  wait_for_previous();
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  const int cg = t & 15, rg = t >> 4;
  const int64_t r0 = (int64_t)blockIdx.x * kF8Block, c0 = (int64_t)blockIdx.y * kF8Block;
  const int64_t row = r0 + rg * 4, col = c0 + cg * 8;
  F8Raw<T, 8> da[4];
  uint2 cgate[4], cup[4];
  float sg[4], su[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t left = row + i < a.rows ? a.cols - col : 0;
    const T *p = static_cast<const T *>(a.da) + (row + i) * a.ldda + col;
    da[i].load(p, vec ? left : min(left, (int64_t)7));
    if (!vec && left >= 8) da[i].set(7, p[7]);
    cgate[i] = f8_eight(a.gate.codes + (row + i) * a.gate.pitch + col, left);
    cup[i] = f8_eight(a.up.codes + (row + i) * a.up.pitch + col, left);
    const int64_t at = scale_at(blockIdx.y, a.sp, min(row + i, a.rows - 1));
    sg[i] = f8_scale_of(__ldg(a.gate.scales + at));
    su[i] = f8_scale_of(__ldg(a.up.scales + at));
  }
  // v[0]: dg, v[1]: du, v[2]: a (fp32 bits)
  uint32_t v[3][4][8];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
      const float2 g2 = f8_two(j < 4 ? cgate[i].x : cgate[i].y, (j >> 1) & 1);
      const float2 u2 = f8_two(j < 4 ? cup[i].x : cup[i].y, (j >> 1) & 1);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const float u = (k ? u2.y : u2.x) * su[i], d = da[i].f(j + k);
        float act, slope;
        act_and_slope<ACT>((k ? g2.y : g2.x) * sg[i], act, slope);
        v[0][i][j + k] = __float_as_uint(d * u * slope);
        v[1][i][j + k] = __float_as_uint(d * act);
        v[2][i][j + k] = __float_as_uint(act * u);
      }
    }
  // dense outputs
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    T *out = static_cast<T *>(k ? a.dup : a.dgate);
    if (!out) continue;
    const int64_t ld = k ? a.lddu : a.lddg;
    const bool wide = f8_pitch_aligned<T>(out, ld);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (row + i >= a.rows) break;
      T *p = out + (row + i) * ld + col;
      if (wide && col + 8 <= a.cols) {
#pragma unroll
        for (int j = 0; j < 8; j += 16 / (int)sizeof(T))
          *reinterpret_cast<uint4 *>(p + j) = f8_pack<T>(&v[k][i][j]);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (col + j < a.cols) p[j] = f8_out<T>(__uint_as_float(v[k][i][j]));
      }
    }
  }
  if (!a.q[0].codes && !a.q[1].codes && !a.qt[0].codes && !a.qt[1].codes && !a.qt[2].codes) return;
  // entries that are not finite count for no scale and take the NaN code
  uint32_t rm[2][4];
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    if (!a.qt[k].codes && (k == 2 || !a.q[k].codes)) continue;
    uint32_t m = 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t r = 0u;
#pragma unroll
      for (int j = 0; j < 8; ++j) r = max(r, v[k][i][j] & 0x7FFFFFFFu);
      if (k < 2) rm[k][i] = r;
      m = max(m, r);
    }
    const bool odd = m >= 0x7F800000u;
    if (odd) {
      record_status(a.status, FQT_ENONFINITE);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t r = 0u;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const uint32_t x = v[k][i][j] & 0x7FFFFFFFu;
          if (x < 0x7F800000u) r = max(r, x);
          else v[k][i][j] = 0x7FFFFFFFu;
        }
        if (k < 2) rm[k][i] = r;
      }
    }
    if (a.qt[k].codes) {
      uint32_t cm[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        uint32_t c = 0u;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t x = v[k][i][j] & 0x7FFFFFFFu;
          c = max(c, odd && x >= 0x7F800000u ? 0u : x);
        }
        cm[j] = max(c, __shfl_xor_sync(0xffffffffu, c, 16));
      }
      if (lane < 16) {
        uint4 *to = reinterpret_cast<uint4 *>(&s.top[k][warp][cg * 8]);
        to[0] = make_uint4(cm[0], cm[1], cm[2], cm[3]);
        to[1] = make_uint4(cm[4], cm[5], cm[6], cm[7]);
      }
    }
  }
  // by rows
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    if (!a.q[k].codes) continue;
#pragma unroll
    for (int o = 8; o > 0; o >>= 1)
#pragma unroll
      for (int i = 0; i < 4; ++i) rm[k][i] = max(rm[k][i], __shfl_xor_sync(0xffffffffu, rm[k][i], o));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int e = f8_exponent(rm[k][i]);
      if (row + i >= a.rows) break;
      if (cg == 0) a.q[k].scales[scale_at(blockIdx.y, a.sp, row + i)] = (uint8_t)(e + 127);
      if (col >= a.cols) continue;
      const float inv = pow2(-e);
      *reinterpret_cast<uint2 *>(a.q[k].codes + (row + i) * a.q[k].pitch + col) =
          make_uint2(f8_codes4<false>(&v[k][i][0], inv), f8_codes4<false>(&v[k][i][4], inv));
    }
  }
  if (!a.qt[0].codes && !a.qt[1].codes && !a.qt[2].codes) return;
  __syncthreads();
  if (t < 3 * kF8Block && a.qt[t / kF8Block].codes) {
    const int k = t / kF8Block, j = t % kF8Block;
    uint32_t m = 0u;
#pragma unroll
    for (int w = 0; w < kF8BackWarps; ++w) m = max(m, s.top[k][w][j]);
    const int e = f8_exponent(m);
    s.inv[k][j] = pow2(-e);
    if (c0 + j < a.cols)
      a.qt[k].scales[scale_at(blockIdx.x, a.spt, c0 + j)] = (uint8_t)(e + 127);
  }
  __syncthreads();
  // a column's 32 words of 4 rows, word w at place w ^ 2 (column / 8)
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    if (!a.qt[k].codes) continue;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float inv = s.inv[k][cg * 8 + j];
      const uint32_t c[4] = {v[k][0][j], v[k][1][j], v[k][2][j], v[k][3][j]};
      s.tr[k][(cg * 8 + j) * 32 + (rg ^ (2 * cg))] = f8_codes4<false>(c, inv);
    }
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    if (!a.qt[k].codes) continue;
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const int at = n * kF8BackThreads + t, j = at >> 3, ch = at & 7;
      if (c0 + j >= a.cols || r0 + ch * 16 >= a.rows) continue;
      const uint2 *pairs = reinterpret_cast<const uint2 *>(s.tr[k] + j * 32);
      const uint2 lo = pairs[(2 * ch) ^ (j >> 3)], hi = pairs[(2 * ch + 1) ^ (j >> 3)];
      *reinterpret_cast<uint4 *>(a.qt[k].codes + (c0 + j) * a.qt[k].pitch + r0 + ch * 16) =
          make_uint4(lo.x, lo.y, hi.x, hi.y);
    }
  }
}

template <typename T, int ACT>
static fqt_status launch_gated_back(const F8GatedBackArgs &a, cudaStream_t st) {
  auto kernel = k_f8_gated_back<T, ACT>;
  static DeviceOnce once;
  const cudaError_t e = allow_smem(kernel, sizeof(F8BackShared), once);
  if (e != cudaSuccess) return cuda_fail(e, "gated backward attribute");
  const dim3 grid((unsigned)((a.rows + kF8Block - 1) / kF8Block),
                  (unsigned)((a.cols + kF8Block - 1) / kF8Block));
  const bool vec = f8_aligned(a.da, 16) && a.ldda * (int64_t)sizeof(T) % 16 == 0;
  return cuda_fail(launch_behind(kernel, grid, kF8BackThreads, sizeof(F8BackShared), st, a, vec),
                   "gated backward launch");
}

template <typename T>
static fqt_status launch_gated_back(const F8GatedBackArgs &a, fqt_act act, cudaStream_t st) {
  switch (act) {
    case FQT_SILU: return launch_gated_back<T, FQT_SILU>(a, st);
    case FQT_GELU: return launch_gated_back<T, FQT_GELU>(a, st);
    case FQT_GELU_TANH: return launch_gated_back<T, FQT_GELU_TANH>(a, st);
    case FQT_RELU: return launch_gated_back<T, FQT_RELU>(a, st);
    default: return launch_gated_back<T, FQT_SIGMOID>(a, st);
  }
}

}  // namespace fqt

using namespace fqt;

static bool act_known(fqt_act act) { return act >= FQT_SILU && act <= FQT_SIGMOID; }

// An output of rows x cols codes: its pointers and its pitch; then its sizes.
static bool codes_fit(const fqt_fp8 *q, int64_t rows, int64_t cols) {
  if (!q) return true;
  fqt_fp8 v = *q;
  v.rows = rows;
  v.cols = cols;
  return f8_good(&v);
}
static void set_codes(fqt_fp8 *q, int64_t rows, int64_t cols) {
  if (!q) return;
  q->rows = rows;
  q->cols = cols;
  q->block_rows = 1;
}

// No two outputs in the same place.
template <int N>
static bool all_apart(const fqt_fp8 *const (&q)[N]) {
  for (int i = 0; i < N; ++i)
    for (int j = i + 1; j < N; ++j)
      if (q[i] && q[j] && (q[i]->codes == q[j]->codes || q[i]->scales == q[j]->scales)) return false;
  return true;
}

extern "C" {

size_t fqt_fp8_gated_matmul_workspace_size(int64_t M, int64_t N, int64_t K) {
  (void)M, (void)N, (void)K;
  return kHeaderBytes;  // the status word
}

fqt_status fqt_fp8_gated_matmul(const fqt_fp8 *A, const fqt_fp8 *Bg, const fqt_fp8 *Bu,
                                fqt_act act, fqt_dtype dtype, void *out, int64_t ldo, fqt_fp8 *q,
                                fqt_fp8 *gate, fqt_fp8 *up, void *workspace, size_t ws_bytes,
                                void *stream) {
  if (!A || !Bg || !Bu || (dtype != FQT_F32 && dtype != FQT_BF16) || !act_known(act))
    return FQT_EINVAL;
  for (const fqt_fp8 *x : {A, Bg, Bu})
    if (x->rows < 0 || x->cols < 0 || x->rows > kF8MaxSize || x->cols > kF8MaxSize ||
        (x->block_rows != 1 && x->block_rows != kF8Block))
      return FQT_EINVAL;
  const int64_t M = A->rows, N = Bg->rows, K = A->cols;
  if (Bg->cols != K || Bu->cols != K || Bu->rows != N) return FQT_EINVAL;
  const size_t es = dtype == FQT_BF16 ? 2 : 4;
  if (M > 0 && N > 0) {  // (an empty tensor's address may be NULL)
    if (!out && !q && !gate && !up) return FQT_EINVAL;
    if (out && (!f8_aligned(out, es) || (M > 1 && (ldo < N || ldo > ((int64_t)1 << 40)))))
      return FQT_EINVAL;
    if (!codes_fit(q, M, N) || !codes_fit(gate, M, N) || !codes_fit(up, M, N)) return FQT_EINVAL;
    if (!all_apart({q, gate, up})) return FQT_EINVAL;
    if (K > 0 && (!f8_good(A) || !f8_good(Bg) || !f8_good(Bu))) return FQT_EINVAL;
    if (!workspace || !f8_aligned(workspace, 256) ||
        ws_bytes < fqt_fp8_gated_matmul_workspace_size(M, N, K))
      return FQT_EWORKSPACE;
  }
  for (fqt_fp8 *x : {q, gate, up}) set_codes(x, M, N);
  if (M == 0 || N == 0) return FQT_OK;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  if (K == 0) {  // empty sums: act(0) 0, and codes of zeros with scale 1
    cudaError_t e = cudaSuccess;
    if (out) e = cudaMemset2DAsync(out, (M > 1 ? ldo : N) * es, 0, N * es, M, st);
    for (const fqt_fp8 *x : {q, gate, up}) {
      if (!x || e != cudaSuccess) continue;
      e = cudaMemset2DAsync(x->codes, x->pitch, 0, N, M, st);
      if (e == cudaSuccess)
        e = cudaMemsetAsync(x->scales, 127, (size_t)((N + 511) / 512 * scale_rows(M) * 4), st);
    }
    return cuda_fail(e, "gated product clear");
  }
  return fp8_gated_matmul(A, Bg, Bu, act, dtype == FQT_BF16, out, ldo, q, gate, up, workspace, st);
}

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
  F8GatedBackArgs a = {};
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
  return dtype == FQT_BF16 ? launch_gated_back<__nv_bfloat16>(a, act, st)
                           : launch_gated_back<float>(a, act, st);
}

}  // extern "C"
