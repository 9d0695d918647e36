// fqt_gated.cu -- both projections of a gated feed-forward block, its activation and its
// product in one kernel:  g = A Bg^T, u = A Bu^T, a = act(g) u
#include "fqt_gated.cuh"

namespace fqt {

// Codes that leave in boxes of 32 rows x 128.
static bool make_map_codes_out(CUtensorMap *m, const fqt_fp8 *q) {
  return make_map_codes(m, q, 32);
}

// CTAs of a cluster that share the K blocks of each of `ctas` CTAs (which themselves come in
// clusters of `holds`), of which the estimate is least: a K block takes ns nanoseconds, meeting
// in shared memory `meet` (which clusters that hold blocks together do anyway), and not all SMs
// have a place in a large cluster.  Few tokens: 0.22 us and 2.3 (1 x 1024 x 4096 7.5 us shared
// by four, 11.3 unshared; 1 x 4096 x 1024 6.2 unshared).  Tiles of 128 tokens: 0.4 and 3.5 (128
// x 1024 x 4096 12.7 shared by eight and 13.7; 300 x 100 x 4000 12.4 and 16.4; 1523 x 336 x 1201
// 8.9 unshared, 11.0 by three).  Sets the K blocks of one, whole groups of scales.
static int share_blocks(int64_t ctas, int holds, int nkb, int ns, int meet, int nsm, int *kb_per) {
  const int groups = (nkb + kF8Group - 1) / kF8Group;
  int best = 1;
  int64_t least = INT64_MAX;
  for (int splits = 1; splits * holds <= kF8Parts && splits <= groups; ++splits) {
    const int per = (groups + splits - 1) / splits * kF8Group, cluster = splits * holds;
    if ((nkb + per - 1) / per != splits) continue;  // as many as another number's
    const int room = cluster > 4 ? nsm * 3 / 4 : cluster > 2 ? nsm * 7 / 8 : nsm;
    if (splits > 1 && ctas * splits > room) break;
    const int64_t rounds = (ctas * splits + nsm - 1) / nsm;
    const int64_t cost = rounds * std::min(per, nkb) * ns + (splits > 1 && holds == 1 ? meet : 0);
    if (cost < least) {
      least = cost;
      best = splits;
      *kb_per = per;
    }
  }
  return best;
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
    g.holds = q || gate || up ? kF8Block / g.part : 1;
    const int64_t run = (int64_t)g.part * g.holds, runs = (N + run - 1) / run;
    const int splits = share_blocks(runs * g.holds, g.holds, g.nkb, 220, 2300, nsm, &g.kb_per);
    g.splits = splits * g.holds;
    g.items = runs * g.splits;
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
  const bool codes = q || gate || up;
  const int64_t n_tiles = (N + kF8Block - 1) / kF8Block;
  const bool pair = nsm >= 2 && (M + 255) / 256 * n_tiles * 8 >= (int64_t)nsm * 3;
  const int rows = pair ? 2 * BM : BM;
  g.m_tiles = (int)((M + rows - 1) / rows);
  g.n_tiles = (int)n_tiles;
  bool narrow = false;
  if (!pair) {
    const int64_t tiles = (int64_t)g.m_tiles * n_tiles, half = g.m_tiles * ((N + 63) / 64);
    g.splits = share_blocks(tiles, 1, g.nkb, 400, 3500, nsm, &g.kb_per);
    // A dense output alone: tiles of half the columns where the estimate is less (a K block 0.27
    // us, the epilogue 0.9 after 1.5): 1523 x 336 x 1201 in bf16 8.9 -> 6.9 us, in fp32 with gelu
    // 11.0 -> 8.2, 128 x 4096 x 1024 in bf16 7.6 -> 6.2.
    auto rounds = [&](int64_t n) { return (n + nsm - 1) / nsm; };
    const int64_t wide = rounds(tiles * g.splits) * std::min(g.kb_per, g.nkb) * 400 +
                         (g.splits > 1 ? 3500 : 1500);
    narrow = !codes && rounds(half) * g.nkb * 270 + 900 < wide;
    if (narrow) {
      g.splits = 1;
      g.kb_per = g.nkb;
      g.n_tiles = (int)((N + 63) / 64);
    }
  }
  g.items = (int64_t)g.m_tiles * g.n_tiles * g.splits;
  g.sa = reinterpret_cast<const uint32_t *>(A->scales);
  g.sb = reinterpret_cast<const uint32_t *>(w->scales);
  g.spa = scale_rows(M);
  g.spb = scale_rows(N);
  g.M = M;
  g.N = N;
  const int es = bf16 ? 2 : 4;
  g.boxes = out && f8_aligned(out, 16) && g.ldo * es % 16 == 0 && N * es % 16 == 0 &&
            g.ldo < ((int64_t)1 << 40) / es;
  if (!make_map_codes(&maps.a, A, BM) || !make_map_codes(&maps.b, Bg, narrow ? 64 : BM) ||
      !make_map_codes(&maps.b2, Bu, narrow ? 64 : BM) ||
      (g.boxes && !make_map_f8_out(&maps.out, out, bf16, M, N, g.ldo)))
    return cuda_fail(cudaErrorUnknown, "FP8 tensor map");
  if (narrow) return launch_f8<128, 2, false, F8_GATED_DENSE>(maps, g, nsm, st);
  // (where K blocks are shared the join writes every kind of output)
  if (g.splits > 1) return launch_f8<256, 1, false, F8_GATED_DENSE>(maps, g, nsm, st);
  if (codes) {
    if ((q && !make_map_codes_out(&maps.q, q)) || (gate && !make_map_codes_out(&maps.gate, gate)) ||
        (up && !make_map_codes_out(&maps.up, up)))
      return cuda_fail(cudaErrorUnknown, "FP8 tensor map");
    if (out)
      return pair ? launch_f8<256, 1, true, F8_GATED_BOTH>(maps, g, nsm, st)
                  : launch_f8<256, 1, false, F8_GATED_BOTH>(maps, g, nsm, st);
    return pair ? launch_f8<256, 1, true, F8_GATED>(maps, g, nsm, st)
                : launch_f8<256, 1, false, F8_GATED>(maps, g, nsm, st);
  }
  return pair ? launch_f8<256, 1, true, F8_GATED_DENSE>(maps, g, nsm, st)
              : launch_f8<256, 1, false, F8_GATED_DENSE>(maps, g, nsm, st);
}

}  // namespace fqt

using namespace fqt;

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
    F8Apart apart;
    apart.writes(out, M, N, es, ldo);
    for (const fqt_fp8 *x : {q, gate, up}) apart.writes(x, M, N);
    if (K > 0)
      for (const fqt_fp8 *x : {A, Bg, Bu}) {
        if (!f8_good(x)) return FQT_EINVAL;
        apart.reads(x);
      }
    if (!apart.ok()) return FQT_EINVAL;
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

}  // extern "C"
