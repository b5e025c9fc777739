// The bf16 GEMMs of the encoder (ViT forward, paper section 3.1, Eq. 1): which epilogue runs on what, and the cut
// of a launch whose last round of large tiles would be partial.  The kernels are in gemm_bf16_tile.h.
#include "gemm_bf16_tile.h"

namespace epd {

bool gemm_bf16_tile_known(int t) { return t == 0 || t == 2 || t == 4 || t == 5 || t == 7 || t == 8; }

constexpr int kQkvBN = 128;

static void launch_gemm_bf16_whole(const GemmArgs& g, hipStream_t s);

// a forced tile, gathered rows, or Q | K columns that do not end on a 256-column boundary (those
// run the 256 x 128 tile): one launch
static bool may_split_rows(const GemmArgs& g) {
  return g.tile_cfg == 0 && !g.gather && !(g.epilogue == EPI_QKV && g.qk_cols % 256 != 0);
}

void plan_gemm_bf16(const GemmArgs& g, int compute_units, int* tile_rows, int* tile_cols, int* body_rows) {
  const long cus = compute_units > 0 ? compute_units : (g.compute_units > 0 ? g.compute_units : num_cus());
  int t = g.tile_cfg > 0 ? g.tile_cfg - 1 : -1, body = 0;
  if (!gemm_bf16_tile_known(t)) {
    const TilePlan p = plan_tiles(g.M, g.N, g.K, g.epilogue, may_split_rows(g), cus);
    t = p.tile; body = p.body_rows;
  }
  if (g.epilogue == EPI_QKV && (t == 0 || t == 5) && g.qk_cols % 256 != 0) t = 2;
  *tile_rows = t == 7 || t == 8 ? 64 : t == 4 ? 128 : t == 5 ? 320 : 256;
  *tile_cols = t == 7 ? 64 : t == 0 || t == 5 ? 256 : 128;
  *body_rows = body;
}

int gemm_bf16_stat_cols(const GemmArgs& g) {
  int rows, cols, body;
  plan_gemm_bf16(g, 0, &rows, &cols, &body);
  return cols < 128 ? cols : 128;
}

void launch_gemm_bf16(const GemmArgs& g, hipStream_t s) {
  if (g.M <= 0 || g.N <= 0) return;
  const TilePlan plan = may_split_rows(g) ? plan_tiles(g.M, g.N, g.K, g.epilogue, true, g.compute_units > 0 ? g.compute_units : num_cus()) : TilePlan{0, 0, 0.0, 0};
  if (plan.body_rows <= 0) { launch_gemm_bf16_whole(g, s); return; }
  const int mb = plan.body_rows;
  GemmArgs body = g, tail = g;
  body.M = mb; body.tile_cfg = plan.tile + 1;
  tail.M = g.M - mb; tail.tile_cfg = plan.tail_tile + 1;
  // everything indexed by the output row moves down by mb rows (vt is indexed through vcol)
  tail.A = (const __bf16*)g.A + (size_t)mb * g.lda;
  if (g.out) tail.out = g.out_f32 ? (void*)((float*)g.out + (size_t)mb * g.ldo) : (void*)((__bf16*)g.out + (size_t)mb * g.ldo);
  if (g.resid) tail.resid = g.resid + (size_t)mb * g.ldr;
  if (g.xb) tail.xb = (__bf16*)g.xb + (size_t)mb * g.ldxb;
  if (g.stats_out) tail.stats_out = g.stats_out + (size_t)mb * g.stats_n;
  if (g.stats_in) tail.stats_in = g.stats_in + (size_t)mb * g.stats_n;
  if (g.rot) tail.rot = g.rot + (size_t)mb * g.rot_pairs;
  if (g.vcol) tail.vcol = g.vcol + mb;
  launch_gemm_bf16_whole(body, s);
  launch_gemm_bf16_whole(tail, s);
}

static void launch_gemm_bf16_whole(const GemmArgs& g, hipStream_t s) {
  switch (g.epilogue) {
    case EPI_STORE:
      if (g.gather) launch_epi<EPI_STORE, OUT_BF16, true>(g, s);
      else if (g.out_f32) launch_epi<EPI_STORE, OUT_F32, false>(g, s);
      else launch_epi<EPI_STORE, OUT_BF16, false>(g, s);
      break;
    case EPI_GELU:
      launch_epi<EPI_GELU, OUT_BF16, false>(g, s);
      break;
    case EPI_RESIDUAL:
      launch_epi<EPI_RESIDUAL, OUT_F32, false>(g, s);
      break;
    case EPI_QKV:
      if (g.qk_cols % kQkvBN == 0) {
        launch_epi<EPI_QKV, OUT_BF16, false>(g, s);
      } else {
        // a column tile would straddle the K | V boundary: run the two parts separately
        GemmArgs qk = g;
        qk.N = g.qk_cols;
        launch_epi<EPI_QKV, OUT_BF16, false>(qk, s);
        GemmArgs v = g;
        v.W = (const __bf16*)g.W + (size_t)g.qk_cols * (g.ldw ? g.ldw : g.K);
        v.bias = g.bias ? (const void*)((const __bf16*)g.bias + g.qk_cols) : nullptr;
        v.N = g.N - g.qk_cols;
        v.qk_cols = 0;
        launch_epi<EPI_QKV, OUT_BF16, false>(v, s);
      }
      break;
  }
}

}  // namespace epd
