// Product of rows in 8 bits with a scale each, y = (x w^T) * x_scale * scale (+ bias), as an operator: the linear layers of the stage
// behind V_m = E(I_m) (paper section 3.1, Eq. 1 and 2) with weights and activations in 8 bits (epd_quant_rows, epd_add_norm).
//
// The sum over k is exact in int32: K <= 131056 and |x w| <= 2^14 stay below 2^31.  It is the bf16 GEMM's loop on bytes: v_mfma_i32_16x16x64_i8
// takes 16 bytes of K of 16 rows a lane group, as the bf16 instruction does, and multiplies twice as many values in the time, so tiles, rings,
// swizzles and waits are those of gemm_bf16_tile.h with K counted in pairs of values.
#include "gemm_bf16_tile.h"
#include "op_error.h"

#include <climits>

namespace epd {

namespace {

template <class T, int OUT>
__global__ __launch_bounds__(T::NT, T::MINBLK) void int8_gemm_kernel(GemmArgs g) {
  // stages, scales of the rows, scales and bias of the columns
  __shared__ __attribute__((aligned(1024))) char lds[T::LDS_BYTES + T::BM * 4 + T::BN * 8];
  const int tiles_n = (g.N + T::BN - 1) / T::BN, tiles_m = (g.M + T::BM - 1) / T::BM;
  g.zeros = zero_bytes;
  int tm, tn;
  tile_coords(xcd_remap(blockIdx.x, gridDim.x), tiles_m, tiles_n, g.group_m, tm, tn);
  gemm_tile<T, EPI_INT8, OUT, false, false, T::PINGPONG, T::PINGPONG>(g, tm * T::BM, tn * T::BN, lds);
}

template <class T> hipError_t launch_int8(const GemmArgs& g, hipStream_t s) {
  const int tiles_m = (g.M + T::BM - 1) / T::BM, tiles_n = (g.N + T::BN - 1) / T::BN;
  GemmArgs a = g;
  a.group_m = raster_group<T>(g, tiles_m, tiles_n, (long)T::MINBLK * num_cus());
  void* args[] = {(void*)&a};
  return hipLaunchKernel(g.out_f32 ? (const void*)int8_gemm_kernel<T, OUT_F32> : (const void*)int8_gemm_kernel<T, OUT_BF16>, dim3(tiles_m * tiles_n), dim3(T::NT), args, 0, s);
}

constexpr int kMaxIn = 131056, kMaxOut = 1 << 20, kMaxTokens = 1 << 22;

epd_status check_cfg(const char* who, const epd_int8_linear_cfg* c) {
  if (!c) return op_fail(EPD_ERR_INVALID_ARG, "%s: cfg is NULL", who);
  if (c->struct_size != sizeof(epd_int8_linear_cfg)) return op_fail(EPD_ERR_INVALID_ARG, "%s: cfg.struct_size %u != %zu", who, c->struct_size, sizeof(epd_int8_linear_cfg));
  if ((c->out_dtype != EPD_F32 && c->out_dtype != EPD_BF16) || (c->use_bias != 0 && c->use_bias != 1)) return op_fail(EPD_ERR_INVALID_ARG, "%s: out_dtype or use_bias invalid", who);
  if (c->in_features <= 0 || c->out_features <= 0 || c->max_tokens <= 0) return op_fail(EPD_ERR_INVALID_ARG, "%s: a size is not positive", who);
  if (c->in_features % 16 || c->in_features > kMaxIn) return op_fail(EPD_ERR_UNSUPPORTED, "%s: in_features %d: a multiple of 16 up to %d", who, c->in_features, kMaxIn);
  if (c->out_features % 8 || c->out_features > kMaxOut) return op_fail(EPD_ERR_UNSUPPORTED, "%s: out_features %d: a multiple of 8 up to %d", who, c->out_features, kMaxOut);
  if ((int64_t)c->in_features * c->out_features >= (1ll << 32)) return op_fail(EPD_ERR_UNSUPPORTED, "%s: in_features * out_features %lld: below 2^32", who, (long long)c->in_features * c->out_features);
  if (c->max_tokens >= kMaxTokens || (int64_t)c->max_tokens * c->out_features >= (1ll << 36)) return op_fail(EPD_ERR_UNSUPPORTED, "%s: max_tokens %d too large", who, c->max_tokens);
  return EPD_OK;
}

uint64_t workspace_bytes(const epd_int8_linear_cfg&) { return 256; }

}  // namespace
}  // namespace epd

using namespace epd;

extern "C" {

uint64_t epd_int8_linear_workspace_bytes(const epd_int8_linear_cfg* cfg) {
  if (check_cfg("epd_int8_linear_workspace_bytes", cfg) != EPD_OK) return 0;
  return workspace_bytes(*cfg);
}

epd_status epd_int8_linear(const epd_int8_linear_cfg* cfg, const epd_int8_linear_weights* w, const void* x, int64_t ld_x, const float* x_scale, int32_t tokens,
                           void* y, int64_t ld_y, void* workspace, uint64_t bytes, void* stream) {
  const char* const who = "epd_int8_linear";
  if (epd_status s = check_cfg(who, cfg)) return s;
  const epd_int8_linear_cfg& c = *cfg;
  const int K = c.in_features, N = c.out_features;
  if (tokens < 0 || tokens > c.max_tokens) return op_fail(EPD_ERR_SHAPE, "%s: tokens %d: 0 .. max_tokens %d", who, tokens, c.max_tokens);
  if (!w || !w->w || !w->scale || (c.use_bias && !w->bias)) return op_fail(EPD_ERR_INVALID_ARG, "%s: a required weight pointer is NULL", who);
  if (((uintptr_t)w->w | (uintptr_t)w->scale | (c.use_bias ? (uintptr_t)w->bias : 0)) % 16) return op_fail(EPD_ERR_UNSUPPORTED, "%s: weights must be aligned to 16 bytes", who);
  if (!workspace || (uintptr_t)workspace % 256) return op_fail(EPD_ERR_WORKSPACE, "%s: workspace is NULL or not 256-byte aligned", who);
  if (bytes < workspace_bytes(c)) return op_fail(EPD_ERR_WORKSPACE, "%s: workspace_bytes %llu < required %llu", who, (unsigned long long)bytes, (unsigned long long)workspace_bytes(c));
  if (tokens == 0) return EPD_OK;
  if (!x || !x_scale || !y) return op_fail(EPD_ERR_INVALID_ARG, "%s: x, x_scale or y is NULL", who);
  if (tokens == 1) { ld_x = K; ld_y = N; }
  // (rows of a wave's tile stay below 2^31 bytes)
  const int64_t most_y = c.out_dtype == EPD_F32 ? kMaxTokens / 2 : kMaxTokens;
  if (ld_x < K || ld_x >= kMaxTokens || ld_x % 16) return op_fail(EPD_ERR_SHAPE, "%s: rows of x are %lld apart: a multiple of 16, in_features %d .. 2^22", who, (long long)ld_x, K);
  if (ld_y < N || ld_y >= most_y || ld_y % 8) return op_fail(EPD_ERR_SHAPE, "%s: rows of y are %lld apart: a multiple of 8, out_features %d .. %lld", who, (long long)ld_y, N, (long long)most_y);
  if (((uintptr_t)x | (uintptr_t)y) % 16) return op_fail(EPD_ERR_UNSUPPORTED, "%s: x and y must be aligned to 16 bytes", who);
  if ((uintptr_t)x_scale % 4) return op_fail(EPD_ERR_INVALID_ARG, "%s: x_scale is not aligned", who);
  GemmArgs g{};
  g.A = x; g.lda = (int)(ld_x / 2); g.W = w->w; g.ldw = K / 2; g.M = tokens; g.N = N; g.K = K / 2;
  g.epilogue = EPI_INT8; g.out = y; g.ldo = (int)ld_y; g.out_f32 = c.out_dtype == EPD_F32;
  g.row_scales = x_scale; g.col_scales = w->scale; g.col_bias = c.use_bias ? w->bias : nullptr;
  const hipError_t e = launch_int8<T4>(g, (hipStream_t)stream);
  return e == hipSuccess ? EPD_OK : op_launch_failed(who, e);
}

}  // extern "C"
