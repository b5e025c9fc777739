// Gated MLP of a transformer block, Y = (act(X Wg^T + bg) * (X Wu^T + bu)) Wd^T + bd, forward and backward: the
// MLP of encoders whose blocks are gated (epd_encode takes it as an activation), and of the stages behind
// V_m = E(I_m) (paper section 3.1, Eq. 1 and 2).
//
// Forward, many tokens: two products of the bf16 GEMM family.  The first makes gate and up columns of the same channels in
// one tile and multiplies them where the accumulators stand (EPI_GATED), so that G and U never meet memory unless a backward
// pass wants them.  Forward, few tokens: see few_tokens_kernel.
// Backward, from dY and the saved G, U:
//   dH = dY Wd;  dU = dH act(G), dG = dH U act'(G), H = act(G) U   in the epilogue of the first product (EPI_DGATED)
//   dX = dG Wg + dU Wu;  dWgu = (dG | dU)^T X;  dWd = dY^T H;  biases: column sums of dG | dU and dY
// Every product is A W^T with K contiguous in both operands; the operands whose rows run along the other axis are turned by
// a transpose kernel first.  Rounded to bf16 on the way, beside the outputs: H, dG and dU, each once, as operands of
// matrix instructions; G and U are kept in fp32, sums are fp32 throughout.
#include "gemm_bf16_tile.h"
#include "op_error.h"

#include <climits>

namespace epd {

// ------------------------------------------------------------------------------ few tokens
// out[t][n] = sum_k X[t][k] W[n][k] (+ bias), t < 16 NB; GATED: W's rows n and N + n are the gate and up rows of channel n, and
// out = act(gate) * up.  Bound: HBM, every weight is read once; so nothing is staged: a lane's 16 bytes of a row of W
// are its operand of the matrix instruction as they come.  A block makes 16 rows of W for all tokens, its waves take K in
// turn, 64 at a time (whole 128-byte lines of the rows), U turns of loads at once, and their sums meet in LDS in the order of
// the waves.
struct FewArgs {
  const void* X; const void* W; const void* bias;
  void* out; void* gu;                 // gu: see GemmArgs (nullptr: not kept)
  int ldx, ldo, ldgu, T, N, K, act;
};

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_few;

template <int NB, int NW, int U, bool GATED>
__global__ __launch_bounds__(64 * NW) void few_tokens_kernel(FewArgs a) {
  constexpr int S = GATED ? 2 : 1;
  __shared__ __attribute__((aligned(16))) float sums[NW][S * NB][16][16];       // [wave][..][token][row]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, g4 = lane >> 4;
  const int n0 = blockIdx.x * 16;
  const uint16_t* const w0 = (const uint16_t*)a.W + (size_t)min(n0 + l16, a.N - 1) * a.K;
  const uint16_t* const wrow[2] = {w0, w0 + (GATED ? (size_t)a.N * a.K : 0)};
  const uint16_t* xrow[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) xrow[b] = (const uint16_t*)a.X + (size_t)min(b * 16 + l16, a.T - 1) * a.ldx;   // rows beyond T repeat the last one: never stored
  f32x4 acc[S][NB];
#pragma unroll
  for (int s = 0; s < S; ++s)
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[s][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto load = [&](const uint16_t* row, int k) {            // 8 values, zeros from K on (K is a multiple of 8)
    bf16x8 v = {};
    if (k < a.K) v = *(const bf16x8*)(row + k);
    return v;
  };
  auto stream = [&](const uint16_t* row, int k) {          // weights: read once
    u32x4_few v = {};
    if (k < a.K) v = __builtin_nontemporal_load((const u32x4_few*)(row + k));
    return __builtin_bit_cast(bf16x8, v);
  };
  for (int k0 = wave * 64; k0 < a.K; k0 += NW * 64 * U) {
    bf16x8 w[U][S][2], x[U][NB][2];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      // the k of an instruction is arbitrary as long as both operands agree: a lane takes 16 consecutive ones
      const int k = k0 + u * NW * 64 + g4 * 16;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int s = 0; s < S; ++s) w[u][s][h] = stream(wrow[s], k + h * 8);
#pragma unroll
        for (int b = 0; b < NB; ++b) x[u][b][h] = load(xrow[b], k + h * 8);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
          for (int b = 0; b < NB; ++b) acc[s][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[u][s][h], x[u][b][h], acc[s][b], 0, 0, 0);
  }
#pragma unroll
  for (int s = 0; s < S; ++s)
#pragma unroll
    for (int b = 0; b < NB; ++b) *(f32x4*)&sums[wave][s * NB + b][l16][g4 * 4] = acc[s][b];
  __syncthreads();
  for (int e = tid; e < NB * 64; e += 64 * NW) {           // four rows of W for a token
    const int b = e >> 6, t = (e >> 2) & 15, r = (e & 3) * 4, m = b * 16 + t, n = n0 + r;
    if (m >= a.T || n >= a.N) continue;                    // N is a multiple of 8
    f32x4 v[S];
#pragma unroll
    for (int s = 0; s < S; ++s) {
      v[s] = *(const f32x4*)&sums[0][s * NB + b][t][r];
#pragma unroll
      for (int i = 1; i < NW; ++i) v[s] += *(const f32x4*)&sums[i][s * NB + b][t][r];
      if (a.bias) {
        const uint2 bb = *(const uint2*)((const uint16_t*)a.bias + s * a.N + n);
        v[s][0] += bf16_bits_to_float(bb.x & 0xffff); v[s][1] += bf16_bits_to_float(bb.x >> 16);
        v[s][2] += bf16_bits_to_float(bb.y & 0xffff); v[s][3] += bf16_bits_to_float(bb.y >> 16);
      }
    }
    f32x4 o = v[0];
    if constexpr (GATED) {
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] = (a.act == 0 ? gate_act<0>(v[0][j]) : a.act == 1 ? gate_act<1>(v[0][j]) : gate_act<2>(v[0][j])) * v[S - 1][j];
      if (a.gu) {
        float* const gu = (float*)a.gu + (size_t)m * a.ldgu + n;
        *(f32x4*)gu = v[0];
        *(f32x4*)(gu + a.N) = v[S - 1];
      }
    }
    *(uint2*)((uint16_t*)a.out + (size_t)m * a.ldo + n) = pack_bf16x4(o[0], o[1], o[2], o[3]);
  }
}

constexpr int kFewTokens = 64;

template <int NW, int U, bool GATED> static hipError_t launch_few(const FewArgs& a, hipStream_t s) {
  void* args[] = {(void*)&a};
  const void* f = a.T <= 16 ? (const void*)few_tokens_kernel<1, NW, U, GATED> : a.T <= 32 ? (const void*)few_tokens_kernel<2, NW, U, GATED> : (const void*)few_tokens_kernel<4, NW, U / 2, GATED>;
  return hipLaunchKernel(f, dim3((a.N + 15) / 16), dim3(64 * NW), args, 0, s);
}

// ------------------------------------------------------------------------------ transpose, column sums
// out[c][r] = in[r][c], r < R, c < C; zeros for R <= r < ldo.  Tiles of 64 x 64 through LDS; bf16: 16 bytes per access on
// both sides (C, ldi, ldo multiples of 8).  Bound: HBM.
template <typename E> struct TransposeArgs { const E* in; E* out; int R, C, ldi, ldo; };

__global__ __launch_bounds__(256) void transpose_bf16_kernel(TransposeArgs<uint16_t> a) {
  __shared__ uint16_t tile[64][66];
  const int tid = threadIdx.x, r0 = blockIdx.x * 64, c0 = blockIdx.y * 64;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = i * 32 + (tid >> 3), c = (tid & 7) * 8;
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (r0 + r < a.R && c0 + c < a.C) v = *(const uint4*)(a.in + (size_t)(r0 + r) * a.ldi + c0 + c);
    uint32_t* const d = (uint32_t*)&tile[r][c];
    d[0] = v.x; d[1] = v.y; d[2] = v.z; d[3] = v.w;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int c = i * 32 + (tid >> 3), r = (tid & 7) * 8;
    if (c0 + c >= a.C || r0 + r >= a.ldo) continue;
    uint32_t v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = (uint32_t)tile[r + 2 * j][c] | (uint32_t)tile[r + 2 * j + 1][c] << 16;
    *(uint4*)(a.out + (size_t)(c0 + c) * a.ldo + r0 + r) = make_uint4(v[0], v[1], v[2], v[3]);
  }
}

__global__ __launch_bounds__(256) void transpose_f32_kernel(TransposeArgs<float> a) {
  __shared__ float tile[64][65];
  const int tid = threadIdx.x, r0 = blockIdx.x * 64, c0 = blockIdx.y * 64;
  for (int i = tid; i < 64 * 64; i += 256) {
    const int r = i >> 6, c = i & 63;
    tile[r][c] = r0 + r < a.R && c0 + c < a.C ? a.in[(size_t)(r0 + r) * a.ldi + c0 + c] : 0.f;
  }
  __syncthreads();
  for (int i = tid; i < 64 * 64; i += 256) {
    const int c = i >> 6, r = i & 63;
    if (c0 + c < a.C && r0 + r < a.ldo) a.out[(size_t)(c0 + c) * a.ldo + r0 + r] = tile[r][c];
  }
}

static hipError_t transpose(bool bf16, const void* in, int ldi, void* out, int ldo, int R, int C, hipStream_t s) {
  const dim3 grid((ldo + 63) / 64, (C + 63) / 64);
  if (bf16) {
    TransposeArgs<uint16_t> a{(const uint16_t*)in, (uint16_t*)out, R, C, ldi, ldo};
    void* args[] = {(void*)&a};
    return hipLaunchKernel((const void*)transpose_bf16_kernel, grid, dim3(256), args, 0, s);
  }
  TransposeArgs<float> a{(const float*)in, (float*)out, R, C, ldi, ldo};
  void* args[] = {(void*)&a};
  return hipLaunchKernel((const void*)transpose_f32_kernel, grid, dim3(256), args, 0, s);
}

// out[r] = sum of in[r][0 .. n): the gradient of a bias, from rows that were turned.  A wave per row, fp32.
template <typename E> __global__ __launch_bounds__(256) void row_sum_kernel(const E* in, E* out, int R, int n, int ld) {
  const int r = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (r >= R) return;
  float sum = 0.f;
  for (int k = lane; k < n; k += 64) sum += (float)in[(size_t)r * ld + k];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
  if (lane == 0) out[r] = (E)sum;
}

static hipError_t row_sums(bool bf16, const void* in, void* out, int R, int n, int ld, hipStream_t s) {
  void* args[] = {(void*)&in, (void*)&out, (void*)&R, (void*)&n, (void*)&ld};
  return hipLaunchKernel(bf16 ? (const void*)row_sum_kernel<__bf16> : (const void*)row_sum_kernel<float>, dim3((R + 3) / 4), dim3(256), args, 0, s);
}

// Columns [c0, c1) of rows of `ld` 16-bit values cleared (c0, c1 multiples of 8).
__global__ __launch_bounds__(256) void clear_columns_kernel(uint16_t* p, int R, int c0, int c1, int ld) {
  const int per = (c1 - c0) / 8, i = blockIdx.x * 256 + threadIdx.x, r = i / per, c = i - r * per;
  if (r < R) *(uint4*)(p + (size_t)r * ld + c0 + c * 8) = make_uint4(0u, 0u, 0u, 0u);
}

// All of a dense array cleared.
template <typename E> __global__ __launch_bounds__(256) void clear_kernel(E* p, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) p[i] = (E)0.f;
}

static hipError_t clear(bool bf16, void* p, int64_t n, hipStream_t s) {
  void* args[] = {(void*)&p, (void*)&n};
  return hipLaunchKernel(bf16 ? (const void*)clear_kernel<__bf16> : (const void*)clear_kernel<float>, dim3((int)std::min<int64_t>((n + 255) / 256, 4096)), dim3(256), args, 0, s);
}

// ------------------------------------------------------------------------------ products
template <int EPI> static void launch_gated_epi(const GemmArgs& g, hipStream_t s) { launch_epi<EPI, OUT_BF16, false, true>(g, s); }

static void launch_gated_whole(const GemmArgs& g, hipStream_t s) {
  if (g.epilogue == EPI_GATED) launch_gated_epi<EPI_GATED>(g, s);
  else if (g.epilogue == EPI_DGATED) launch_gated_epi<EPI_DGATED>(g, s);
  else launch_gated_epi<EPI_STORE>(g, s);
}

// EPI_STORE, EPI_GATED or EPI_DGATED with operands that are not read past their ends; cut as the encoder's are.
void launch_gemm_bf16_gated(const GemmArgs& g, hipStream_t s) {
  if (g.M <= 0 || g.N <= 0) return;
  const TilePlan plan = g.tile_cfg == 0 ? plan_tiles(g.M, g.N, g.K, g.epilogue, true, g.compute_units > 0 ? g.compute_units : num_cus()) : TilePlan{0, 0, 0.0, 0};
  if (plan.body_rows <= 0) { launch_gated_whole(g, s); return; }
  const size_t mb = plan.body_rows;
  GemmArgs body = g, tail = g;
  body.M = (int)mb; body.tile_cfg = plan.tile + 1;
  tail.M = g.M - (int)mb; tail.tile_cfg = plan.tail_tile + 1;
  tail.A = (const __bf16*)g.A + mb * g.lda;
  if (g.out) tail.out = (__bf16*)g.out + mb * g.ldo;
  if (g.gu) tail.gu = (float*)g.gu + mb * g.ldgu;
  if (g.dgu) tail.dgu = (__bf16*)g.dgu + mb * g.lddgu;
  if (g.stats_in) tail.stats_in = g.stats_in + mb * g.stats_n;
  launch_gated_whole(body, s);
  launch_gated_whole(tail, s);
}

}  // namespace epd

using namespace epd;

namespace {

// ------------------------------------------------------------------ workspace layout (bytes)
struct GatedLayout {
  int es, Tp, P2, Dp;                   // element size; tokens, 2 F and D padded to whole K steps (bf16)
  size_t h, wd_t, wgu_t, dgu, dgu_t, h_t, x_t, dy_t, total;
};

GatedLayout gated_layout(const epd_gated_mlp_cfg& c) {
  GatedLayout L;
  const bool bf = c.dtype == EPD_BF16;
  auto up = [](size_t v, size_t a) { return (v + a - 1) / a * a; };
  const size_t D = c.hidden, F = c.mlp_dim, T = c.max_tokens;
  L.es = bf ? 2 : 4;
  L.Tp = (int)(bf ? up(T, 64) : T); L.P2 = (int)(bf ? up(2 * F, 64) : 2 * F); L.Dp = (int)(bf ? up(D, 8) : D);
  size_t off = 0;
  auto take = [&](size_t elements) { const size_t o = off; off = up(off + elements * L.es, 256); return o; };
  L.h = take(T * F);
  L.wd_t = L.wgu_t = L.dgu = L.dgu_t = L.h_t = L.x_t = L.dy_t = 0;
  if (c.training) {
    L.wd_t = take(F * L.Dp);
    L.wgu_t = take(D * L.P2);
    L.dgu = take(T * L.P2);
    L.dgu_t = take(2 * F * L.Tp);
    L.h_t = take(F * L.Tp);
    L.x_t = take(D * L.Tp);
    L.dy_t = take(D * L.Tp);
  }
  L.total = off;
  return L;
}

constexpr int kMaxTokens = 1 << 22;      // and leading dimensions: 320 rows stay below 2^32 bytes

epd_status check_cfg(const char* who, const epd_gated_mlp_cfg* c) {
  if (!c) return op_fail(EPD_ERR_INVALID_ARG, "%s: cfg is NULL", who);
  if (c->struct_size != sizeof(epd_gated_mlp_cfg)) return op_fail(EPD_ERR_INVALID_ARG, "%s: cfg.struct_size %u != %zu", who, c->struct_size, sizeof(epd_gated_mlp_cfg));
  if ((c->dtype != EPD_F32 && c->dtype != EPD_BF16) || (c->use_bias != 0 && c->use_bias != 1) || (c->training != 0 && c->training != 1))
    return op_fail(EPD_ERR_INVALID_ARG, "%s: dtype, use_bias or training invalid", who);
  if (c->act != EPD_SWIGLU && c->act != EPD_GEGLU_ERF && c->act != EPD_GEGLU_TANH) return op_fail(EPD_ERR_INVALID_ARG, "%s: act %d is not a gated activation", who, c->act);
  if (c->hidden <= 0 || c->mlp_dim <= 0 || c->max_tokens <= 0) return op_fail(EPD_ERR_INVALID_ARG, "%s: a size is not positive", who);
  if (c->dtype == EPD_BF16 && (c->hidden % 8 || c->mlp_dim % 8)) return op_fail(EPD_ERR_UNSUPPORTED, "%s: bf16: hidden and mlp_dim must be multiples of 8", who);
  if (c->hidden > 65536 || c->mlp_dim > 131072 || (int64_t)c->hidden * c->mlp_dim >= (1ll << 30))
    return op_fail(EPD_ERR_UNSUPPORTED, "%s: hidden %d, mlp_dim %d: at most 65536, 131072 and 2^30 together", who, c->hidden, c->mlp_dim);
  if (c->max_tokens >= kMaxTokens || (int64_t)c->max_tokens * c->mlp_dim >= (1ll << 36) || (int64_t)c->max_tokens * c->hidden >= (1ll << 36))
    return op_fail(EPD_ERR_UNSUPPORTED, "%s: max_tokens %d too large", who, c->max_tokens);
  return EPD_OK;
}

epd_status check_rows(const char* who, const char* name, const epd_gated_mlp_cfg& c, const void* p, int64_t ld) {
  if (!p) return op_fail(EPD_ERR_INVALID_ARG, "%s: %s is NULL", who, name);
  if (ld < c.hidden || ld >= kMaxTokens) return op_fail(EPD_ERR_SHAPE, "%s: rows of %s are %lld apart: hidden %d .. 2^22 - 1", who, name, (long long)ld, c.hidden);
  if (c.dtype == EPD_BF16 ? ((uintptr_t)p % 16 || ld % 8) : (uintptr_t)p % 4)
    return op_fail(EPD_ERR_UNSUPPORTED, "%s: rows of %s must start on 16 bytes (bf16) or 4 (fp32)", who, name);
  return EPD_OK;
}

epd_status check_call(const char* who, const epd_gated_mlp_cfg* c, const epd_gated_mlp_weights* w, int32_t tokens, const void* workspace, uint64_t bytes) {
  if (epd_status s = check_cfg(who, c)) return s;
  if (tokens < 0 || tokens > c->max_tokens) return op_fail(EPD_ERR_SHAPE, "%s: tokens %d: 0 .. max_tokens %d", who, tokens, c->max_tokens);
  if (!w || !w->gate_up_w || !w->down_w || (c->use_bias && (!w->gate_up_b || !w->down_b))) return op_fail(EPD_ERR_INVALID_ARG, "%s: a required weight pointer is NULL", who);
  const uintptr_t all = (uintptr_t)w->gate_up_w | (uintptr_t)w->down_w | (c->use_bias ? (uintptr_t)w->gate_up_b | (uintptr_t)w->down_b : 0);
  if (all % (c->dtype == EPD_BF16 ? 16 : 4)) return op_fail(EPD_ERR_UNSUPPORTED, "%s: weights must be aligned to 16 bytes (bf16) or 4 (fp32)", who);
  if (!workspace || (uintptr_t)workspace % 256) return op_fail(EPD_ERR_WORKSPACE, "%s: workspace is NULL or not 256-byte aligned", who);
  const size_t need = gated_layout(*c).total;
  if (bytes < need) return op_fail(EPD_ERR_WORKSPACE, "%s: workspace_bytes %llu < required %zu", who, (unsigned long long)bytes, need);
  return EPD_OK;
}

int act_code(const epd_gated_mlp_cfg& c) { return c.act == EPD_SWIGLU ? 2 : c.act == EPD_GEGLU_TANH ? 1 : 0; }

// Launches of the GEMM families report through the runtime's last error, which may hold one that the program left
// there: only a new one counts, and the program's stays.
struct LastError {
  const hipError_t before = hipPeekAtLastError();
  hipError_t now() const {
    const hipError_t e = hipPeekAtLastError();
    if (e == before) return hipSuccess;
    (void)hipGetLastError();
    return e;
  }
};

void gemm(const epd_gated_mlp_cfg& c, GemmArgs& g, hipStream_t s) {
  if (c.dtype == EPD_BF16) launch_gemm_bf16_gated(g, s);
  else launch_gemm_f32(g, s);
}

}  // namespace

extern "C" {

uint64_t epd_gated_mlp_workspace_bytes(const epd_gated_mlp_cfg* cfg) {
  if (check_cfg("epd_gated_mlp_workspace_bytes", cfg) != EPD_OK) return 0;
  return gated_layout(*cfg).total;
}

epd_status epd_gated_mlp(const epd_gated_mlp_cfg* cfg, const epd_gated_mlp_weights* w, const void* x, int64_t ld_x, int32_t tokens, void* y, int64_t ld_y,
                         void* saved, void* workspace, uint64_t workspace_bytes, void* stream) {
  const char* const who = "epd_gated_mlp";
  if (epd_status s = check_call(who, cfg, w, tokens, workspace, workspace_bytes)) return s;
  if (tokens == 0) return EPD_OK;
  const epd_gated_mlp_cfg& c = *cfg;
  if (epd_status s = check_rows(who, "x", c, x, ld_x)) return s;
  if (epd_status s = check_rows(who, "y", c, y, ld_y)) return s;
  if ((uintptr_t)saved % (c.dtype == EPD_BF16 ? 16 : 4)) return op_fail(EPD_ERR_UNSUPPORTED, "%s: saved must be aligned to 16 bytes (bf16) or 4 (fp32)", who);
  const GatedLayout L = gated_layout(c);
  const bool bf = c.dtype == EPD_BF16;
  const int D = c.hidden, F = c.mlp_dim, T = tokens;
  void* const H = (char*)workspace + L.h;
  hipStream_t st = (hipStream_t)stream;
  if (bf && T <= kFewTokens) {
    FewArgs a{x, w->gate_up_w, c.use_bias ? w->gate_up_b : nullptr, H, saved, (int)ld_x, F, 2 * F, T, F, D, act_code(c)};
    hipError_t e = launch_few<4, 4, true>(a, st);
    FewArgs b{H, w->down_w, c.use_bias ? w->down_b : nullptr, y, nullptr, F, (int)ld_y, 0, T, D, F, 0};
    if (e == hipSuccess) e = launch_few<8, 4, false>(b, st);
    if (e != hipSuccess) return op_fail(EPD_ERR_HIP, "%s: kernel launch failed: %s", who, hipGetErrorString(e));
    return EPD_OK;
  }
  const LastError last;
  {
    GemmArgs g{};
    g.A = x; g.lda = (int)ld_x; g.W = w->gate_up_w; g.bias = c.use_bias ? w->gate_up_b : nullptr;
    g.M = T; g.N = bf ? (F + 15) / 16 * 32 : 2 * F; g.K = D; g.epilogue = EPI_GATED; g.act = act_code(c);
    g.gate_rows = F; g.out = H; g.ldo = F; g.gu = saved; g.ldgu = 2 * F;
    gemm(c, g, st);
  }
  {
    GemmArgs g{};
    g.A = H; g.lda = F; g.W = w->down_w; g.bias = c.use_bias ? w->down_b : nullptr;
    g.M = T; g.N = D; g.K = F; g.epilogue = EPI_STORE; g.out = y; g.ldo = (int)ld_y;
    gemm(c, g, st);
  }
  if (hipError_t e = last.now()) return op_fail(EPD_ERR_HIP, "%s: kernel launch failed: %s", who, hipGetErrorString(e));
  return EPD_OK;
}

epd_status epd_gated_mlp_backward(const epd_gated_mlp_cfg* cfg, const epd_gated_mlp_weights* w, const void* x, int64_t ld_x, const void* dy, int64_t ld_dy,
                                  int32_t tokens, const void* saved, const epd_gated_mlp_grads* grads, void* workspace, uint64_t workspace_bytes, void* stream) {
  const char* const who = "epd_gated_mlp_backward";
  if (epd_status s = check_call(who, cfg, w, tokens, workspace, workspace_bytes)) return s;
  const epd_gated_mlp_cfg& c = *cfg;
  if (!c.training) return op_fail(EPD_ERR_INVALID_ARG, "%s: cfg.training is 0", who);
  if (!grads) return op_fail(EPD_ERR_INVALID_ARG, "%s: grads is NULL", who);
  if (!c.use_bias && (grads->gate_up_b || grads->down_b)) return op_fail(EPD_ERR_INVALID_ARG, "%s: gradients of biases wanted, use_bias is 0", who);
  const bool bf = c.dtype == EPD_BF16;
  const uintptr_t all = (uintptr_t)grads->gate_up_w | (uintptr_t)grads->down_w | (uintptr_t)grads->gate_up_b | (uintptr_t)grads->down_b | (uintptr_t)saved;
  if (all % (bf ? 16 : 4)) return op_fail(EPD_ERR_UNSUPPORTED, "%s: gradients and saved must be aligned to 16 bytes (bf16) or 4 (fp32)", who);
  const int64_t D = c.hidden, F = c.mlp_dim;
  hipStream_t st = (hipStream_t)stream;
  hipError_t e = hipSuccess;
  auto ok = [&](hipError_t r) { if (e == hipSuccess) e = r; return e == hipSuccess; };
  auto failed = [&]() { return op_fail(EPD_ERR_HIP, "%s: kernel launch failed: %s", who, hipGetErrorString(e)); };
  if (tokens == 0) {                     // sums over no token
    if (grads->gate_up_w) ok(clear(bf, grads->gate_up_w, 2 * F * D, st));
    if (grads->down_w && e == hipSuccess) ok(clear(bf, grads->down_w, D * F, st));
    if (grads->gate_up_b && e == hipSuccess) ok(clear(bf, grads->gate_up_b, 2 * F, st));
    if (grads->down_b && e == hipSuccess) ok(clear(bf, grads->down_b, D, st));
    return e == hipSuccess ? EPD_OK : failed();
  }
  if (epd_status s = check_rows(who, "x", c, x, ld_x)) return s;
  if (epd_status s = check_rows(who, "dy", c, dy, ld_dy)) return s;
  if (!saved) return op_fail(EPD_ERR_INVALID_ARG, "%s: saved is NULL", who);
  if (grads->dx) if (epd_status s = check_rows(who, "dx", c, grads->dx, grads->ld_dx)) return s;
  const GatedLayout L = gated_layout(c);
  char* const ws = (char*)workspace;
  const int T = tokens, Tp = bf ? (T + 63) / 64 * 64 : T, P2 = L.P2;
  const bool want_gu = grads->gate_up_w || grads->gate_up_b, want_d = grads->down_w || grads->down_b;
  const LastError last;
  if (grads->dx || want_gu || grads->down_w) {
    // dH = dY Wd, and at once dG, dU and H
    if (!ok(transpose(bf, w->down_w, (int)F, ws + L.wd_t, L.Dp, (int)D, (int)F, st))) return failed();
    GemmArgs g{};
    g.A = dy; g.lda = (int)ld_dy; g.W = ws + L.wd_t; g.ldw = L.Dp;
    g.M = T; g.N = (int)F; g.K = (int)D; g.epilogue = EPI_DGATED; g.act = act_code(c);
    g.gate_rows = (int)F; g.gu = (void*)saved; g.ldgu = (int)(2 * F); g.dgu = ws + L.dgu; g.lddgu = P2; g.out = ws + L.h; g.ldo = (int)F;
    gemm(c, g, st);
  }
  if (grads->dx) {                       // dX = (dG | dU) Wgu
    if (P2 != 2 * F) {
      int r = T, c0 = (int)(2 * F), c1 = P2;
      uint16_t* p = (uint16_t*)(ws + L.dgu);
      void* args[] = {(void*)&p, (void*)&r, (void*)&c0, (void*)&c1, (void*)&c1};
      const int64_t n = (int64_t)T * ((P2 - 2 * F) / 8);
      if (!ok(hipLaunchKernel((const void*)clear_columns_kernel, dim3((int)((n + 255) / 256)), dim3(256), args, 0, st))) return failed();
    }
    if (!ok(transpose(bf, w->gate_up_w, (int)D, ws + L.wgu_t, P2, (int)(2 * F), (int)D, st))) return failed();
    GemmArgs g{};
    g.A = ws + L.dgu; g.lda = P2; g.W = ws + L.wgu_t; g.ldw = P2;
    g.M = T; g.N = (int)D; g.K = P2; g.epilogue = EPI_STORE; g.out = grads->dx; g.ldo = (int)grads->ld_dx;
    gemm(c, g, st);
  }
  if (want_gu) {                         // dWgu = (dG | dU)^T X
    if (!ok(transpose(bf, ws + L.dgu, P2, ws + L.dgu_t, Tp, T, (int)(2 * F), st))) return failed();
    if (grads->gate_up_b && !ok(row_sums(bf, ws + L.dgu_t, grads->gate_up_b, (int)(2 * F), T, Tp, st))) return failed();
    if (grads->gate_up_w) {
      if (!ok(transpose(bf, x, (int)ld_x, ws + L.x_t, Tp, T, (int)D, st))) return failed();
      GemmArgs g{};
      g.A = ws + L.dgu_t; g.lda = Tp; g.W = ws + L.x_t; g.ldw = Tp;
      g.M = (int)(2 * F); g.N = (int)D; g.K = Tp; g.epilogue = EPI_STORE; g.out = grads->gate_up_w; g.ldo = (int)D;
      gemm(c, g, st);
    }
  }
  if (want_d) {                          // dWd = dY^T H
    if (!ok(transpose(bf, dy, (int)ld_dy, ws + L.dy_t, Tp, T, (int)D, st))) return failed();
    if (grads->down_b && !ok(row_sums(bf, ws + L.dy_t, grads->down_b, (int)D, T, Tp, st))) return failed();
    if (grads->down_w) {
      if (!ok(transpose(bf, ws + L.h, (int)F, ws + L.h_t, Tp, T, (int)F, st))) return failed();
      GemmArgs g{};
      g.A = ws + L.dy_t; g.lda = Tp; g.W = ws + L.h_t; g.ldw = Tp;
      g.M = (int)D; g.N = (int)F; g.K = Tp; g.epilogue = EPI_STORE; g.out = grads->down_w; g.ldo = (int)F;
      gemm(c, g, st);
    }
  }
  ok(last.now());
  return e == hipSuccess ? EPD_OK : failed();
}

}  // extern "C"
