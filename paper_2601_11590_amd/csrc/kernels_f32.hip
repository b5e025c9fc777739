// fp32 kernels of the Encode-stage library (ViT forward, paper section 3.1, Eq. 1): the
// configuration whose storage type is fp32 must multiply and accumulate in true fp32.  The
// contractions run on the fp32 matrix instruction, v_mfma_f32_16x16x4_f32 (fused fp32 multiply-adds,
// twice the vector rate); everything else is vector arithmetic.
//
// What bounds the small calls this path serves (one 224 x 224 image: 256 tokens, hidden 256) is
// latency and idle compute units, so work is cut fine: 16 x 16 output tiles whose K is split over the
// waves of a block, 16-query attention tiles whose keys are split over the waves.  Operands go from
// memory straight to registers: the k a lane group supplies to an instruction is arbitrary as long
// as both operands agree, so a lane takes four consecutive k of its row (one 16-byte load) and feeds
// them to four instructions.
#include "epd_internal.h"

#include <algorithm>
#include <type_traits>

namespace epd {

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));

// ------------------------------------------------------------------------------ GEMM
__device__ __forceinline__ float gelu_f32(float v, int act) {
  if (act == 0) return 0.5f * v * (1.0f + erff(v * 0.70710678118654752440f));
  float u = 0.79788456080286535588f * (v + 0.044715f * v * v * v);
  return 0.5f * v * (1.0f + tanhf(u));
}

// Gate of a gated MLP: act(g), and its derivative d (see gate_act_d of the bf16 kernels for the formulas).
__device__ __forceinline__ float gate_f32(float g, int act, float& d) {
  if (act == 0) {
    const float cdf = 0.5f * (1.0f + erff(g * 0.70710678118654752440f));
    d = cdf + g * 0.39894228040143267794f * expf(-0.5f * g * g);
    return g * cdf;
  }
  if (act == 1) {
    const float z = fminf(g * g, 1e30f), u = 0.79788456080286535588f * (g + 0.044715f * z * g), t = tanhf(u);
    d = 0.5f * (1.0f + t) + 0.5f * g * (1.0f - t * t) * 0.79788456080286535588f * (1.0f + 3.0f * 0.044715f * z);
    return 0.5f * g * (1.0f + t);
  }
  const float p = 1.0f / (1.0f + expf(-g));
  d = p * (1.0f + g * (1.0f - p));
  return g * p;
}

// The sums of a block in LDS to where they go.
template <int BT, int LD, int COPIES, int NT, bool OPS>
__device__ __forceinline__ void f32_epilogue(const GemmArgs& g, const int m0, const int n0, float (*acc_lds)[BT][LD]) {
  // epilogue: a thread takes 4 consecutive columns (whole rotary pairs) of a row
  const float* bias = (const float*)g.bias;
  float* out = (float*)g.out;
  for (int e = threadIdx.x; e < BT * BT / 4; e += NT) {
    const int r = e / (BT / 4), c = (e - r * (BT / 4)) * 4;
    const int m = m0 + r, n = n0 + c;
    if (m >= g.M || n >= g.N) continue;
    f32x4 v = *(const f32x4*)&acc_lds[0][r][c];
#pragma unroll
    for (int w = 1; w < COPIES; ++w) v += *(const f32x4*)&acc_lds[w][r][c];
    const int left = min(4, g.N - n);
    if (OPS && g.epilogue != EPI_STORE) {
      float* const gu = (float*)g.gu + (size_t)m * g.ldgu;
      if (g.epilogue == EPI_GATED) {
        for (int j = 0; j < left; j += 2) {
          const int ch = (n + j) >> 1;
          const float gate = v[j] + (bias ? bias[ch] : 0.f), up = v[j + 1] + (bias ? bias[g.gate_rows + ch] : 0.f);
          float d;
          out[(size_t)m * g.ldo + ch] = gate_f32(gate, g.act, d) * up;
          if (g.gu) { gu[ch] = gate; gu[g.gate_rows + ch] = up; }
        }
      } else {
        float* const dgu = (float*)g.dgu + (size_t)m * g.lddgu;
        for (int j = 0; j < left; ++j) {
          float d;
          const float up = gu[g.gate_rows + n + j], a = gate_f32(gu[n + j], g.act, d);
          dgu[n + j] = v[j] * up * d;
          dgu[g.gate_rows + n + j] = v[j] * a;
          out[(size_t)m * g.ldo + n + j] = a * up;
        }
      }
      continue;
    }
    if (bias)
      for (int j = 0; j < left; ++j) v[j] += bias[n + j];
    if (g.epilogue == EPI_QKV && g.rot) {
#pragma unroll
      for (int j = 0; j < 4; j += 2) {
        if (n + j + 1 < g.N && n + j < g.qk_cols) {          // even column; pair = (n + j, n + j + 1)
          const float2 cs = g.rot[(size_t)m * g.rot_pairs + (((n + j) % g.head_dim) >> 1)];
          const float a = v[j], b = v[j + 1];
          v[j] = a * cs.x - b * cs.y;
          v[j + 1] = a * cs.y + b * cs.x;
        }
      }
    }
    if (g.epilogue == EPI_GELU) {
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = gelu_f32(v[j], g.act);
    }
    float* dst = g.epilogue == EPI_RESIDUAL ? g.resid + (size_t)m * g.ldr + n : out + (size_t)m * g.ldo + n;
    if (left == 4 && ((size_t)dst & 15) == 0) {
      if (g.epilogue == EPI_RESIDUAL) v += *(const f32x4*)dst;
      *(f32x4*)dst = v;
    } else {
      for (int j = 0; j < left; ++j) dst[j] = g.epilogue == EPI_RESIDUAL ? dst[j] + v[j] : v[j];
    }
  }
}

// A block of NW waves.  SPLIT: all of them share one 16 T x 16 T tile and take its K in turn, 32 at a
// time, and their sums meet in LDS; otherwise NW = 4 and each has a tile of its own, 2 x 2.
// OPS: a product of the gated MLP.  EPI_GATED (column 2 c of the product is channel c's gate, 2 c + 1 its up factor),
// EPI_DGATED, or EPI_STORE; either operand may stand with its rows along memory (a_rows, w_rows): a lane's four k are then
// four rows, and the 16 lanes of a block read 64 bytes of each, so nothing is transposed first.
// VEC: rows start 16-byte aligned and K (and a gathered piece) is a multiple of 4; otherwise 16-byte
// loads from any float's address, and the last of a row taken apart.
template <int T, int NW, bool SPLIT> struct F32Tile {
  static constexpr int WT = 16 * T, BT = SPLIT ? WT : 2 * WT;       // wave and block tile
  static constexpr int LD = BT + 4, COPIES = SPLIT ? NW : 1;
};
template <int T, int NW, bool SPLIT, bool VEC, bool OPS>
__device__ __forceinline__ void gemm_f32_tile(const GemmArgs& g, const int m0, const int n0, float (*acc_lds)[F32Tile<T, NW, SPLIT>::BT][F32Tile<T, NW, SPLIT>::LD]) {
  constexpr int WT = F32Tile<T, NW, SPLIT>::WT, BT = F32Tile<T, NW, SPLIT>::BT, COPIES = F32Tile<T, NW, SPLIT>::COPIES;
  constexpr int KS = 32;                                     // k per step and wave: two 16-byte loads per row
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, g4 = lane >> 4;
  const int wm = SPLIT ? 0 : (wave >> 1) * WT, wn = SPLIT ? 0 : (wave & 1) * WT;
  const float* const A = (const float*)g.A;
  const float* const W = (const float*)g.W;
  const int kc = g.gather ? g.K / g.gather_n : g.K;          // width of one gathered piece

  const float *arow[T], *wrow[T];
  int am[T];
#pragma unroll
  for (int t = 0; t < T; ++t) {                              // rows beyond the matrix repeat the last one: never stored
    am[t] = min(m0 + wm + t * 16 + l16, g.M - 1);
    arow[t] = A + (size_t)am[t] * (OPS && g.a_rows ? 1 : g.lda);
    int n = min(n0 + wn + t * 16 + l16, g.N - 1);
    if (OPS && g.epilogue == EPI_GATED) n = (n >> 1) + (n & 1) * g.gate_rows;
    wrow[t] = W + (size_t)n * (OPS ? (g.w_rows ? 1 : g.ldw) : g.K);
  }
  auto load4 = [&](const float* row, int k) {                // row[k .. k + 3], zero from K on
    if constexpr (VEC) {
      const f32x4 v = *(const f32x4*)(row + min(k, g.K - 4));
      return k < g.K ? v : f32x4{0.f, 0.f, 0.f, 0.f};
    } else {
      // 16 bytes at any float's address; four loads of four made K = 1023 slower than 64 x 64 vector tiles were
      // (32 768 x 256: 722 us against 473; 312 this way)
      f32x4 v;
      if (k + 4 <= g.K) {
        v = *(const f32x4_any*)(row + k);
      } else {
#pragma unroll
        for (int c = 0; c < 4; ++c) v[c] = k + c < g.K ? row[k + c] : 0.f;
      }
      return v;
    }
  };
  [[maybe_unused]] auto load_rows = [&](const float* row, size_t ld, int k) {       // rows along memory: row[k ld], ...
    f32x4 v;
#pragma unroll
    for (int c = 0; c < 4; ++c) v[c] = row[(size_t)min(k + c, g.K - 1) * ld];
#pragma unroll
    for (int c = 0; c < 4; ++c) if (k + c >= g.K) v[c] = 0.f;
    return v;
  };
  auto load_a = [&](int t, int k) {
    if constexpr (OPS) return g.a_rows ? load_rows(arow[t], g.lda, k) : load4(arow[t], k);
    if (!g.gather) return load4(arow[t], k);
    f32x4 v;
    if constexpr (VEC) {
      const int kk = min(k, g.K - 4), piece = kk / kc;
      v = *(const f32x4*)(A + (size_t)g.gather[(size_t)am[t] * g.gather_n + piece] * g.lda + (kk - piece * kc));
      if (k >= g.K) v = f32x4{0.f, 0.f, 0.f, 0.f};
    } else {
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int kk = min(k + c, g.K - 1), piece = kk / kc;
        v[c] = A[(size_t)g.gather[(size_t)am[t] * g.gather_n + piece] * g.lda + (kk - piece * kc)];
        if (k + c >= g.K) v[c] = 0.f;
      }
    }
    return v;
  };

  f32x4 acc[T][T];                                           // [n][m]: a lane holds 4 consecutive n of one m
#pragma unroll
  for (int i = 0; i < T; ++i)
#pragma unroll
    for (int j = 0; j < T; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  constexpr int KSTEP = SPLIT ? NW * KS : KS;
  f32x4 fa[2][T][2], fw[2][T][2];
  auto fetch = [&](int buf, int k0) {
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        fa[buf][t][h] = load_a(t, k0 + h * 16 + g4 * 4);
        if constexpr (OPS) fw[buf][t][h] = g.w_rows ? load_rows(wrow[t], g.ldw, k0 + h * 16 + g4 * 4) : load4(wrow[t], k0 + h * 16 + g4 * 4);
        else fw[buf][t][h] = load4(wrow[t], k0 + h * 16 + g4 * 4);
      }
  };
  auto multiply = [&](int buf) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int i = 0; i < T; ++i)
#pragma unroll
          for (int j = 0; j < T; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(fw[buf][i][h][c], fa[buf][j][h][c], acc[i][j], 0, 0, 0);
  };
  int k0 = SPLIT ? wave * KS : 0;
  if (k0 < g.K) fetch(0, k0);
  for (; k0 < g.K; k0 += 2 * KSTEP) {
    if (k0 + KSTEP < g.K) fetch(1, k0 + KSTEP);
    multiply(0);
    if (k0 + KSTEP >= g.K) break;
    if (k0 + 2 * KSTEP < g.K) fetch(0, k0 + 2 * KSTEP);
    multiply(1);
  }
#pragma unroll
  for (int i = 0; i < T; ++i)
#pragma unroll
    for (int j = 0; j < T; ++j)
      *(f32x4*)&acc_lds[SPLIT ? wave : 0][wm + j * 16 + l16][wn + i * 16 + g4 * 4] = acc[i][j];
  __syncthreads();

  f32_epilogue<BT, F32Tile<T, NW, SPLIT>::LD, COPIES, 64 * NW, OPS>(g, m0, n0, acc_lds);
}

// 64 x 64 tiles of the gated MLP's products (OPS of gemm_f32_tile) with both operands through LDS, 32 k a step and the next two steps' in
// registers meanwhile; four waves of 32 x 32.  Rows are padded to 36 floats: the 16 rows of a fragment's 16-byte reads lie in different banks.
// Bound: the fp32 matrix instructions, two thirds of whose rate long calls reach.
struct F32Lds { static constexpr int BT = 64, BK = 32, LDK = BK + 4, LD = BT + 4, FLOATS = 4 * BT * LDK; };

// An operand's rows along k: a thread has 4 k of rows tid / 8 and 32 further; across (element k of row r at k * ld + r): 4 rows of k = tid / 16
// and 16 further.  Rows beyond the matrix repeat its last one: they only feed sums that are never stored.
template <bool ACROSS> struct F32Operand {
  const float* at[2];
  size_t step;                         // floats from one k to the next
  int last;                            // across: of the thread's 4 rows the last one that exists, 0 at least
  __device__ __forceinline__ F32Operand(const void* base, int ld, int r0, int rows, int gate_rows) {
    const int tid = threadIdx.x;
    if constexpr (ACROSS) {
      const int r = min(r0 + (tid & 15) * 4, rows - 1);
      step = ld; last = min(3, rows - 1 - r);
#pragma unroll
      for (int i = 0; i < 2; ++i) at[i] = (const float*)base + r + (size_t)((tid >> 4) + i * 16) * ld;
    } else {
      step = 1; last = 3;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        int r = min(r0 + (tid >> 3) + i * 32, rows - 1);
        if (gate_rows) r = (r >> 1) + (r & 1) * gate_rows;
        at[i] = (const float*)base + (size_t)r * ld + (tid & 7) * 4;
      }
    }
  }
  // a whole step; EDGE: the tile has rows beyond the matrix (across)
  template <bool EDGE> __device__ __forceinline__ void load(f32x4* v, int k0) const {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float* const p = at[i] + (size_t)k0 * step;
      if constexpr (ACROSS && EDGE) {
#pragma unroll
        for (int c = 0; c < 4; ++c) v[i][c] = p[min(c, last)];
      } else {
        v[i] = *(const f32x4_any*)p;
      }
    }
  }
  // the last step of a K that is no multiple of 32: zeros from K on
  __device__ __forceinline__ void load_rest(f32x4* v, int k0, int K) const {
    const int tid = threadIdx.x;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int k = k0 + (ACROSS ? (tid >> 4) + i * 16 : (tid & 7) * 4);
      const float* const p = at[i] + (size_t)k0 * step;
#pragma unroll
      for (int c = 0; c < 4; ++c) v[i][c] = (ACROSS ? k : k + c) < K ? p[ACROSS ? min(c, last) : c] : 0.f;
    }
  }
  __device__ __forceinline__ void put(const f32x4* v, float* t) const {
    const int tid = threadIdx.x;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if constexpr (ACROSS) {
#pragma unroll
        for (int c = 0; c < 4; ++c) t[((tid & 15) * 4 + c) * F32Lds::LDK + (tid >> 4) + i * 16] = v[i][c];
      } else {
        *(f32x4*)&t[((tid >> 3) + i * 32) * F32Lds::LDK + (tid & 7) * 4] = v[i];
      }
    }
  }
};

template <bool AK, bool WK, bool EDGE>
__device__ __forceinline__ void gemm_f32_lds_loop(const GemmArgs& g, const int m0, const int n0, float* const lds, f32x4 (*acc)[2]) {
  constexpr int BT = F32Lds::BT, BK = F32Lds::BK, LDK = F32Lds::LDK;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, g4 = lane >> 4, wm = (wave >> 1) * 32, wn = (wave & 1) * 32;
  float* const tile[2] = {lds, lds + 2 * BT * LDK};          // A, W: two stages each
  const F32Operand<AK> A(g.A, g.lda, m0, g.M, 0);
  const F32Operand<WK> W(g.W, g.ldw, n0, g.N, g.epilogue == EPI_GATED ? g.gate_rows : 0);
  auto multiply = [&](int s) {
    const float* const ta = tile[0] + s * BT * LDK + (wm + l16) * LDK + g4 * 4;
    const float* const tw = tile[1] + s * BT * LDK + (wn + l16) * LDK + g4 * 4;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      f32x4 fa[2], fw[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) { fa[j] = *(const f32x4*)(ta + j * 16 * LDK + h * 16); fw[j] = *(const f32x4*)(tw + j * 16 * LDK + h * 16); }
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(fw[i][c], fa[j][c], acc[i][j], 0, 0, 0);
    }
  };
  const int whole = g.K / BK;
  if (whole) {
    // loads beyond the last whole step repeat it, so that every step issues as many and waits for the older ones only
    auto load = [&](f32x4* a, f32x4* w, int i) { const int k0 = min(i, whole - 1) * BK; A.template load<EDGE>(a, k0); W.template load<EDGE>(w, k0); };
    f32x4 va[2][2], vw[2][2];
    load(va[1], vw[1], 0);
    load(va[0], vw[0], 1);
    A.put(va[1], tile[0]); W.put(vw[1], tile[1]);
    load(va[1], vw[1], 2);
    auto step = [&](auto STAGE, int i) {                     // stage s and register set s
      constexpr int s = decltype(STAGE)::value;
      __syncthreads();                                       // stage s is written; stage s ^ 1 has been read
      multiply(s);
      A.put(va[s], tile[0] + (s ^ 1) * BT * LDK); W.put(vw[s], tile[1] + (s ^ 1) * BT * LDK);
      load(va[s], vw[s], i + 3);
    };
    for (int i = 0; i < whole; i += 2) {
      step(std::integral_constant<int, 0>{}, i);
      if (i + 1 >= whole) break;
      step(std::integral_constant<int, 1>{}, i + 1);
    }
  }
  if (whole * BK < g.K) {
    f32x4 a[2], w[2];
    A.load_rest(a, whole * BK, g.K); W.load_rest(w, whole * BK, g.K);
    __syncthreads();                                         // both stages have been read
    A.put(a, tile[0]); W.put(w, tile[1]);
    __syncthreads();
    multiply(0);
  }
}

__device__ __forceinline__ void gemm_f32_lds_tile(const GemmArgs& g, const int m0, const int n0, float* const lds) {
  constexpr int BT = F32Lds::BT;
  f32x4 acc[2][2];                                           // [n][m]: a lane holds 4 consecutive n of one m
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const bool edge = m0 + BT > g.M || n0 + BT > g.N;
  if (!g.w_rows) gemm_f32_lds_loop<false, false, false>(g, m0, n0, lds, acc);
  else if (!g.a_rows && !edge) gemm_f32_lds_loop<false, true, false>(g, m0, n0, lds, acc);
  else if (!g.a_rows) gemm_f32_lds_loop<false, true, true>(g, m0, n0, lds, acc);
  else if (!edge) gemm_f32_lds_loop<true, true, false>(g, m0, n0, lds, acc);
  else gemm_f32_lds_loop<true, true, true>(g, m0, n0, lds, acc);
  __syncthreads();
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, g4 = lane >> 4;
  auto* const out = (float (*)[BT][F32Lds::LD])lds;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) *(f32x4*)&out[0][(wave >> 1) * 32 + j * 16 + l16][(wave & 1) * 32 + i * 16 + g4 * 4] = acc[i][j];
  __syncthreads();
  f32_epilogue<BT, F32Lds::LD, 1, 256, true>(g, m0, n0, out);
}

template <int T, int NW, bool SPLIT, bool VEC>
__global__ __launch_bounds__(64 * NW) void gemm_f32_kernel(GemmArgs g) {
  using F = F32Tile<T, NW, SPLIT>;
  __shared__ __attribute__((aligned(16))) float acc_lds[F::COPIES][F::BT][F::LD];
  gemm_f32_tile<T, NW, SPLIT, VEC, false>(g, blockIdx.y * F::BT, blockIdx.x * F::BT, acc_lds);
}

// Up to three products and two sets of column sums in one launch: products of the sizes this path serves leave most of the
// chip idle, and what is left of a launch is its latency (8 ... 14 us each, the backward pass of 257 tokens through 256 x 1024
// was 12 launches and 79 us).  Blocks first[i] .. first[i + 1] - 1 make product i; then 16 columns of a sum each, 16 rows at a time.
// The product that block b is of, and its number there; the group's sums follow as product a.n.
__device__ __forceinline__ int group_member(const F32Group& a, int& b) {
  int i = 0;
  while (i < a.n && b >= a.first[i + 1]) ++i;
  b -= a.first[i];
  return i;
}

template <int NW> __device__ __forceinline__ void group_sums(const F32Group& a, int b, float* const part) {      // part: [RG][16]
  const int blocks0 = (a.sum[0].cols + 15) / 16;
  const F32Sum& s = a.sum[b >= blocks0];
  if (b >= blocks0) b -= blocks0;
  constexpr int RG = 64 * NW / 16;
  const int c = b * 16 + (threadIdx.x & 15), r0 = threadIdx.x >> 4;
  float v = 0.f;
  if (c < s.cols) {
#pragma unroll 8
    for (int r = r0; r < s.rows; r += RG) v += s.in[(size_t)r * s.ld + c];
  }
  part[threadIdx.x] = v;
  __syncthreads();
  if (threadIdx.x < 16 && c < s.cols) {
    for (int k = 1; k < RG; ++k) v += part[k * 16 + threadIdx.x];
    s.out[c] = v;
  }
}

template <int T, int NW, bool SPLIT, bool VEC>
__global__ __launch_bounds__(64 * NW) void gemm_f32_group_kernel(F32Group a) {
  using F = F32Tile<T, NW, SPLIT>;
  __shared__ __attribute__((aligned(16))) float acc_lds[F::COPIES][F::BT][F::LD];
  static_assert(sizeof(acc_lds) >= 64 * NW * sizeof(float), "partial sums");
  int b = blockIdx.x;
  const int i = group_member(a, b);
  if (i == a.n) { group_sums<NW>(a, b, &acc_lds[0][0][0]); return; }
  const int tiles_n = (a.g[i].N + F::BT - 1) / F::BT, tm = b / tiles_n;
  gemm_f32_tile<T, NW, SPLIT, VEC, true>(a.g[i], tm * F::BT, (b - tm * tiles_n) * F::BT, acc_lds);
}

__global__ __launch_bounds__(256, 4) void gemm_f32_lds_group_kernel(F32Group a) {
  __shared__ __attribute__((aligned(16))) float lds[F32Lds::FLOATS];
  int b = blockIdx.x;
  const int i = group_member(a, b);
  if (i == a.n) { group_sums<4>(a, b, lds); return; }
  const int tiles_n = (a.g[i].N + F32Lds::BT - 1) / F32Lds::BT, tm = b / tiles_n;
  gemm_f32_lds_tile(a.g[i], tm * F32Lds::BT, (b - tm * tiles_n) * F32Lds::BT, lds);
}

static int group_blocks(F32Group& a, int bt) {
  a.first[0] = 0;
  for (int i = 0; i < a.n; ++i) a.first[i + 1] = a.first[i] + ((a.g[i].M + bt - 1) / bt) * ((a.g[i].N + bt - 1) / bt);
  return a.first[a.n] + (a.sum[0].cols + 15) / 16 + (a.sum[1].cols + 15) / 16;
}

template <int T, int NW> static hipError_t launch_group_f32(F32Group& a, hipStream_t s) {
  bool vec = true;
  for (int i = 0; i < a.n; ++i) {
    const GemmArgs& g = a.g[i];
    vec = vec && (g.a_rows || (g.K % 4 == 0 && g.lda % 4 == 0 && (size_t)g.A % 16 == 0)) && (g.w_rows || (g.K % 4 == 0 && g.ldw % 4 == 0 && (size_t)g.W % 16 == 0));
  }
  void* args[] = {(void*)&a};
  const int blocks = group_blocks(a, F32Tile<T, NW, true>::BT);
  return hipLaunchKernel(vec ? (const void*)gemm_f32_group_kernel<T, NW, true, true> : (const void*)gemm_f32_group_kernel<T, NW, true, false>, dim3(blocks), dim3(64 * NW), args, 0, s);
}

static hipError_t launch_lds_group_f32(F32Group& a, hipStream_t s) {
  void* args[] = {(void*)&a};
  const int blocks = group_blocks(a, F32Lds::BT);
  return hipLaunchKernel((const void*)gemm_f32_lds_group_kernel, dim3(blocks), dim3(256), args, 0, s);
}

void count_f32(F32Group& a, int M, int N, int K) {
  a.t16 += (long)((M + 15) / 16) * ((N + 15) / 16);
  a.t32 += (long)((M + 31) / 32) * ((N + 31) / 32);
  a.k = std::max(a.k, K);
  a.flops += 2.0 * M * N * K;
  ++a.products;
}

// Tiles through LDS where their work is long against the longest chain of steps (0.75 us each: 32 k): 1024 x 4096, 512 tokens forward 250 -> 170 us and
// backward 474 -> 318, 2048 tokens 957 -> 470 (109 TFLOP/s) and 1941 -> 1010; 512 x 2048 backward, 1000 tokens 256 -> 210, 512 tokens 133, but 142
// through LDS; 64 x 256, 8192 tokens 118, but 258.  One long product alone pays sooner, its chains share the units with nothing: down of 1000 x
// 512 x 2048 71 -> 50.  Below that, K over eight waves: 16 x 16 tiles while they are few, or while one of the
// products is a few tiles of a long K (the backward pass of 257 tokens, 256 x 1024: 23 us; 27 in 32 x 32 tiles, 34 with K over four waves),
// else 32 x 32.  A launch has fewer than 2^32 threads: 512 for each 32 x 32 tile, and for 16 columns of a sum (2 F + D of them, below 2^19).
hipError_t launch_gemm_f32_group(F32Group& a, hipStream_t s) {
  if (a.t32 >= (1l << 23) - (1l << 15)) return launch_lds_group_f32(a, s);
  if (a.flops >= (a.products == 1 && a.k >= 1024 ? 1e6 : 1.4e6) * a.k) return launch_lds_group_f32(a, s);
  if (a.t16 <= 1024 || (a.k >= 1024 && a.t16 <= 3500)) return launch_group_f32<1, 8>(a, s);
  return launch_group_f32<2, 8>(a, s);
}

template <int T, int NW, bool SPLIT> static void launch_tile_f32(const GemmArgs& g, hipStream_t s) {
  constexpr int BT = SPLIT ? 16 * T : 32 * T;
  const dim3 grid((g.N + BT - 1) / BT, (g.M + BT - 1) / BT);
  const int piece = g.gather ? g.K / g.gather_n : g.K;
  const bool vec = piece % 4 == 0 && g.lda % 4 == 0 && (((size_t)g.A | (size_t)g.W) & 15) == 0;
  if (vec) hipLaunchKernelGGL((gemm_f32_kernel<T, NW, SPLIT, true>), grid, dim3(64 * NW), 0, s, g);
  else hipLaunchKernelGGL((gemm_f32_kernel<T, NW, SPLIT, false>), grid, dim3(64 * NW), 0, s, g);
}

// Tile by how many waves it gives a chip of 1024 SIMDs: 16 x 16 tiles with K split over four waves (or
// eight, where there are few tiles and K is long) up to about four waves per SIMD, then 32 x 32 tiles
// with K split over four, then 64 x 64 blocks of four wave tiles, which read an operand byte least
// often.  One 256-token image (hidden 256, six products of 256 x 256 x 256 ... 1024): 4 - 9 us each, 41
// together, where 64 x 64 tiles of vector arithmetic took 34 - 144 and 428 together.
void launch_gemm_f32(const GemmArgs& g, hipStream_t s) {
  if (g.M <= 0 || g.N <= 0) return;
  if (g.epilogue == EPI_GATED) {                   // an encoder's gated MLP
    F32Group a{};
    a.n = 1;
    a.g[0] = g;
    a.g[0].ldw = g.ldw ? g.ldw : g.K;
    count_f32(a, g.M, g.N, g.K);
    (void)launch_gemm_f32_group(a, s);             // a failure is the runtime's last error, as those of the other launches
    return;
  }
  const long t16 = (long)((g.M + 15) / 16) * ((g.N + 15) / 16), t32 = (long)((g.M + 31) / 32) * ((g.N + 31) / 32);
  if (t16 <= 256 && g.K >= 512) launch_tile_f32<1, 8, true>(g, s);
  else if (t16 <= 1024) launch_tile_f32<1, 4, true>(g, s);
  else if (t32 <= 2048) launch_tile_f32<2, 4, true>(g, s);
  else launch_tile_f32<2, 4, false>(g, s);
}

// ------------------------------------------------------------------------------ attention
// One block = 16 query rows of one segment and head; its NW waves take the keys in turn, 32 at a
// time, each with its own running maximum and sum (softmax in fp32 with expf), and merge at the end.
// Scores are computed transposed, S^T = K Q^T: a lane then holds the scores of ONE query (lane % 16)
// against keys 4 (lane / 16) .. + 3 of each 16, which is where the second product, O^T = V^T P^T,
// wants its second operand if instruction j takes key 4 (lane / 16) + j from lane group lane / 16.
// 256 tokens, 4 heads of 64: 8.7 us (64 blocks of 8 waves), 232 with one thread per query row.
constexpr int F32_BQ = 16, F32_BKV = 32;

template <int DH, int NW>
__global__ __launch_bounds__(64 * NW) void attn_f32_kernel(AttnArgs a) {
  constexpr int DC = (DH + 15) / 16;       // 16-channel chunks
  constexpr int LDO = DC * 16 + 4;
  __shared__ __attribute__((aligned(16))) float o_lds[NW][F32_BQ][LDO];
  __shared__ float m_lds[NW][F32_BQ], l_lds[NW][F32_BQ];
  const AttnWork w = a.work[blockIdx.x];
  const int head = blockIdx.y, D = a.num_heads * DH;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, g4 = lane >> 4;
  const float* const base = (const float*)a.qkv + head * DH;
  const int seg_end = w.seg_start + w.seg_len;

  // channel 16 i + 4 g4 + c of a row is the k of instruction (i, c) that lane group g4 supplies
  f32x4 q[DC];
  const float* const qrow = base + (size_t)min(w.q0 + l16, seg_end - 1) * a.ld_qkv;
#pragma unroll
  for (int i = 0; i < DC; ++i) {
    const int d = 16 * i + 4 * g4;
    q[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (d < DH) q[i] = *(const f32x4*)(qrow + d) * a.scale;
  }
  f32x4 o[DC];
#pragma unroll
  for (int i = 0; i < DC; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;            // of query l16, over the keys this lane group has seen (m: of all groups)

  for (int kv0 = w.seg_start + wave * F32_BKV; kv0 < seg_end; kv0 += NW * F32_BKV) {
    f32x4 kf[2][DC];
    float vf[2][4][DC];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const float* kr = base + D + (size_t)min(kv0 + 16 * b + l16, seg_end - 1) * a.ld_qkv;
#pragma unroll
      for (int i = 0; i < DC; ++i) {
        const int d = 16 * i + 4 * g4;
        kf[b][i] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (d < DH) kf[b][i] = *(const f32x4*)(kr + d);
      }
    }
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float* vr = base + 2 * D + (size_t)min(kv0 + 16 * b + 4 * g4 + j, seg_end - 1) * a.ld_qkv;
#pragma unroll
        for (int i = 0; i < DC; ++i) vf[b][j][i] = vr[min(16 * i + l16, DH - 1)];   // channels beyond DH are never stored
      }
    f32x4 s[2];
    float mt = -INFINITY;
    const float m0 = m;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      s[b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < DC; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c) s[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[b][i][c], q[i][c], s[b], 0, 0, 0);
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        if (kv0 + 16 * b + 4 * g4 + v >= seg_end) s[b][v] = -INFINITY;
        mt = fmaxf(mt, s[b][v]);
      }
    }
    mt = fmaxf(mt, __shfl_xor(mt, 16));
    mt = fmaxf(mt, __shfl_xor(mt, 32));
    m = fmaxf(m, mt);
    // scores may all be -inf (a product beyond the range): those of a wave's share of the keys, of weight
    // zero beside the other waves' -- the maximum subtracted must be finite
    const float mn = m == -INFINITY ? 0.f : m;
    const float alpha = expf(m0 - mn);     // first keys: exp(-inf) = 0
    l *= alpha;
#pragma unroll
    for (int i = 0; i < DC; ++i) o[i] *= alpha;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        s[b][v] = expf(s[b][v] - mn);      // masked entries: exp(-inf) = 0
        l += s[b][v];
      }
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < DC; ++i) o[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[b][j][i], s[b][j], o[i], 0, 0, 0);
  }
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
#pragma unroll
  for (int i = 0; i < DC; ++i) *(f32x4*)&o_lds[wave][l16][16 * i + 4 * g4] = o[i];
  if (lane < 16) { m_lds[wave][l16] = m; l_lds[wave][l16] = l; }
  __syncthreads();
  for (int e = tid; e < F32_BQ * DH; e += 64 * NW) {
    const int r = e / DH, d = e - r * DH;
    if (w.q0 + r >= seg_end) continue;
    float mx = m_lds[0][r];
#pragma unroll
    for (int x = 1; x < NW; ++x) mx = fmaxf(mx, m_lds[x][r]);
    float num = 0.f, den = 0.f;
#pragma unroll
    for (int x = 0; x < NW; ++x) {
      const float f = expf(m_lds[x][r] - mx);                // a wave without keys: exp(-inf) = 0
      num = fmaf(f, o_lds[x][r][d], num);
      den = fmaf(f, l_lds[x][r], den);
    }
    ((float*)a.out)[(size_t)(w.q0 + r) * a.ld_out + head * DH + d] = num / den;
  }
}

bool launch_attn_f32(const AttnArgs& a, hipStream_t s) {
  if (a.num_work <= 0) return true;
  if (a.q_tile != F32_BQ) return false;
#define EPD_ATTN_F32(DH)                                                                             \
  case DH: {                                                                                         \
    constexpr int NW = DH <= 64 ? 8 : 4;                                                             \
    for (AttnArgs c = a; c.num_work > 0; c.num_work -= kMaxGrid, c.work += kMaxGrid)                 \
      hipLaunchKernelGGL((attn_f32_kernel<DH, NW>), dim3(std::min(c.num_work, kMaxGrid), a.num_heads), \
                         dim3(64 * NW), 0, s, c);                                                    \
    return true;                                                                                     \
  }
  switch (a.head_dim) {
    EPD_ATTN_F32(8);
    EPD_ATTN_F32(16);
    EPD_ATTN_F32(32);
    EPD_ATTN_F32(64);
    EPD_ATTN_F32(72);
    EPD_ATTN_F32(80);
    EPD_ATTN_F32(96);
    EPD_ATTN_F32(128);
    default:
      return false;
  }
#undef EPD_ATTN_F32
}

}  // namespace epd
