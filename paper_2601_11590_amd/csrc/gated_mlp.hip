// Gated MLP of a transformer block, Y = (act(X Wg^T + bg) * (X Wu^T + bu)) Wd^T + bd, forward and backward: the
// MLP of encoders whose blocks are gated (epd_encode takes it as an activation), and of the stages behind
// V_m = E(I_m) (paper section 3.1, Eq. 1 and 2).
//
// Forward, many tokens: two products of the bf16 GEMM family.  The first makes gate and up columns of the same channels in
// one tile and multiplies them where the accumulators stand (EPI_GATED), so that G and U never meet memory unless a backward
// pass wants them.  Forward, few tokens: see few_tokens_kernel.
// Backward, from dY and the saved H, P, Q (fp32: G, U):
//   dH = dY Wd;  dU = dH P, dG = dH Q with the saved P = act(G), Q = U act'(G)   in the epilogue of the first product (EPI_DGATED)
//   dX = dG Wg + dU Wu;  dWgu = (dG | dU)^T X;  dWd = dY^T H;  biases: column sums of dG | dU and dY
// Every product is A W^T.  Where K runs along the rows of an operand the ping-pong loop reads it transposed from LDS; products
// too small for its tiles have the operand turned by a kernel first, whichever the model prices lower.  Rounded to bf16 on the way, beside the outputs: H, dG and dU, each once, as operands of
// matrix instructions; P and Q are kept in 20 bits (keep_channels), sums are fp32 throughout.
#include "gemm_bf16_tile.h"
#include "op_error.h"

#include <climits>

namespace epd {

// ------------------------------------------------------------------------------ few tokens
// out[t][n] = sum_k X[t][k] W[n][k] (+ bias), t < 16 NB; GATED: W's rows n and N + n are the gate and up rows of channel n, and
// out = act(gate) * up.  Bound: HBM, every weight is read once.  A block makes 16 rows of W (of both halves) for all tokens; its
// waves take K in turn, 64 at a time, each with a ring of S stages of its own in LDS, which direct loads of 8 rows x 128 bytes
// fill and nobody else reads, so no wave waits for another until their sums meet, in the order of the waves.
//   What it replaced loaded the operands of the matrix instructions straight to registers, 16 rows x 64 bytes an instruction: half
// lines of twice as many rows (3200 x 12 800, 16 tokens: gate and up 52 -> 33.6 us, 3.2 -> 4.9 TB/s, down 32 -> 20.7, 2.6 -> 4.0).  Up to how many tokens: few_up, few_down.
struct FewArgs {
  const void* X; const void* W; const void* bias;
  void* out;
  void *keep_p, *keep_q, *keep_low;    // see GemmArgs (nullptr: not kept)
  int ldx, ldo, T, N, K, act;
};

// N blocks of 16 rows x 64 k of a stage: f[2 * block + k half]; one asm block with its wait, as read_frags
#define EPD_DSR(d, a, o) "ds_read_b128 %" #d ", %" #a " offset:%" #o "\n\t"
template <int N> __device__ __forceinline__ void read_stage(bf16x8* f, uint32_t a0, uint32_t a1) {
  static_assert(N == 1 || N == 2 || N == 4, "blocks");
  if constexpr (N == 1)
    asm volatile(EPD_DSR(0, 2, 4) EPD_DSR(1, 3, 4) "s_waitcnt lgkmcnt(0)" : "=&v"(f[0]), "=&v"(f[1]) : "v"(a0), "v"(a1), "n"(0) : "memory");
  else if constexpr (N == 2)
    asm volatile(EPD_DSR(0, 4, 6) EPD_DSR(2, 4, 7) EPD_DSR(1, 5, 6) EPD_DSR(3, 5, 7) "s_waitcnt lgkmcnt(0)"
                 : "=&v"(f[0]), "=&v"(f[1]), "=&v"(f[2]), "=&v"(f[3]) : "v"(a0), "v"(a1), "n"(0), "n"(2048) : "memory");
  else
    read_frags<4, 0>(f, a0, a1);
}
#undef EPD_DSR

template <int NB, int NW, int S, bool GATED, bool NT>
__global__ __launch_bounds__(64 * NW) void few_tokens_kernel(FewArgs a) {
  constexpr int WB = GATED ? 2 : 1, STAGE = (WB + NB) * 2048, L = 2 * (WB + NB);     // blocks of 16 rows of W; bytes and loads per stage
  static_assert((S - 1) * L < 64 && S >= 2, "load counter");
  static_assert(WB * NB * 1024 <= S * STAGE, "sums");
  __shared__ __attribute__((aligned(1024))) char lds[NW * S * STAGE];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, g4 = lane >> 4, lrow = lane >> 3;
  const int n0 = blockIdx.x * 16;
  char* const ring = lds + wave * S * STAGE;
  // a load brings 8 rows of 64 k; chunk c (8 k) of row r lies in slot c ^ swz(r) of its 128 bytes, so that the 16 rows of a fragment's
  // read lie in different banks.  Rows past the last one repeat it: they only feed sums that are never stored.
  auto swz = [](int row) { return (row >> 1) & 7; };
  uint32_t w_off[2], x_off[2 * NB];
  int k_at[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int r = h * 8 + lrow;
    k_at[h] = ((lane & 7) ^ swz(r)) * 8;
    w_off[h] = ((uint32_t)(min(n0 + r, a.N - 1) - n0) * (uint32_t)a.K + k_at[h]) * 2u;
#pragma unroll
    for (int b = 0; b < NB; ++b) x_off[b * 2 + h] = ((uint32_t)min(b * 16 + r, a.T - 1) * (uint32_t)a.ldx + k_at[h]) * 2u;
  }
  const int nk = (a.K + 63) / 64;
  const bool ragged = a.K % 64 != 0;                       // K is a multiple of 8: whole chunks come from zeros
  auto issue = [&](int slot, int kt) {
    auto from = [&](const char* base, uint32_t off, int h) {
      return ragged && kt == nk - 1 && kt * 64 + k_at[h] >= a.K ? (const char*)zero_bytes : base + (size_t)kt * 128 + (size_t)off;
    };
    char* const to = ring + slot * STAGE;
#pragma unroll
    for (int w = 0; w < WB; ++w)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const char* const p = from((const char*)a.W + ((size_t)n0 + (size_t)w * a.N) * a.K * 2, w_off[h], h);
        __builtin_amdgcn_global_load_lds(EPD_GPTR(p), EPD_LPTR(to + w * 2048 + h * 1024), 16, 0, NT ? 2 : 0);       // 2: non-temporal
      }
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const char* const p = from((const char*)a.X, x_off[b * 2 + h], h);
        __builtin_amdgcn_global_load_lds(EPD_GPTR(p), EPD_LPTR(to + (WB + b) * 2048 + h * 1024), 16, 0, 0);
      }
  };
  f32x4 acc[WB][NB];
#pragma unroll
  for (int s = 0; s < WB; ++s)
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[s][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int steps = wave < nk ? (nk - wave + NW - 1) / NW : 0;
#pragma unroll
  for (int s = 0; s < S - 1; ++s) if (s < steps) issue(s, wave + s * NW);
  const uint32_t rd = (uint32_t)(size_t)EPD_LPTR(ring) + l16 * 128 + ((g4 ^ swz(l16)) * 16);
  int slot = 0;
  for (int i = 0; i < steps; ++i) {
    if (i + S - 1 < steps) {                               // into the slot read last: those reads have returned
      issue(slot == 0 ? S - 1 : slot - 1, wave + (i + S - 1) * NW);
      wait_vmcnt<(S - 1) * L>();
    } else {
      wait_vmcnt<0>();
    }
    bf16x8 w[2 * WB], x[2 * NB];
    const uint32_t at = rd + slot * STAGE;
    read_stage<WB>(w, at, at ^ 64u);
    read_stage<NB>(x, at + WB * 2048, (at ^ 64u) + WB * 2048);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int s = 0; s < WB; ++s)
#pragma unroll
        for (int b = 0; b < NB; ++b) acc[s][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[2 * s + h], x[2 * b + h], acc[s][b], 0, 0, 0);
    if (++slot == S) slot = 0;
  }
  __syncthreads();                                         // the rings are dead from here on
  auto* const sums = (float (*)[WB * NB][16][16])lds;      // [wave][..][token][row]
#pragma unroll
  for (int s = 0; s < WB; ++s)
#pragma unroll
    for (int b = 0; b < NB; ++b) *(f32x4*)&sums[wave][s * NB + b][l16][g4 * 4] = acc[s][b];
  __syncthreads();
  for (int e = tid; e < NB * 64; e += 64 * NW) {           // four rows of W for a token
    const int b = e >> 6, t = (e >> 2) & 15, r = (e & 3) * 4, m = b * 16 + t, n = n0 + r;
    if (m >= a.T || n >= a.N) continue;                    // N is a multiple of 8
    f32x4 v[WB];
#pragma unroll
    for (int s = 0; s < WB; ++s) {
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
      float p[4], q[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float gate = v[0][j], up = v[WB - 1][j];
        if (a.keep_p) {
          q[j] = (a.act == 0 ? gate_act_d<0>(gate, p[j]) : a.act == 1 ? gate_act_d<1>(gate, p[j]) : gate_act_d<2>(gate, p[j])) * up;
          o[j] = p[j] * up;
        } else {
          o[j] = (a.act == 0 ? gate_act<0>(gate) : a.act == 1 ? gate_act<1>(gate) : gate_act<2>(gate)) * up;
        }
      }
      if (a.keep_p) {
        const size_t at = (size_t)m * a.N + n;
        uint2 ph, qh;
        uint32_t low;
        keep_channels(p, q, ph, qh, low);
        *(uint2*)((uint16_t*)a.keep_p + at) = ph;
        *(uint2*)((uint16_t*)a.keep_q + at) = qh;
        *(uint32_t*)((uint8_t*)a.keep_low + at) = low;
      }
    }
    *(uint2*)((uint16_t*)a.out + (size_t)m * a.ldo + n) = pack_bf16x4(o[0], o[1], o[2], o[3]);
  }
}

// The same for one token, where matrix instructions would have 15 empty columns and X as much traffic as W: a channel's row (GATED: its
// two rows) per wave, or per block with the K of its four waves in turn, 16 bytes a lane straight to registers.  Bound: HBM (gate and up of
// 3200 x 12 800: 24.6 us; few_tokens_kernel 28.4; both products 40.3 us, 6.1 TB/s, on other weights each time, 38.6 on the same, which the
// last-level cache holds in part).
template <int SPLIT, int U, bool GATED, bool NT>
__global__ __launch_bounds__(256) void one_token_kernel(FewArgs a) {
  constexpr int WB = GATED ? 2 : 1;
  __shared__ float part[4][WB];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int n = SPLIT == 1 ? blockIdx.x * 4 + wave : blockIdx.x;
  if (n >= a.N) return;                                    // SPLIT 1: whole waves, which no barrier waits for
  const uint16_t* const X = (const uint16_t*)a.X;
  const uint16_t* const row = (const uint16_t*)a.W + (size_t)n * a.K;
  const size_t up = (size_t)a.N * a.K;
  float sum[WB] = {};
  for (int k0 = (SPLIT == 1 ? 0 : wave) * 512 + lane * 8; k0 < a.K; k0 += 512 * SPLIT * U) {
    u32x4 w[U][WB], x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = k0 + u * 512 * SPLIT;                  // K is a multiple of 8
      const bool in = k < a.K;
      x[u] = in ? *(const u32x4*)(X + k) : u32x4{};
#pragma unroll
      for (int s = 0; s < WB; ++s) w[u][s] = in ? (NT ? __builtin_nontemporal_load((const u32x4*)(row + s * up + k)) : *(const u32x4*)(row + s * up + k)) : u32x4{};
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int s = 0; s < WB; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          sum[s] = fmaf(__uint_as_float(w[u][s][i] << 16), __uint_as_float(x[u][i] << 16), sum[s]);
          sum[s] = fmaf(__uint_as_float(w[u][s][i] & 0xffff0000u), __uint_as_float(x[u][i] & 0xffff0000u), sum[s]);
        }
  }
#pragma unroll
  for (int s = 0; s < WB; ++s)
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum[s] += __shfl_xor(sum[s], o);
  if constexpr (SPLIT == 4) {
    if (lane == 0) {
#pragma unroll
      for (int s = 0; s < WB; ++s) part[wave][s] = sum[s];
    }
    __syncthreads();
#pragma unroll
    for (int s = 0; s < WB; ++s) sum[s] = (part[0][s] + part[1][s]) + (part[2][s] + part[3][s]);
  }
  if (lane != 0 || (SPLIT == 4 && wave != 0)) return;
#pragma unroll
  for (int s = 0; s < WB; ++s)
    if (a.bias) sum[s] += bf16_bits_to_float(((const uint16_t*)a.bias)[s * a.N + n]);
  float o = sum[0];
  if constexpr (GATED) {
    const float gate = sum[0], u = sum[WB - 1];
    if (a.keep_p) {
      float p[4] = {}, q[4] = {};
      q[0] = (a.act == 0 ? gate_act_d<0>(gate, p[0]) : a.act == 1 ? gate_act_d<1>(gate, p[0]) : gate_act_d<2>(gate, p[0])) * u;
      o = p[0] * u;
      uint2 ph, qh;
      uint32_t low;
      keep_channels(p, q, ph, qh, low);
      ((uint16_t*)a.keep_p)[n] = (uint16_t)ph.x; ((uint16_t*)a.keep_q)[n] = (uint16_t)qh.x; ((uint8_t*)a.keep_low)[n] = (uint8_t)low;
    } else {
      o = (a.act == 0 ? gate_act<0>(gate) : a.act == 1 ? gate_act<1>(gate) : gate_act<2>(gate)) * u;
    }
  }
  ((__bf16*)a.out)[n] = (__bf16)o;
}

// Which of the two products these kernels take, the others' being the GEMM's (K in parts where that is cheaper).  Weights not in any cache, us:
//   gate and up  1024 x 4096: 32 tokens 6.3 (GEMM 9.8), 64 8.1 (10.2);  3200 x 12 800: 16 30.9 (35.4), 32 37.1 (37.0), 33 41.6 (37.4), 64 48.6 (40.9);
//                2048 x 6144: 33 15.7 (15.8), 64 17.2 (16.5)
//   down         512 x 2048: 64 5.7 (6.9);  1024 x 4096: 32 7.5 (8.2), 33 8.7 (8.1);  1152 x 4304: 16 9.5 (8.8);  3200 x 12 800: 16 20.1 (21.1), 32 25.6 (22.5)
constexpr size_t kL2s = 32u << 20;     // bytes
bool few_up(int T, int D, int F) { return T <= 32 || (T <= 64 && (size_t)4 * D * F <= kL2s); }
bool few_down(int T, int F) { return T <= 16 || (T <= 64 && T * F <= 1 << 17); }

// One token: rows of up to 2048 a wave each (gate and up, K = 1024 4.9 us, a block each 5.8; K = 3200 25.7 and 24.6; down, K = 4096 4.2 and
// 3.7, 12 800 18.2 and 15.4).  More: waves per block and stages are the fastest of two to four choices each at hidden 1024, 1152,
// 3200 and 4096 (they lie within 10 %).
template <bool GATED, bool NT> static hipError_t launch_few_as(const FewArgs& a, hipStream_t s) {
  void* args[] = {(void*)&a};
  if (a.T == 1) {
    const bool split = a.K > 2048;
    const void* f = split ? (const void*)one_token_kernel<4, GATED ? 2 : 4, GATED, NT> : (const void*)one_token_kernel<1, 4, GATED, NT>;
    return hipLaunchKernel(f, dim3(split ? a.N : (a.N + 3) / 4), dim3(256), args, 0, s);
  }
  constexpr int NW1 = GATED ? 4 : 8, NW2 = GATED ? 2 : 8, S2 = GATED ? 4 : 3, NW4 = GATED ? 2 : 4;
  const void* f;
  int nw;
  if (a.T <= 16) { f = (const void*)few_tokens_kernel<1, NW1, 3, GATED, NT>; nw = NW1; }
  else if (a.T <= 32 || (GATED && NT)) { f = (const void*)few_tokens_kernel<2, NW2, S2, GATED, NT>; nw = NW2; }       // (see few_up)
  else { f = (const void*)few_tokens_kernel<4, NW4, 3, GATED, NT && !GATED>; nw = NW4; }
  return hipLaunchKernel(f, dim3((a.N + 15) / 16), dim3(64 * nw), args, 0, s);
}

// Weights beyond the L2s together (32 MB) are read as non-temporal, past what X stays in: 16 tokens through 3200 x 12 800, gate and
// up 33.8 -> 30.7 us, down 20.9 -> 20.1; through 4096 x 14 336 43.7 -> 39.1 and 24.6 -> 23.1.  Smaller ones may still be there from the call before, which
// that would undo: both of 1024 x 4096 again and again 10.0 us, non-temporal 11.3 (on other weights each time 12.3 and 11.9).
template <bool GATED> static hipError_t launch_few(const FewArgs& a, hipStream_t s) {
  return (size_t)(GATED ? 2 : 1) * a.N * a.K * 2 > kL2s ? launch_few_as<GATED, true>(a, s) : launch_few_as<GATED, false>(a, s);
}

// ------------------------------------------------------------------------------ transpose, column sums
// out[c][r] = in[r][c], r < R, c < C; zeros for R <= r < ldo.  Tiles of 64 x 64 through LDS, 16 bytes per access on
// both sides (C, ldi, ldo multiples of 8).  Bound: HBM.
struct TransposeArgs { const uint16_t* in; uint16_t* out; int R, C, ldi, ldo; };

__global__ __launch_bounds__(256) void transpose_bf16_kernel(TransposeArgs a) {
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

static hipError_t transpose(const void* in, int ldi, void* out, int ldo, int R, int C, hipStream_t s) {
  TransposeArgs a{(const uint16_t*)in, (uint16_t*)out, R, C, ldi, ldo};
  void* args[] = {(void*)&a};
  return hipLaunchKernel((const void*)transpose_bf16_kernel, dim3((ldo + 63) / 64, (C + 63) / 64), dim3(256), args, 0, s);
}

// Column sums for the gradients of the biases, in two steps with fixed orders: partial sums of rows, fp32, then these over the
// parts.  (dG | dU leaves its partial sums in the epilogue that makes it.)
struct PartSums { const __bf16* in; float* out; int rows, cols, ld, per; };       // out[p][c] over rows p * per ...
__global__ __launch_bounds__(256) void part_sums_kernel(PartSums a) {
  const int c = (blockIdx.y * 256 + threadIdx.x) * 8, r0 = blockIdx.x * a.per, r1 = min(r0 + a.per, a.rows);
  if (c >= a.cols) return;
  float v[8] = {};
#pragma unroll 4
  for (int r = r0; r < r1; ++r) {
    const bf16x8 x = *(const bf16x8*)(a.in + (size_t)r * a.ld + c);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] += (float)x[j];
  }
  float* const to = a.out + (size_t)blockIdx.x * a.cols + c;
  *(float4*)to = make_float4(v[0], v[1], v[2], v[3]);
  *(float4*)(to + 4) = make_float4(v[4], v[5], v[6], v[7]);
}

struct SumParts { const float* in; __bf16* out; int parts, cols; };
struct SumPartsArgs { SumParts job[2]; int blocks0; };                            // blocks of 16 columns: those of job 0, then of job 1
__global__ __launch_bounds__(256) void sum_parts_kernel(SumPartsArgs a) {
  __shared__ float part[16][16];
  const bool second = (int)blockIdx.x >= a.blocks0;
  const SumParts& s = a.job[second];
  const int l = threadIdx.x & 15, c = ((int)blockIdx.x - (second ? a.blocks0 : 0)) * 16 + l, g = threadIdx.x >> 4;
  float v = 0.f;
  if (c < s.cols) {
#pragma unroll 8
    for (int p = g; p < s.parts; p += 16) v += s.in[(size_t)p * s.cols + c];
  }
  part[g][l] = v;
  __syncthreads();
  if (g == 0 && c < s.cols) {
#pragma unroll
    for (int i = 1; i < 16; ++i) v += part[i][l];
    s.out[c] = (__bf16)v;
  }
}

// out[m][c] = sum_p in[p][m][c] + bias[c], parts of a cut K in their order.  Bound: the caches they are still in, and HBM.
struct JoinArgs { const float* in; const __bf16* bias; __bf16* out; int parts, M, N, ldo; };
constexpr int kSplits = 8, kSplitRows = 8192, kPartK = 256;       // parts, their rows together, and the shortest part
__global__ __launch_bounds__(256) void join_kernel(JoinArgs a) {
  const int i = blockIdx.x * 256 + threadIdx.x, row = i / (a.N / 8), c = (i - row * (a.N / 8)) * 8;
  if (row >= a.M) return;
  const float* const from = a.in + (size_t)row * a.N + c;
  const size_t step = (size_t)a.M * a.N;
  f32x4 v[kSplits][2];
#pragma unroll
  for (int p = 0; p < kSplits; ++p)
    if (p < a.parts) { v[p][0] = *(const f32x4*)(from + p * step); v[p][1] = *(const f32x4*)(from + p * step + 4); }
  f32x4 lo = v[0][0], hi = v[0][1];
#pragma unroll
  for (int p = 1; p < kSplits; ++p)
    if (p < a.parts) { lo += v[p][0]; hi += v[p][1]; }
  if (a.bias) {
    const bf16x8 b = *(const bf16x8*)(a.bias + c);
#pragma unroll
    for (int j = 0; j < 4; ++j) { lo[j] += (float)b[j]; hi[j] += (float)b[4 + j]; }
  }
  const uint2 x = pack_bf16x4(lo[0], lo[1], lo[2], lo[3]), y = pack_bf16x4(hi[0], hi[1], hi[2], hi[3]);
  *(uint4*)(a.out + (size_t)row * a.ldo + c) = make_uint4(x.x, x.y, y.x, y.y);
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
template <int EPI> static hipError_t launch_gated_epi(const GemmArgs& g, hipStream_t s) {
  switch (g.tile_cfg - 1) {
    case 0: return launch_clamped<T0, EPI>(g, s);
    case 2: return launch_clamped<T2, EPI>(g, s);
    case 5: return launch_clamped<T5, EPI>(g, s);
    case 7: return launch_clamped<T7, EPI>(g, s);
    case 8: return launch_clamped<T8, EPI>(g, s);
    default: return launch_clamped<T4, EPI>(g, s);
  }
}

// operands that stand [K, rows]: the tiles of the ping-pong loop (both: those whose wave rows are whole blocks of 64)
template <int EPI> static hipError_t launch_w_rows(const GemmArgs& g, hipStream_t s) {
  if (g.tile_cfg == 3) return launch_clamped<T2, EPI, 2>(g, s);
  if (g.tile_cfg == 6) return launch_clamped<T5, EPI, 2>(g, s);
  return launch_clamped<T0, EPI, 2>(g, s);
}

static hipError_t launch_both_rows(const GemmArgs& a, const GemmArgs* b, hipStream_t s) {
  return a.tile_cfg == 3 ? launch_pair<T2>(a, b, s) : launch_pair<T0>(a, b, s);
}

static hipError_t launch_gated_whole(const GemmArgs& g, hipStream_t s) {
  if (g.a_rows) return launch_both_rows(g, nullptr, s);
  if (g.w_rows && g.epilogue == EPI_DGATED) return launch_w_rows<EPI_DGATED>(g, s);
  if (g.w_rows) return launch_w_rows<EPI_STORE>(g, s);
  if (g.epilogue == EPI_GATED) return launch_gated_epi<EPI_GATED>(g, s);
  if (g.epilogue == EPI_DGATED) return launch_gated_epi<EPI_DGATED>(g, s);
  return launch_gated_epi<EPI_STORE>(g, s);
}

// Time of a launch of these products in us: per round of blocks alpha * K / 1024 + beta[epilogue] (the last round, of a
// share f of the blocks, last0 + last1 * f of that), and `launch`.  Fitted to 200 shapes in every tile (hidden 1024, 1152 and 3200, 65 ... 32 768
// tokens, forward and backward products, random operands): 7 ... 12 % off in the mean, and the tile it ranks first is within 3 % of the
// fastest in 288 of 308 choices, 0.7 % off in the mean.  (Constants fitted to launches on other buffers each time are 0.5 % off there
// and leave whole passes 2 ... 7 % slower: they price the second launch of a cut higher than it costs inside a pass.)  The encoder's own planner (plan_tiles) ranks its
// launches beside attention and keeps its constants; it offers 256 x 128 tiles to residual adds only, which here win wherever a narrow
// output fills one round of them (6272 x 1024 x 8192: 93 us, 112 in 128 x 128 tiles, 142 in 256 x 256).
//   An operand that stands [K, rows] costs alpha what reading fragments in halves of 8 bytes costs: a factor for W, and for both
// (0: no kernel).  25 600 x 3200 x 8192 in 256 x 256 tiles 1093 us, 1044 with both operands turned, which takes 170 more; 8192 x 3200 x
// 25 600, W alone, 1072 and 1065 + 60.
struct ProductTile { int cfg, bm, bn, blocks; double last0, last1, alpha, launch, beta[4], rows_w, rows_both; };     // beta: store, gated, gated and kept, dgated
constexpr ProductTile kProductTiles[] = {
  {0, 256, 256, 1, 0.62, 0.28, 23.8, 3.4, {6.0, 6.9, 13.2, 24.4}, 1.02, 1.07},
  {2, 256, 128, 1, 0.62, 0.25, 14.1, 3.9, {4.1, 3.9, 9.0, 12.7}, 1.10, 1.18},
  {4, 128, 128, 2, 0.51, 0.44, 16.1, 3.4, {2.5, 0.6, 3.8, 7.0}, 0.0, 0.0},
  {5, 320, 256, 1, 0.64, 0.30, 28.4, 1.7, {8.9, 10.1, 17.3, 34.0}, 1.04, 0.0},
  {7, 64, 64, 2, 0.54, 0.49, 6.6, 3.1, {1.3, 1.5, 2.0, 1.7}, 0.0, 0.0},
  {8, 64, 128, 2, 0.48, 0.55, 10.3, 3.4, {1.9, 1.1, 2.3, 2.7}, 0.0, 0.0},
};

static double rows_factor(const ProductTile& t, const GemmArgs& g) { return g.a_rows ? t.rows_both : g.w_rows ? t.rows_w : 1.0; }      // 0: the tile has no such kernel

static long product_tiles(const ProductTile& t, long M, long N) { return ((M + t.bm - 1) / t.bm) * ((N + t.bn - 1) / t.bn); }

static double tiles_cost(const ProductTile& t, long tiles, double K, int kind, long cus) {
  const long slots = cus * t.blocks, full = tiles / slots, rest = tiles % slots;
  return t.launch + ((double)full + (rest ? t.last0 + t.last1 * (double)rest / (double)slots : 0.0)) * (t.alpha * K / 1024.0 + t.beta[kind]);
}

static double product_cost(const ProductTile& t, long M, long N, double K, int kind, long cus) { return tiles_cost(t, product_tiles(t, M, N), K, kind, cus); }

// One launch of the cheapest tile, or whole rounds of a large one and the rest of the rows in the cheapest for them:
// 8192 x 3200 x 25 600 is 416 tiles of 256 x 256, priced two rounds (1075 us); 6080 rows in one round of 320 x 256 and 2112 in one of 256 x 128 take 980.
static TilePlan plan_product(const GemmArgs& g, long cus) {
  const int kind = g.epilogue == EPI_GATED ? (g.keep_p ? 2 : 1) : g.epilogue == EPI_DGATED ? 3 : 0;
  auto best_tile = [&](long rows, double& cost) {
    int best = 0;
    cost = 1e300;
    for (const ProductTile& t : kProductTiles) {
      const double f = rows_factor(t, g), c = product_cost(t, rows, g.N, f * g.K, kind, cus);
      if (f > 0.0 && c < cost) { cost = c; best = t.cfg; }
    }
    return best;
  };
  TilePlan plan = {0, 0, 0.0, 0};
  plan.tile = best_tile(g.M, plan.cost);
  const double keep = 0.95 * plan.cost;          // a second launch has to be worth it: nothing hides its ramp
  for (const ProductTile& t : kProductTiles) {
    const double f = rows_factor(t, g);
    if (t.blocks != 1 || f == 0.0) continue;     // the large tiles
    const long tm = ((long)g.M + t.bm - 1) / t.bm, tn = ((long)g.N + t.bn - 1) / t.bn, full = tm * tn / cus;
    for (long rounds = full; rounds >= 1 && rounds >= full - 1; --rounds) {
      const long body = std::min(rounds * cus / tn, (long)g.M / t.bm) * t.bm;
      if (body < 1 || body >= g.M) continue;
      double tail;
      const int tail_tile = best_tile(g.M - body, tail);
      const double cost = product_cost(t, body, g.N, f * g.K, kind, cus) + tail;
      if (cost < keep && cost < plan.cost) plan = {t.cfg, (int)body, cost, tail_tile};
    }
  }
  return plan;
}

static int tile_rows(int tile) { return tile == 5 ? 320 : tile == 4 ? 128 : tile >= 7 ? 64 : 256; }

// EPI_STORE, EPI_GATED or EPI_DGATED with operands that are not read past their ends.  filled: the rows of g.sums that the
// launches fill (two per tile along M).
hipError_t launch_gemm_bf16_gated(const GemmArgs& args, hipStream_t s, int* filled) {
  if (args.M <= 0 || args.N <= 0) return hipSuccess;
  GemmArgs g = args;
  TilePlan plan = {0, 0, 0.0, 0};
  if (g.tile_cfg == 0) {
    plan = plan_product(g, g.compute_units > 0 ? g.compute_units : num_cus());
    g.tile_cfg = plan.tile + 1;
  }
  auto sum_rows = [](const GemmArgs& x) { return (x.M + tile_rows(x.tile_cfg - 1) - 1) / tile_rows(x.tile_cfg - 1) * 2; };
  if (plan.body_rows <= 0) {
    if (filled) *filled = sum_rows(g);
    return launch_gated_whole(g, s);
  }
  const size_t mb = plan.body_rows;
  GemmArgs body = g, tail = g;
  body.M = (int)mb;
  tail.M = g.M - (int)mb; tail.tile_cfg = plan.tail_tile + 1;
  tail.A = (const __bf16*)g.A + (g.a_rows ? mb : mb * g.lda);
  tail.sum_row0 = g.sum_row0 + sum_rows(body);
  if (g.out) tail.out = (__bf16*)g.out + mb * g.ldo;
  if (g.keep_p) {
    tail.keep_p = (uint16_t*)g.keep_p + mb * g.gate_rows;
    tail.keep_q = (uint16_t*)g.keep_q + mb * g.gate_rows;
    tail.keep_low = (uint8_t*)g.keep_low + mb * g.gate_rows;
  }
  if (g.dgu) tail.dgu = (__bf16*)g.dgu + mb * g.lddgu;
  if (g.stats_in) tail.stats_in = g.stats_in + mb * g.stats_n;
  if (filled) *filled = sum_rows(body) + sum_rows(tail);
  if (hipError_t e = launch_gated_whole(body, s)) return e;
  return launch_gated_whole(tail, s);
}

// A product whose operands stand [K, rows] (g.a_rows, g.w_rows): as they stand, or turned into a_t and w_t (rows of round_up(K, 8))
// first, which costs a pass over them at about 4.5 TB/s and a launch each.
struct Turned { GemmArgs g; bool turn; double cost; };
static Turned plan_turned(const GemmArgs& g, void* a_t, void* w_t) {
  const long cus = num_cus();
  GemmArgs t = g;
  double turn = 0.0;
  t.K = (g.K + 7) / 8 * 8;
  if (g.a_rows) { t.A = a_t; t.lda = t.K; t.a_rows = 0; turn += 3.0 + 4.0 * g.K * (double)g.M / 4.5e6; }
  if (g.w_rows) { t.W = w_t; t.ldw = t.K; t.w_rows = 0; turn += 3.0 + 4.0 * g.K * (double)g.N / 4.5e6; }
  turn += plan_product(t, cus).cost;
  const double stands = plan_product(g, cus).cost;
  return turn < stands ? Turned{t, true, turn} : Turned{g, false, stands};
}

// Few rows leave most of the chip without a tile: K cut into parts then fills it, at the price of fp32 sums that another kernel joins:
// 128 x 1024 x 4096 19.6 -> 8.9 us, 512 x 3200 x 12 800 75.8 -> 46.7, 128 and 1024 rows x 3200 x 25 600 with W across its rows 181 -> 48.9 and 277 ->
// 149.  Priced as its tiles (5 % less: the sums' stores cost less than the rounding to bf16) and the traffic of the sums; over 90 sizes the choice
// between this and one pass is 1.1 % off in the mean, 12 % at most.
struct SplitPlan { int tile, parts, k_part; double cost; };
static SplitPlan plan_split(const GemmArgs& g, long cus) {
  SplitPlan plan = {0, 1, g.K, 1e300};
  for (const ProductTile& t : kProductTiles) {
    const double f = rows_factor(t, g);
    if ((t.cfg != 0 && t.cfg != 2 && t.cfg != 7) || f == 0.0) continue;      // (the others' best lie within 1 % of these)
    for (int n = 2; n <= kSplits && (int64_t)n * g.M <= kSplitRows && g.K / n >= kPartK; ++n) {
      const int k_part = (g.K + 64 * n - 1) / (64 * n) * 64, parts = (g.K + k_part - 1) / k_part;
      const double c = 0.95 * tiles_cost(t, product_tiles(t, g.M, g.N) * parts, f * k_part, 0, cus) + 3.0 + (4.0 * parts + 2.0) * g.M * (double)g.N / 4e6;
      if (c < plan.cost) plan = {t.cfg, parts, k_part, c};
    }
  }
  return plan;
}

static hipError_t launch_parts(const GemmArgs& g, const SplitPlan& p, float* sums, hipStream_t s) {
  GemmArgs x = g;
  x.out = sums;
  hipError_t e;
  if (g.w_rows) e = p.tile == 2 ? launch_split<T2, 2>(x, p.parts, p.k_part, s) : launch_split<T0, 2>(x, p.parts, p.k_part, s);
  else if (p.tile == 7) e = launch_split<T7, 0>(x, p.parts, p.k_part, s);
  else e = p.tile == 2 ? launch_split<T2, 0>(x, p.parts, p.k_part, s) : launch_split<T0, 0>(x, p.parts, p.k_part, s);
  if (e != hipSuccess) return e;
  JoinArgs j{sums, (const __bf16*)g.bias, (__bf16*)g.out, p.parts, g.M, g.N, g.ldo};
  void* args[] = {(void*)&j};
  return hipLaunchKernel((const void*)join_kernel, dim3((g.M * (g.N / 8) + 255) / 256), dim3(256), args, 0, s);
}

// parts: room for kSplitRows (or kSplits * M) rows of fp32 sums, or nullptr; sum_rows: see launch_gemm_bf16_gated
static hipError_t launch_product(const GemmArgs& g, void* a_t, void* w_t, float* parts, hipStream_t s, int* sum_rows = nullptr) {
  const Turned t = plan_turned(g, a_t, w_t);
  if (parts) {
    const SplitPlan p = plan_split(g, num_cus());
    if (p.cost < t.cost) return launch_parts(g, p, parts, s);
  }
  if (t.turn && g.a_rows) if (hipError_t e = transpose(g.A, g.lda, a_t, t.g.lda, g.K, g.M, s)) return e;
  if (t.turn && g.w_rows) if (hipError_t e = transpose(g.W, g.ldw, w_t, t.g.ldw, g.K, g.N, s)) return e;
  return launch_gemm_bf16_gated(t.g, s, sum_rows);
}

// Two products of one K whose operands stand [K, rows], each wanted or not: in one launch, whose rounds they share, where that is
// priced lower than one after the other.  The choice does not depend on which are wanted, so that a gradient has the same bits in every
// call.
static hipError_t launch_products(const GemmArgs& a, bool want_a, const GemmArgs& b, bool want_b, void* a_t, void* w_t, hipStream_t s) {
  if (!want_a && !want_b) return hipSuccess;
  const long cus = num_cus();
  double least = plan_turned(a, a_t, w_t).cost + plan_turned(b, a_t, w_t).cost;
  int tile = -1;
  for (const ProductTile& t : kProductTiles) {
    if (t.rows_both == 0.0) continue;
    const double c = tiles_cost(t, product_tiles(t, a.M, a.N) + product_tiles(t, b.M, b.N), t.rows_both * a.K, 0, cus);
    if (c < least) { least = c; tile = t.cfg; }
  }
  if (tile >= 0) {
    GemmArgs first = want_a ? a : b;
    first.tile_cfg = tile + 1;
    return launch_both_rows(first, want_a && want_b ? &b : nullptr, s);
  }
  if (want_a) if (hipError_t e = launch_product(a, a_t, w_t, nullptr, s)) return e;
  return want_b ? launch_product(b, a_t, w_t, nullptr, s) : hipSuccess;
}

}  // namespace epd

using namespace epd;

namespace {

// ------------------------------------------------------------------ workspace layout (bytes)
struct GatedLayout {
  int es;                               // element size
  size_t h, parts, dgu, a_t, w_t, sums_gu, sums_d, total;
};

constexpr int kParts = 512, kPartRows = 16;            // partial sums of dY at most, of 16 rows or more each (6272 x 1024 in 64 rows each: 10 us, not 5)
int part_rows(int tokens) { return std::max(kPartRows, (tokens + kParts - 1) / kParts); }

GatedLayout gated_layout(const epd_gated_mlp_cfg& c) {
  GatedLayout L;
  const bool bf = c.dtype == EPD_BF16;
  auto up = [](size_t v, size_t a) { return (v + a - 1) / a * a; };
  const size_t D = c.hidden, F = c.mlp_dim, T = c.max_tokens;
  L.es = bf ? 2 : 4;
  size_t off = 0;
  auto take = [&](size_t bytes) { const size_t o = off; off = up(off + bytes, 256); return o; };
  L.h = take(T * F * L.es);
  // sums of parts of K, of Y and dX (a few rows of Y take none, nor a short K)
  const bool parts = (c.training && 2 * c.mlp_dim >= 2 * kPartK) || (!few_down(c.max_tokens, c.mlp_dim) && c.mlp_dim >= 2 * kPartK);
  L.parts = take(bf && parts ? std::min<size_t>(T * kSplits, kSplitRows) * D * 4 : 0);
  L.dgu = L.a_t = L.w_t = L.sums_gu = L.sums_d = 0;
  if (c.training) L.dgu = take(T * 2 * F * L.es);
  if (c.training && bf) {
    const size_t Tp = up(T, 8);
    L.a_t = take(std::max(2 * F, D) * Tp * L.es);                                   // (dG | dU)^T, dY^T
    L.w_t = take(std::max(std::max(D, F) * Tp, 2 * F * D) * L.es);                  // X^T, H^T, Wd^T, Wgu^T
    L.sums_gu = take(c.use_bias ? (up(T, 64) / 32 + 2) * 2 * F * 4 : 0);            // two rows per tile of 64 rows or more; a cut launch has a tile more
    L.sums_d = take(c.use_bias ? std::min<size_t>(kParts, (T + kPartRows - 1) / kPartRows) * D * 4 : 0);
  }
  L.total = off;
  return L;
}

// What a forward call leaves for the backward pass.  bf16: H, P, Q and the bytes that P and Q share (keep_channels), [tokens, F]
// each; fp32: G | U.
struct Saved { void *h, *p, *q, *low; size_t total; };

Saved saved_parts(const epd_gated_mlp_cfg& c, void* saved, int64_t tokens) {
  const size_t n = (size_t)tokens * c.mlp_dim;
  Saved s{saved, nullptr, nullptr, nullptr, 0};
  if (c.dtype == EPD_F32) { s.total = n * 8; return s; }
  const size_t part = (n * 2 + 255) / 256 * 256;
  if (saved) { s.p = (char*)saved + part; s.q = (char*)saved + 2 * part; s.low = (char*)saved + 3 * part; }
  s.total = 3 * part + n;
  return s;
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
  if (c->hidden > 65536 || c->mlp_dim > kGatedMlpDim || (int64_t)c->hidden * c->mlp_dim >= (1ll << 30))
    return op_fail(EPD_ERR_UNSUPPORTED, "%s: hidden %d, mlp_dim %d: at most 65536, %d and 2^30 together", who, c->hidden, c->mlp_dim, kGatedMlpDim);
  if (c->max_tokens >= kMaxTokens || (int64_t)c->max_tokens * std::max(c->mlp_dim, c->hidden) >= kGatedElements[c->dtype])
    return op_fail(EPD_ERR_UNSUPPORTED, "%s: max_tokens %d too large", who, c->max_tokens);
  return EPD_OK;
}

// Rows of X, Y or a gradient; what the row of a single token would be apart from the next is not looked at.
epd_status check_rows(const char* who, const char* name, const epd_gated_mlp_cfg& c, const void* p, int64_t& ld, int tokens) {
  if (tokens == 1) ld = c.hidden;
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

}  // namespace

extern "C" {

uint64_t epd_gated_mlp_workspace_bytes(const epd_gated_mlp_cfg* cfg) {
  if (check_cfg("epd_gated_mlp_workspace_bytes", cfg) != EPD_OK) return 0;
  return gated_layout(*cfg).total;
}

uint64_t epd_gated_mlp_saved_bytes(const epd_gated_mlp_cfg* cfg, int32_t tokens) {
  if (check_cfg("epd_gated_mlp_saved_bytes", cfg) != EPD_OK) return 0;
  if (tokens < 0 || tokens > cfg->max_tokens) { op_fail(EPD_ERR_SHAPE, "epd_gated_mlp_saved_bytes: tokens %d: 0 .. max_tokens %d", tokens, cfg->max_tokens); return 0; }
  return saved_parts(*cfg, nullptr, tokens).total;
}

epd_status epd_gated_mlp(const epd_gated_mlp_cfg* cfg, const epd_gated_mlp_weights* w, const void* x, int64_t ld_x, int32_t tokens, void* y, int64_t ld_y,
                         void* saved, void* workspace, uint64_t workspace_bytes, void* stream) {
  const char* const who = "epd_gated_mlp";
  if (epd_status s = check_call(who, cfg, w, tokens, workspace, workspace_bytes)) return s;
  if (tokens == 0) return EPD_OK;
  const epd_gated_mlp_cfg& c = *cfg;
  if (epd_status s = check_rows(who, "x", c, x, ld_x, tokens)) return s;
  if (epd_status s = check_rows(who, "y", c, y, ld_y, tokens)) return s;
  if ((uintptr_t)saved % (c.dtype == EPD_BF16 ? 16 : 4)) return op_fail(EPD_ERR_UNSUPPORTED, "%s: saved must be aligned to 16 bytes (bf16) or 4 (fp32)", who);
  const GatedLayout L = gated_layout(c);
  const bool bf = c.dtype == EPD_BF16;
  const int D = c.hidden, F = c.mlp_dim, T = tokens;
  const Saved keep = saved_parts(c, saved, T);
  void* const H = bf && saved ? keep.h : (char*)workspace + L.h;
  hipStream_t st = (hipStream_t)stream;
  GemmArgs up{}, down{};
  up.A = x; up.lda = (int)ld_x; up.W = w->gate_up_w; up.ldw = D; up.bias = c.use_bias ? w->gate_up_b : nullptr;
  up.M = T; up.N = bf ? (F + 15) / 16 * 32 : 2 * F; up.K = D; up.epilogue = EPI_GATED; up.act = act_code(c);
  up.gate_rows = F; up.out = H; up.ldo = F;
  if (bf) { up.keep_p = keep.p; up.keep_q = keep.q; up.keep_low = keep.low; }
  else { up.gu = saved; up.ldgu = 2 * F; }
  down.A = H; down.lda = F; down.W = w->down_w; down.ldw = F; down.bias = c.use_bias ? w->down_b : nullptr;
  down.M = T; down.N = D; down.K = F; down.epilogue = EPI_STORE; down.out = y; down.ldo = (int)ld_y;
  hipError_t e;
  if (bf) {
    if (few_up(T, D, F)) {
      const FewArgs a{x, up.W, up.bias, H, keep.p, keep.q, keep.low, up.lda, F, T, F, D, up.act};
      e = launch_few<true>(a, st);
    } else {
      e = launch_gemm_bf16_gated(up, st, nullptr);
    }
    if (e == hipSuccess && few_down(T, F)) {
      const FewArgs a{H, down.W, down.bias, y, nullptr, nullptr, nullptr, F, down.ldo, T, D, F, 0};
      e = launch_few<false>(a, st);
    } else if (e == hipSuccess) {
      e = launch_product(down, nullptr, nullptr, (float*)((char*)workspace + L.parts), st);
    }
  } else {
    F32Group a{}, b{};
    a.n = b.n = 1;
    a.g[0] = up; b.g[0] = down;
    count_f32(a, up.M, up.N, up.K);
    count_f32(b, down.M, down.N, down.K);
    e = launch_gemm_f32_group(a, st);
    if (e == hipSuccess) e = launch_gemm_f32_group(b, st);
  }
  return e == hipSuccess ? EPD_OK : op_launch_failed(who, e);
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
  auto failed = [&]() { return op_launch_failed(who, e); };
  if (tokens == 0) {                     // sums over no token
    if (grads->gate_up_w) ok(clear(bf, grads->gate_up_w, 2 * F * D, st));
    if (grads->down_w && e == hipSuccess) ok(clear(bf, grads->down_w, D * F, st));
    if (grads->gate_up_b && e == hipSuccess) ok(clear(bf, grads->gate_up_b, 2 * F, st));
    if (grads->down_b && e == hipSuccess) ok(clear(bf, grads->down_b, D, st));
    return e == hipSuccess ? EPD_OK : failed();
  }
  if (epd_status s = check_rows(who, "x", c, x, ld_x, tokens)) return s;
  if (epd_status s = check_rows(who, "dy", c, dy, ld_dy, tokens)) return s;
  if (!saved) return op_fail(EPD_ERR_INVALID_ARG, "%s: saved is NULL", who);
  int64_t ld_dx = grads->ld_dx;
  if (grads->dx) if (epd_status s = check_rows(who, "dx", c, grads->dx, ld_dx, tokens)) return s;
  const GatedLayout L = gated_layout(c);
  char* const ws = (char*)workspace;
  const int T = tokens, iD = c.hidden, iF = c.mlp_dim;
  const bool want_gu = grads->gate_up_w || grads->gate_up_b, want_h = grads->dx || want_gu || (!bf && grads->down_w);
  // dH = dY Wd, and at once dG and dU (fp32: and H)
  GemmArgs dh{}, dx{}, dgu{}, dd{};
  dh.A = dy; dh.lda = (int)ld_dy; dh.M = T; dh.N = iF; dh.K = iD; dh.epilogue = EPI_DGATED; dh.act = act_code(c);
  dh.gate_rows = iF; dh.dgu = ws + L.dgu; dh.lddgu = 2 * iF;
  const Saved keep = saved_parts(c, (void*)saved, T);
  if (bf) { dh.keep_p = keep.p; dh.keep_q = keep.q; dh.keep_low = keep.low; }
  else { dh.gu = (void*)saved; dh.ldgu = 2 * iF; dh.out = ws + L.h; dh.ldo = iF; }
  // dX = (dG | dU) Wgu,  dWgu = (dG | dU)^T X,  dWd = dY^T H
  dx.A = ws + L.dgu; dx.lda = 2 * iF; dx.M = T; dx.N = iD; dx.K = 2 * iF; dx.epilogue = EPI_STORE; dx.out = grads->dx; dx.ldo = (int)ld_dx;
  dgu.M = 2 * iF; dgu.N = iD; dgu.epilogue = EPI_STORE; dgu.out = grads->gate_up_w; dgu.ldo = iD;
  dd.M = iD; dd.N = iF; dd.epilogue = EPI_STORE; dd.out = grads->down_w; dd.ldo = iF;
  dh.W = w->down_w; dh.ldw = iF; dh.w_rows = 1;
  dx.W = w->gate_up_w; dx.ldw = iD; dx.w_rows = 1;
  dgu.A = ws + L.dgu; dgu.lda = 2 * iF; dgu.a_rows = 1; dgu.W = x; dgu.ldw = (int)ld_x; dgu.w_rows = 1; dgu.K = T;
  dd.A = dy; dd.lda = (int)ld_dy; dd.a_rows = 1; dd.W = bf ? keep.h : ws + L.h; dd.ldw = iF; dd.w_rows = 1; dd.K = T;
  if (!bf) {
    F32Group a{}, b{};
    a.n = 1; a.g[0] = dh;
    count_f32(a, dh.M, dh.N, dh.K);
    for (const GemmArgs* g : {&dx, &dgu, &dd}) count_f32(b, g->M, g->N, g->K);
    if (want_h && !ok(launch_gemm_f32_group(a, st))) return failed();
    if (grads->dx) b.g[b.n++] = dx;
    if (grads->gate_up_w) b.g[b.n++] = dgu;
    if (grads->down_w) b.g[b.n++] = dd;
    if (grads->gate_up_b) b.sum[0] = F32Sum{(const float*)(ws + L.dgu), (float*)grads->gate_up_b, T, 2 * iF, 2 * iF};
    if (grads->down_b) b.sum[1] = F32Sum{(const float*)dy, (float*)grads->down_b, T, iD, (int)ld_dy};
    if ((b.n || b.sum[0].cols || b.sum[1].cols) && !ok(launch_gemm_f32_group(b, st))) return failed();
    return EPD_OK;
  }
  SumPartsArgs sums{};
  if (want_h) {
    if (grads->gate_up_b) dh.sums = (float*)(ws + L.sums_gu);
    int rows = 0;
    if (!ok(launch_product(dh, nullptr, ws + L.w_t, nullptr, st, &rows))) return failed();
    if (grads->gate_up_b) sums.job[0] = SumParts{dh.sums, (__bf16*)grads->gate_up_b, rows, 2 * iF};
  }
  if (grads->down_b) {
    const int per = part_rows(T), parts = (T + per - 1) / per;
    PartSums p{(const __bf16*)dy, (float*)(ws + L.sums_d), T, iD, (int)ld_dy, per};
    void* args[] = {(void*)&p};
    if (!ok(hipLaunchKernel((const void*)part_sums_kernel, dim3(parts, (iD + 2047) / 2048), dim3(256), args, 0, st))) return failed();
    sums.job[1] = SumParts{p.out, (__bf16*)grads->down_b, parts, iD};
  }
  if (sums.job[0].cols || sums.job[1].cols) {
    sums.blocks0 = (sums.job[0].cols + 15) / 16;
    void* args[] = {(void*)&sums};
    if (!ok(hipLaunchKernel((const void*)sum_parts_kernel, dim3(sums.blocks0 + (sums.job[1].cols + 15) / 16), dim3(256), args, 0, st))) return failed();
  }
  if (grads->dx && !ok(launch_product(dx, nullptr, ws + L.w_t, (float*)(ws + L.parts), st))) return failed();
  if (!ok(launch_products(dgu, grads->gate_up_w, dd, grads->down_w, ws + L.a_t, ws + L.w_t, st))) return failed();
  return EPD_OK;
}

}  // extern "C"
