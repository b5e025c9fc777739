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

// Bound: large products by the matrix cores and the clock that the power limit leaves them (32 768 x 3200 x 12 800: 1074 us, 2.5 POP/s at 1394 W of the
// board's 1400; on zeros 831 us at 1070 W); those of few rounds by the last, which is not full, and the epilogue, which nothing hides (7057 x 1152 x
// 4304: 42.5 us; its operations at that rate 28).
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

template <class T> hipError_t launch_whole(const GemmArgs& g, hipStream_t s) {
  const int tiles_m = (g.M + T::BM - 1) / T::BM, tiles_n = (g.N + T::BN - 1) / T::BN;
  GemmArgs a = g;
  a.group_m = raster_group<T>(g, tiles_m, tiles_n, (long)T::MINBLK * num_cus());
  void* args[] = {(void*)&a};
  return hipLaunchKernel(g.out_f32 ? (const void*)int8_gemm_kernel<T, OUT_F32> : (const void*)int8_gemm_kernel<T, OUT_BF16>, dim3(tiles_m * tiles_n), dim3(T::NT), args, 0, s);
}

// K in parts of k_part (pairs of values, a multiple of 64), each a block's own: int32 sums [part][M][N] for int8_scale_kernel.  Few rows leave most
// of the chip idle: 200 x 12 800 x 3200 19.1 + 4.0 us, whole 32.0; 1000 rows 47.3 + 6.3, whole 67.4.  (Weights of three products in turn, which the
// chip's last cache holds; out of HBM 25 and 57 together.)
struct SplitArgs { GemmArgs g; int k_part; };
template <class T> __global__ __launch_bounds__(T::NT, T::MINBLK) void int8_split_kernel(SplitArgs p) {
  __shared__ __attribute__((aligned(1024))) char lds[T::LDS_BYTES + T::BM * 4 + T::BN * 8];
  GemmArgs g = p.g;
  g.zeros = zero_bytes;
  const int tiles_n = (g.N + T::BN - 1) / T::BN, tiles_m = (g.M + T::BM - 1) / T::BM;
  const int t = xcd_remap(blockIdx.x, gridDim.x), part = t / (tiles_m * tiles_n), k0 = part * p.k_part;
  g.A = (const uint16_t*)g.A + k0;
  g.W = (const uint16_t*)g.W + k0;
  g.out = (int*)g.out + (size_t)part * g.M * g.N;
  g.K = min(p.k_part, g.K - k0);
  int tm, tn;
  tile_coords(t - part * (tiles_m * tiles_n), tiles_m, tiles_n, g.group_m, tm, tn);
  gemm_tile<T, EPI_INT8_SUMS, OUT_F32, false, false, T::PINGPONG, T::PINGPONG>(g, tm * T::BM, tn * T::BN, lds);
}

// y = sum of the parts * scales + bias, eight columns a thread.  Bound: latency, a launch and a read of what the last kernel wrote.
struct ScaleArgs { const int* in; const float *row_scales, *col_scales, *col_bias; void* out; int parts, M, N, ldo; };
constexpr int kSplits = 8, kPartK = 256;                          // parts at most, and the shortest one in pairs
constexpr int64_t kSplitSums = 1 << 24;                           // sums of all parts at most: 64 MB
template <typename T> __global__ __launch_bounds__(256) void int8_scale_kernel(ScaleArgs a) {
  const int i = blockIdx.x * 256 + threadIdx.x, row = i / (a.N / 8), c = (i - row * (a.N / 8)) * 8;
  if (row >= a.M) return;
  const int* const from = a.in + (size_t)row * a.N + c;
  const size_t step = (size_t)a.M * a.N;
  i32x4 v[kSplits][2];
#pragma unroll
  for (int p = 0; p < kSplits; ++p)
    if (p < a.parts) { v[p][0] = *(const i32x4*)(from + p * step); v[p][1] = *(const i32x4*)(from + p * step + 4); }
  const float rs = a.row_scales[row];
  f32x4 o[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    i32x4 sum = v[0][h];
#pragma unroll
    for (int p = 1; p < kSplits; ++p) if (p < a.parts) sum += v[p][h];
    const f32x4 cs = *(const f32x4*)(a.col_scales + c + 4 * h), cb = a.col_bias ? *(const f32x4*)(a.col_bias + c + 4 * h) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < 4; ++j) o[h][j] = fmaf((float)sum[j] * rs, cs[j], cb[j]);
  }
  if constexpr (sizeof(T) == 4) {
    float* const to = (float*)a.out + (size_t)row * a.ldo + c;
    *(f32x4*)to = o[0]; *(f32x4*)(to + 4) = o[1];
  } else {
    const uint2 x = pack_bf16x4(o[0][0], o[0][1], o[0][2], o[0][3]), y = pack_bf16x4(o[1][0], o[1][1], o[1][2], o[1][3]);
    *(uint4*)((uint16_t*)a.out + (size_t)row * a.ldo + c) = make_uint4(x.x, x.y, y.x, y.y);
  }
}

template <class T> hipError_t launch_parts(const GemmArgs& g, int parts, int k_part, void* sums, hipStream_t s) {
  const int tiles_m = (g.M + T::BM - 1) / T::BM, tiles_n = (g.N + T::BN - 1) / T::BN;
  SplitArgs p{g, k_part};
  p.g.out = sums; p.g.ldo = g.N;
  GemmArgs of_part = g;
  of_part.K = k_part;
  p.g.group_m = raster_group<T>(of_part, tiles_m, tiles_n, (long)T::MINBLK * num_cus());
  void* args[] = {(void*)&p};
  if (hipError_t e = hipLaunchKernel((const void*)int8_split_kernel<T>, dim3(tiles_m * tiles_n * parts), dim3(T::NT), args, 0, s)) return e;
  ScaleArgs j{(const int*)sums, g.row_scales, g.col_scales, g.col_bias, g.out, parts, g.M, g.N, g.ldo};
  void* jargs[] = {(void*)&j};
  return hipLaunchKernel(g.out_f32 ? (const void*)int8_scale_kernel<float> : (const void*)int8_scale_kernel<__bf16>, dim3((g.M * (g.N / 8) + 255) / 256), dim3(256), jargs, 0, s);
}

// ------------------------------------------------------------------------------ few tokens
struct FewArgs {
  const void *X, *W;
  const float *x_scales, *scales, *bias;
  void* out;
  int ldx, ldo, T, N, K, out_f32;    // ldx, K: bytes
};

__device__ __forceinline__ void store_one(const FewArgs& a, int t, int n, int sum) {
  const float v = fmaf((float)sum * a.x_scales[t], a.scales[n], a.bias ? a.bias[n] : 0.f);
  if (a.out_f32) ((float*)a.out)[(size_t)t * a.ldo + n] = v;
  else ((__bf16*)a.out)[(size_t)t * a.ldo + n] = (__bf16)v;
}

// One token: R rows of W a wave, or a block with K of its four waves in turn, 16 bytes a lane and access straight to registers, four
// products an instruction.  Bound: the weights' way to the chip: 3200 x 12 800 8.3 us, 4.9 TB/s, out of its last cache, 9.3 us, 4.4 TB/s, out of HBM.
template <int SPLIT, int R, int U>
__global__ __launch_bounds__(256) void int8_one_kernel(FewArgs a) {
  __shared__ int part[4][R];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int n0 = (SPLIT == 1 ? blockIdx.x * 4 + wave : blockIdx.x) * R;
  if (n0 >= a.N) return;                                   // SPLIT 1: whole waves, which no barrier waits for; N is a multiple of 8, R divides it
  const uint8_t* const X = (const uint8_t*)a.X;
  const uint8_t* const row = (const uint8_t*)a.W + (size_t)n0 * a.K;
  int sum[R] = {};
  for (int k0 = ((SPLIT == 1 ? 0 : wave) * 64 + lane) * 16; k0 < a.K; k0 += 1024 * SPLIT * U) {
    i32x4 w[U][R], x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = k0 + u * 1024 * SPLIT;                 // K is a multiple of 16
      const bool in = k < a.K;
      x[u] = in ? *(const i32x4*)(X + k) : i32x4{};
#pragma unroll
      for (int r = 0; r < R; ++r) w[u][r] = in ? *(const i32x4*)(row + (size_t)r * a.K + k) : i32x4{};
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[r] = __builtin_amdgcn_sdot4(w[u][r][i], x[u][i], sum[r], false);
  }
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum[r] += __shfl_xor(sum[r], o);
  if constexpr (SPLIT == 4) {
    if (lane == 0) {
#pragma unroll
      for (int r = 0; r < R; ++r) part[wave][r] = sum[r];
    }
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int r = 0; r < R; ++r) sum[r] = (part[0][r] + part[1][r]) + (part[2][r] + part[3][r]);
  }
#pragma unroll
  for (int r = 0; r < R; ++r) if (lane == r) store_one(a, 0, n0 + r, sum[r]);
}

// Up to 16 NB tokens: a block makes 16 rows of W for all of them; its waves take K in turn, 128 at a time, each with a ring of S stages of
// its own in LDS, which direct loads of 8 rows x 128 bytes fill and nobody else reads, so no wave waits for another until their sums meet.
// Bound: the weights' way to the chip, each read once: 16 tokens through 3200 x 12 800 9.1 ... 9.7 us, 4.2 ... 4.5 TB/s, out of its last cache, 10.9 out of HBM.
#define EPD_DSR(d, a, o) "ds_read_b128 %" #d ", %" #a " offset:%" #o "\n\t"
template <int N> __device__ __forceinline__ void read_stage(bf16x8* f, uint32_t a0, uint32_t a1) {      // one asm block with its wait, as read_frags
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

template <int NB, int NW, int S>
__global__ __launch_bounds__(64 * NW) void int8_few_kernel(FewArgs a) {
  constexpr int STAGE = (1 + NB) * 2048, L = 2 * (1 + NB);                         // bytes and loads per stage
  static_assert((S - 1) * L < 64 && S >= 2, "load counter");
  static_assert(NB * 1024 <= S * STAGE, "sums");
  __shared__ __attribute__((aligned(1024))) char lds[NW * S * STAGE];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, g4 = lane >> 4, lrow = lane >> 3;
  const int n0 = blockIdx.x * 16;
  char* const ring = lds + wave * S * STAGE;
  // chunk c (16 bytes) of row r lies in slot c ^ swz(r) of its 128 bytes, so that the 16 rows of a fragment's read lie in different banks.
  // Rows past the last one repeat it: they only feed sums that are never stored.
  auto swz = [](int row) { return (row >> 1) & 7; };
  uint32_t w_off[2], x_off[2 * NB];
  int k_at[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int r = h * 8 + lrow;
    k_at[h] = ((lane & 7) ^ swz(r)) * 16;
    w_off[h] = (uint32_t)(min(n0 + r, a.N - 1) - n0) * (uint32_t)a.K + k_at[h];
#pragma unroll
    for (int b = 0; b < NB; ++b) x_off[b * 2 + h] = (uint32_t)min(b * 16 + r, a.T - 1) * (uint32_t)a.ldx + k_at[h];
  }
  const int nk = (a.K + 127) / 128;
  const bool ragged = a.K % 128 != 0;                      // K is a multiple of 16: whole chunks come from zeros
  auto issue = [&](int slot, int kt) {
    auto from = [&](const char* base, uint32_t off, int h) {
      return ragged && kt == nk - 1 && kt * 128 + k_at[h] >= a.K ? (const char*)zero_bytes : base + (size_t)kt * 128 + (size_t)off;
    };
    char* const to = ring + slot * STAGE;
#pragma unroll
    for (int h = 0; h < 2; ++h)
      __builtin_amdgcn_global_load_lds(EPD_GPTR(from((const char*)a.W + (size_t)n0 * a.K, w_off[h], h)), EPD_LPTR(to + h * 1024), 16, 0, 0);
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        __builtin_amdgcn_global_load_lds(EPD_GPTR(from((const char*)a.X, x_off[b * 2 + h], h)), EPD_LPTR(to + (1 + b) * 2048 + h * 1024), 16, 0, 0);
  };
  f32x4 acc[NB];                                           // int32 sums (see mfma16)
#pragma unroll
  for (int b = 0; b < NB; ++b) acc[b] = f32x4{0.f, 0.f, 0.f, 0.f};
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
    bf16x8 w[2], x[2 * NB];
    const uint32_t at = rd + slot * STAGE;
    read_stage<1>(w, at, at ^ 64u);
    read_stage<NB>(x, at + 2048, (at ^ 64u) + 2048);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int b = 0; b < NB; ++b) acc[b] = mfma16<true>(w[h], x[2 * b + h], acc[b]);
    if (++slot == S) slot = 0;
  }
  __syncthreads();                                         // the rings are dead from here on
  auto* const sums = (int (*)[NB][16][16])lds;             // [wave][..][token][row]
#pragma unroll
  for (int b = 0; b < NB; ++b) *(f32x4*)&sums[wave][b][l16][g4 * 4] = acc[b];
  __syncthreads();
  for (int e = tid; e < NB * 64; e += 64 * NW) {           // four rows of W for a token
    const int b = e >> 6, t = (e >> 2) & 15, r = (e & 3) * 4, m = b * 16 + t, n = n0 + r;
    if (m >= a.T || n >= a.N) continue;                    // N is a multiple of 8
    i32x4 v = *(const i32x4*)&sums[0][b][t][r];
#pragma unroll
    for (int i = 1; i < NW; ++i) v += *(const i32x4*)&sums[i][b][t][r];
    const f32x4 cs = *(const f32x4*)(a.scales + n), cb = a.bias ? *(const f32x4*)(a.bias + n) : f32x4{0.f, 0.f, 0.f, 0.f};
    const float rs = a.x_scales[m];
    f32x4 o;
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] = fmaf((float)v[j] * rs, cs[j], cb[j]);
    if (a.out_f32) *(f32x4*)((float*)a.out + (size_t)m * a.ldo + n) = o;
    else *(uint2*)((uint16_t*)a.out + (size_t)m * a.ldo + n) = pack_bf16x4(o[0], o[1], o[2], o[3]);
  }
}

// Which calls these kernels take, the others' being the GEMM's.  Weights not in L2, us (K x N):
//   17 tokens  3200 x 12 800 11.1 (GEMM 11.0), 3200 x 9600 9.0 (10.5), 12 800 x 3200 10.0 (11.8)
//   32 tokens  3200 x 12 800 11.9 (11.2), 3200 x 9600 9.1 (10.4), 12 800 x 3200 13.1 (13.0), 1024 x 4096 4.1 (5.9)
//   64 tokens  1152 x 4304 4.9 (6.7), 4096 x 1024 6.0 (7.7), 4096 x 4096 8.2 (9.5), 3200 x 6400 8.3 (10.2), 1024 x 8192 5.2 (6.3), 6144 x 2048 8.2 (9.6);
//              but 3200 x 9600 14.3 (10.5), 1152 x 16 384 9.0 (7.0), 12 800 x 3200 18.0 (13.8)
bool takes_few(int T, int K, int N) { return T <= 32 || (T <= 64 && N <= 8192 && K <= 8192); }

// One token: rows of up to 4096 bytes two a wave, longer ones a block each (3200 x 12 800 8.3 us, 8.8 with a block each; 12 800 x 3200 8.4 and
// 7.8).  More: waves and stages are the fastest of ten choices at the sizes above, within 10 %: two waves of four stages where there are many
// blocks (16 tokens through 3200 x 12 800 9.1 us, with four waves 10.0), four otherwise (through 12 800 x 3200 10.2, with two 12); the rings
// of 64 tokens and four waves fill a unit's LDS, so beyond a block per unit two waves it is (2048 x 6144 6.5, with four 8.4; 2048 x 4096 5.7 and 5.2).
// Reading the weights as non-temporal is no faster at any of them (16 tokens through 3200 x 12 800: 9.9).
hipError_t launch_few(const GemmArgs& g, hipStream_t s) {
  FewArgs a{g.A, g.W, g.row_scales, g.col_scales, g.col_bias, g.out, g.lda * 2, g.ldo, g.M, g.N, g.K * 2, g.out_f32};
  void* args[] = {(void*)&a};
  if (a.T == 1) {
    if (a.K > 4096) return hipLaunchKernel((const void*)int8_one_kernel<4, 1, 4>, dim3(a.N), dim3(256), args, 0, s);
    return hipLaunchKernel((const void*)int8_one_kernel<1, 2, 4>, dim3((a.N + 7) / 8), dim3(256), args, 0, s);
  }
  const void* f;
  int nw = 4;
  if (a.T <= 16 && a.N > 8192) { f = (const void*)int8_few_kernel<1, 2, 4>; nw = 2; }
  else if (a.T <= 16) f = (const void*)int8_few_kernel<1, 4, 4>;
  else if (a.T <= 32) f = (const void*)int8_few_kernel<2, 4, 3>;
  else if (a.N > 4096) { f = (const void*)int8_few_kernel<4, 2, 3>; nw = 2; }
  else f = (const void*)int8_few_kernel<4, 4, 3>;
  return hipLaunchKernel(f, dim3((a.N + 15) / 16), dim3(64 * nw), args, 0, s);
}

// ------------------------------------------------------------------------------ plans
hipError_t launch_tile(const GemmArgs& g, int tile, hipStream_t s) {
  switch (tile) {
    case 0: return launch_whole<T0>(g, s);
    case 2: return launch_whole<T2>(g, s);
    case 5: return launch_whole<T5>(g, s);
    case 7: return launch_whole<T7>(g, s);
    case 8: return launch_whole<T8>(g, s);
    default: return launch_whole<T4>(g, s);
  }
}

hipError_t launch_split(const GemmArgs& g, int tile, int parts, int k_part, void* sums, hipStream_t s) {
  switch (tile) {
    case 0: return launch_parts<T0>(g, parts, k_part, sums, s);
    case 2: return launch_parts<T2>(g, parts, k_part, sums, s);
    case 8: return launch_parts<T8>(g, parts, k_part, sums, s);
    default: return launch_parts<T7>(g, parts, k_part, sums, s);
  }
}

// Time of a launch in us: per round of blocks alpha * K / 2048 + beta (bf16 or fp32 out; the last round, of a share f of the blocks, last0 +
// last1 * f of that), and `launch`.  Fitted to 194 shapes in every tile (17 ... 32 768 tokens, K 32 ... 12 800, N 16 ... 12 800, weights not in L2):
// 5 ... 10 % off in the mean.  Over these shapes, whole and in parts, what it ranks first is 1.3 % slower than the fastest in the mean, 19 % at
// most (568 tokens, 12 800 x 3200: 48.8 us, 41.1), and within 3 % in 166.
struct Int8Tile { int cfg, bm, bn, blocks; double last0, last1, launch, alpha, beta[2]; bool parts; };
constexpr Int8Tile kInt8Tiles[] = {
  {0, 256, 256, 1, 0.64, 0.34, 1.5, 25.3, {8.1, 10.3}, true},
  {2, 256, 128, 1, 0.69, 0.35, 1.5, 14.3, {5.3, 6.5}, true},
  {4, 128, 128, 2, 0.64, 0.47, 1.5, 15.5, {3.6, 4.7}, false},
  {5, 320, 256, 1, 0.69, 0.32, 1.5, 28.4, {9.5, 12.0}, false},
  {7, 64, 64, 2, 0.56, 0.58, 3.0, 6.3, {1.6, 2.1}, true},
  {8, 64, 128, 2, 0.55, 0.56, 2.7, 10.2, {2.1, 2.9}, true},
};

struct Int8Plan { int tile, body_rows, tail_tile, parts, k_part; double cost; };

long int8_tiles(const Int8Tile& t, long M, long N) { return ((M + t.bm - 1) / t.bm) * ((N + t.bn - 1) / t.bn); }

double int8_cost(const Int8Tile& t, long tiles, double K, bool f32, long cus) {
  const long slots = cus * t.blocks, full = tiles / slots, rest = tiles % slots;
  return t.launch + ((double)full + (rest ? t.last0 + t.last1 * (double)rest / (double)slots : 0.0)) * (t.alpha * K / 1024.0 + t.beta[f32]);
}

// One launch of the cheapest tile; whole rounds of a large one and the rest of the rows in the cheapest for them, where that is 5 % less; or
// (few rows) K in parts, whose sums cost a launch and their traffic, where that is 6 % less (closer calls are decided better without: over the
// shapes above 1.57 % off with no such margin, 1.33 % with it, 1.73 % at 15 %).
Int8Plan plan_int8(const GemmArgs& g, long cus) {
  const bool f32 = g.out_f32;
  Int8Plan plan = {0, 0, 0, 1, g.K, 1e300};
  auto best_tile = [&](long rows, double& cost) {
    int best = 0;
    cost = 1e300;
    for (const Int8Tile& t : kInt8Tiles) {
      const double c = int8_cost(t, int8_tiles(t, rows, g.N), g.K, f32, cus);
      if (c < cost) { cost = c; best = t.cfg; }
    }
    return best;
  };
  plan.tile = best_tile(g.M, plan.cost);
  const double whole = plan.cost;
  for (const Int8Tile& t : kInt8Tiles) {
    if (t.blocks != 1) continue;
    const long tn = ((long)g.N + t.bn - 1) / t.bn, full = int8_tiles(t, g.M, g.N) / cus;
    for (long rounds = full; rounds >= 1 && rounds >= full - 1; --rounds) {
      const long body = std::min(rounds * cus / tn, (long)g.M / t.bm) * t.bm;
      if (body < 1 || body >= g.M) continue;
      double tail;
      const int tail_tile = best_tile(g.M - body, tail);
      const double c = int8_cost(t, int8_tiles(t, body, g.N), g.K, f32, cus) + tail;
      if (c < 0.95 * whole && c < plan.cost) plan = {t.cfg, (int)body, tail_tile, 1, g.K, c};
    }
  }
  for (const Int8Tile& t : kInt8Tiles)
    for (int n = 2; t.parts && n <= kSplits && (int64_t)n * g.M * g.N <= kSplitSums && g.K / n >= kPartK; ++n) {
      const int k_part = (g.K + 64 * n - 1) / (64 * n) * 64, parts = (g.K + k_part - 1) / k_part;
      const double c = 0.96 * int8_cost(t, int8_tiles(t, g.M, g.N) * parts, k_part, true, cus) + 2.0 + 0.95e-6 * parts * g.M * (double)g.N;
      if (1.06 * c < whole && c < plan.cost) plan = {t.cfg, 0, 0, parts, k_part, c};
    }
  return plan;
}

hipError_t launch_product(const GemmArgs& g, void* sums, hipStream_t s) {
  const Int8Plan p = plan_int8(g, num_cus());
  if (p.parts > 1) return launch_split(g, p.tile, p.parts, p.k_part, sums, s);
  if (!p.body_rows) return launch_tile(g, p.tile, s);
  GemmArgs body = g, tail = g;
  const size_t mb = p.body_rows;
  body.M = p.body_rows;
  tail.M = g.M - p.body_rows;
  tail.A = (const uint16_t*)g.A + mb * g.lda;
  tail.out = g.out_f32 ? (void*)((float*)g.out + mb * g.ldo) : (void*)((__bf16*)g.out + mb * g.ldo);
  tail.row_scales = g.row_scales + mb;
  if (hipError_t e = launch_tile(body, p.tile, s)) return e;
  return launch_tile(tail, p.tail_tile, s);
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

uint64_t workspace_bytes(const epd_int8_linear_cfg& c) {             // sums of parts of K; 256 where there are none
  const int64_t parts = std::min(kSplits, c.in_features / 2 / kPartK);
  return parts < 2 ? 256 : ((uint64_t)std::min(parts * c.max_tokens * c.out_features, kSplitSums) * 4 + 255) / 256 * 256;
}

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
  if (ld_x < K || ld_x >= kMaxTokens || ld_x % 16) return op_fail(EPD_ERR_SHAPE, "%s: rows of x are %lld apart: a multiple of 16, in_features %d .. 2^22 - 16", who, (long long)ld_x, K);
  if (ld_y < N || ld_y >= most_y || ld_y % 8) return op_fail(EPD_ERR_SHAPE, "%s: rows of y are %lld apart: a multiple of 8, out_features %d .. %lld", who, (long long)ld_y, N, (long long)most_y - 8);
  if (((uintptr_t)x | (uintptr_t)y) % 16) return op_fail(EPD_ERR_UNSUPPORTED, "%s: x and y must be aligned to 16 bytes", who);
  if ((uintptr_t)x_scale % 4) return op_fail(EPD_ERR_INVALID_ARG, "%s: x_scale is not aligned", who);
  GemmArgs g{};
  g.A = x; g.lda = (int)(ld_x / 2); g.W = w->w; g.ldw = K / 2; g.M = tokens; g.N = N; g.K = K / 2;
  g.epilogue = EPI_INT8; g.out = y; g.ldo = (int)ld_y; g.out_f32 = c.out_dtype == EPD_F32;
  g.row_scales = x_scale; g.col_scales = w->scale; g.col_bias = c.use_bias ? w->bias : nullptr;
  const hipError_t e = takes_few(tokens, K, N) ? launch_few(g, (hipStream_t)stream) : launch_product(g, workspace, (hipStream_t)stream);
  return e == hipSuccess ? EPD_OK : op_launch_failed(who, e);
}

}  // extern "C"
