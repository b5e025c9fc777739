// The norm at the entry of a block of the stage behind V_m = E(I_m) (paper section 3.1, Eq. 1 and 2) as an operator: the residual's addition,
// RMS norm and, for a product in 8 bits, the rows' rounding to 8 bits with a scale each; its backward pass; and the same rounding for rows
// that are not normalised (weights, activations), and back.
//
//   s = x + r;   y = s / sqrt(mean(s^2) + eps) * gain;   m = max(max |y|, 2^-100), q = rint(y * (127 / m)), scale = m / 127
// s is not rounded before y is made of it.  Backward, at the s that was kept: n = s * rstd, g = dy * gain,
//   dx = ds + rstd * (g - n * mean(g n)),   dgain = sum over rows of dy * n
// rstd is made again: its sum passes over the row beside that of g n.
// Bound: HBM, each row is read once, held in registers as fp32 between its sums and its results, and written once (backward, beyond 16 384
// columns: read twice, once out of a cache).  32 768 x 3200 with its sum and 8 bits 5.7 TB/s, backward 30 000 x 1024 4.8.
//
#include "op_error.h"
#include "rows.h"

#include <algorithm>
#include <cmath>

namespace epd {

namespace {

constexpr int kNormDim = 65536;
constexpr float kLeastMax = 7.888609052210118e-31f;       // 2^-100: 127 / m stays finite, rows of zeros need no case of their own

__device__ __forceinline__ void store_q8(int8_t* p, int left, const float* v, float to_q) {
  int q[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) q[i] = (int)rintf(v[i] * to_q);
  if (left >= 8) {
    pair1 u;
#pragma unroll
    for (int h = 0; h < 2; ++h)
      u[h] = (uint32_t)(q[4 * h] & 255) | (uint32_t)(q[4 * h + 1] & 255) << 8 | (uint32_t)(q[4 * h + 2] & 255) << 16 | (uint32_t)q[4 * h + 3] << 24;
    *(pair1*)p = u;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) if (i < left) p[i] = (int8_t)q[i];
  }
}

struct Sum { static __device__ __forceinline__ float of(float a, float b) { return a + b; } };
struct Most { static __device__ __forceinline__ uint32_t of(uint32_t a, uint32_t b) { return a > b ? a : b; } };

template <class Op, class V> __device__ __forceinline__ V with_lane(V v, uint32_t other) { return Op::of(v, __builtin_bit_cast(V, other)); }
template <class Op, int CTRL, class V> __device__ __forceinline__ V with_dpp(V v) {
  return with_lane<Op>(v, (uint32_t)__builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}
// Sum or maximum over the row's TPR threads, in an order of its own whatever else the block does; every thread gets it.  Lanes meet in
// vector instructions, without LDS.
template <class Op, int TPR, class V> __device__ __forceinline__ V row_reduce(V v, void* lds) {
  v = with_dpp<Op, 0xB1>(v);                               // quad_perm 1,0,3,2
  v = with_dpp<Op, 0x4E>(v);                               // quad_perm 2,3,0,1
  v = with_dpp<Op, 0x141>(v);                              // row_half_mirror
  if constexpr (TPR > 8) {
    v = with_dpp<Op, 0x140>(v);                            // row_mirror
    const uint32_t a = __builtin_bit_cast(uint32_t, v);
    const auto r = __builtin_amdgcn_permlane16_swap(a, a, false, false);
    v = Op::of(__builtin_bit_cast(V, (uint32_t)r[0]), __builtin_bit_cast(V, (uint32_t)r[1]));
    const uint32_t b = __builtin_bit_cast(uint32_t, v);
    const auto q = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    v = Op::of(__builtin_bit_cast(V, (uint32_t)q[0]), __builtin_bit_cast(V, (uint32_t)q[1]));
  }
  if constexpr (TPR > 64) {                                // the block is one row
    V* const part = (V*)lds;
    __syncthreads();                                       // (of the reduction before)
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int i = 1; i < TPR / 64; ++i) v = Op::of(v, part[i]);
  }
  return v;
}
// Two sums at once.
template <int TPR> __device__ __forceinline__ void row_sums(float& a, float& b, float* lds) {
  a = row_reduce<Sum, TPR < 64 ? TPR : 64>(a, nullptr);
  b = row_reduce<Sum, TPR < 64 ? TPR : 64>(b, nullptr);
  if constexpr (TPR > 64) {
    float2* const part = (float2*)lds;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = make_float2(a, b);
    __syncthreads();
    float2 v = part[0];
#pragma unroll
    for (int i = 1; i < TPR / 64; ++i) { const float2 w = part[i]; v.x += w.x; v.y += w.y; }
    a = v.x; b = v.y;
  }
}

// Mean squares that fp32 does not hold: a sum beyond it, or, where eps does not hide it, so small a mean that squares lost bits.  Those rows' sums are
// made again of their values times 2^shift, and eps times its square: once where they are large, twice where they are smallest.  The other rows' bits
// stay as without this, and their times within 2 % (32 768 x 3200 with its sum and 8 bits 197 us either way, 10 000 x 2048 28.4 and 29.0).  Every
// thread of a row has the same mean, bit by bit, so all go the same way; rows of zeros or with a NaN or an infinity end as they would have.
constexpr float kLeastMean = 7.888609052210118e-31f;      // 2^-100: what is below the last bit of a square, 2^-150, is 2^-50 of it
constexpr int kScalings = 2;
__device__ __forceinline__ bool fp32_holds(float mean) { return mean >= kLeastMean && mean < __builtin_inff(); }
__device__ __forceinline__ int scale_step(float mean) { return mean < 1.f ? 64 : -80; }
// 1 / sqrt(mean) of the row itself, given the mean of the scaled values; beyond fp32 its largest number.
__device__ __forceinline__ float row_rstd(float mean, int shift) {
  const float rstd = 1.0f / sqrtf(mean);
  return shift && mean > 0.f ? fminf(ldexpf(rstd, shift), 3.402823466e38f) : rstd;
}

struct NormArgs {
  const void *x, *r, *gain;          // x or r may be nullptr, and any output
  void *sum, *y;
  int8_t* q;
  float* scale;
  int64_t ld_x, ld_r, ld_sum, ld_y, ld_q;
  int rows, D;
  float eps, inv_d;
};
struct NormGradArgs {
  const void *s, *dy, *ds, *gain;    // ds may be nullptr
  void *dx, *dr;                     // or nullptr
  float* parts;                      // [blocks][D], or nullptr
  int64_t ld_s, ld_dy, ld_ds, ld_dx, ld_dr;
  int rows, D, per;                  // rows of each group of threads
  float eps, inv_d;
};

// Threads per row (a wave: four rows a block; more: the block) and chunks of eight per thread.
template <typename T, typename R, int TPR, int U, bool NORM>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void norm_kernel(NormArgs a) {
  __shared__ uint32_t lds[TPR > 64 ? TPR / 64 : 1];
  constexpr int RPB = TPR < 256 ? 256 / TPR : 1;
  static_assert(TPR == 8 || TPR == 64 || TPR >= 256, "eight lanes, a wave or a block per row");
  const int row = blockIdx.x * RPB + (int)threadIdx.x / TPR, at = (int)threadIdx.x % TPR;
  if (row >= a.rows) return;                               // whole groups of lanes, which only meet each other
  float v[U][8];
  const T* const x = a.x ? (const T*)a.x + (int64_t)row * a.ld_x : nullptr;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int e = (u * TPR + at) * 8, left = a.D - e;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[u][i] = 0.f;
    if (x && left > 0) load8(x + e, left, v[u]);
  }
  if constexpr (NORM) {
    if (a.r) {
      const R* const r = (const R*)a.r + (int64_t)row * a.ld_r;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int e = (u * TPR + at) * 8, left = a.D - e;
        if (left <= 0) continue;
        float w[8];
        load8(r + e, left, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[u][i] += w[i];
      }
    }
    if (a.sum) {
      R* const s = (R*)a.sum + (int64_t)row * a.ld_sum;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int e = (u * TPR + at) * 8, left = a.D - e;
        if (left > 0) store8(s + e, left, v[u]);
      }
    }
    if (!a.y && !a.q) return;
    float ss = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = fmaf(v[u][i], v[u][i], ss);
    ss = row_reduce<Sum, TPR>(ss, lds);
    float mean = fmaf(ss, a.inv_d, a.eps);
    int shift = 0;
    for (int j = 0; j < kScalings && __builtin_expect(!fp32_holds(mean), 0); ++j) {
      shift += scale_step(mean);
      ss = 0.f;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < 8; ++i) { const float w = ldexpf(v[u][i], shift); ss = fmaf(w, w, ss); }
      mean = fmaf(row_reduce<Sum, TPR>(ss, lds), a.inv_d, ldexpf(a.eps, 2 * shift));
    }
    const float rstd = row_rstd(mean, shift);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int e = (u * TPR + at) * 8, left = a.D - e;
      if (left <= 0) continue;
      float g[8];
      load8((const T*)a.gain + e, left, g);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[u][i] = v[u][i] * rstd * g[i];
    }
    if (a.y) {
      T* const y = (T*)a.y + (int64_t)row * a.ld_y;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int e = (u * TPR + at) * 8, left = a.D - e;
        if (left > 0) store8(y + e, left, v[u]);
      }
    }
    if (!a.q) return;
  }
  // magnitudes as bit patterns: a NaN lies above infinity, infinity above every number
  uint32_t most = 0;
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int i = 0; i < 8; ++i) most = Most::of(most, __float_as_uint(v[u][i]) & 0x7fffffffu);
  most = row_reduce<Most, TPR>(most, lds);
  const bool finite = most < 0x7f800000u;
  const float m = fmaxf(__uint_as_float(most), kLeastMax), to_q = 127.0f / m;
  if (at == 0) a.scale[row] = finite ? m * (1.0f / 127.0f) : __uint_as_float(0x7fc00000u);
  int8_t* const q = a.q + (int64_t)row * a.ld_q;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int e = (u * TPR + at) * 8, left = a.D - e;
    if (left <= 0) continue;
    if (!finite) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[u][i] = 0.f;
    }
    store_q8(q + e, left, v[u], to_q);
  }
}

// Rows [group * per, ...) of a group of TPR threads, whose sums of dy * n stay in registers; those of a block's groups meet in LDS,
// in the order of the groups, and the blocks' in gain_kernel.
template <typename T, typename R, int TPR, int U>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void norm_grad_kernel(NormGradArgs a) {
  constexpr int RPB = TPR < 256 ? 256 / TPR : 1;
  __shared__ float lds[RPB > 1 ? (RPB - 1) * U * TPR * 8 : 2 * TPR / 64];
  const int group = (int)threadIdx.x / TPR, at = (int)threadIdx.x % TPR;
  const int64_t r0 = ((int64_t)blockIdx.x * RPB + group) * a.per;
  const int r1 = (int)min(r0 + a.per, (int64_t)a.rows);
  float sums[U][8];
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int i = 0; i < 8; ++i) sums[u][i] = 0.f;
  // AHEAD: the next row's loads go out before this row's sums (bf16, 30 000 x 1024 51 us, without 68; 10 000 x 2048 36 and 43; 16 384 x 3200 106
  // and 134), where registers allow: 6000 x 8000 in two chunks of 512 threads 98, without 89.
  // AGAIN: rows of four chunks a thread and more are read again for the results, out of the caches, as floats of all would not stay in registers (3000
  // x 30 000 201 us, spilled 318; 1500 x 65 536 with an fp32 residual 425 and 1136).  Of eight chunks a thread 12 to 18 registers still spill.
  constexpr bool AHEAD = U == 1 || (U == 2 && TPR < 512), AGAIN = U >= 4;
  struct Raw {
    typename raw8_of<R>::type s, o;
    typename raw8_of<T>::type d;
  } next[AHEAD ? U : 1];
  auto fetch = [&](int64_t row, int u, Raw& to) {
    const int e = (u * TPR + at) * 8, left = a.D - e;
    if (left <= 0) return;
    load_raw8((const R*)a.s + row * a.ld_s + e, left, to.s);
    load_raw8((const T*)a.dy + row * a.ld_dy + e, left, to.d);
    if (a.ds) load_raw8((const R*)a.ds + row * a.ld_ds + e, left, to.o);
  };
  if constexpr (AHEAD) {
#pragma unroll
    for (int u = 0; u < U; ++u) if (r0 < r1) fetch(r0, u, next[u]);
  }
  for (int64_t row = r0; row < r1; ++row) {
    float s[AGAIN ? 1 : U][8], d[AGAIN ? 1 : U][8], o[AGAIN ? 1 : U][8];
    float ss = 0.f, gn = 0.f;
    auto held = [&](int u) {                               // chunk u as floats
      const int k = AGAIN ? 0 : u;
#pragma unroll
      for (int i = 0; i < 8; ++i) s[k][i] = d[k][i] = o[k][i] = 0.f;
      if (a.D <= (u * TPR + at) * 8) return;
      Raw now;
      if constexpr (AHEAD) now = next[u]; else fetch(row, u, now);
      from_raw8(now.s, s[k]);
      from_raw8(now.d, d[k]);
      if (a.ds) from_raw8(now.o, o[k]);
    };
    if constexpr (!AGAIN) {
#pragma unroll
      for (int u = 0; u < U; ++u) held(u);
    }
    if constexpr (AHEAD) {
#pragma unroll
      for (int u = 0; u < U; ++u) if (row + 1 < r1) fetch(row + 1, u, next[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int e = (u * TPR + at) * 8, left = a.D - e, k = AGAIN ? 0 : u;
      if constexpr (AGAIN) held(u);
      if (left <= 0) continue;
      float g[8];
      load8((const T*)a.gain + e, left, g);
#pragma unroll
      for (int i = 0; i < 8; ++i) { ss = fmaf(s[k][i], s[k][i], ss); gn = fmaf(d[k][i] * g[i], s[k][i], gn); }
    }
    row_sums<TPR>(ss, gn, lds);
    float var = fmaf(ss, a.inv_d, a.eps);
    int shift = 0;
    for (int j = 0; j < kScalings && __builtin_expect(!fp32_holds(var), 0); ++j) {
      shift += scale_step(var);
      ss = gn = 0.f;
#pragma unroll(AGAIN ? 1 : U)
      for (int u = 0; u < U; ++u) {
        const int e = (u * TPR + at) * 8, left = a.D - e, k = AGAIN ? 0 : u;
        if constexpr (AGAIN) held(u);
        if (left <= 0) continue;
        float g[8];
        load8((const T*)a.gain + e, left, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) { const float v = ldexpf(s[k][i], shift); ss = fmaf(v, v, ss); gn = fmaf(d[k][i] * g[i], v, gn); }
      }
      row_sums<TPR>(ss, gn, lds);
      var = fmaf(ss, a.inv_d, ldexpf(a.eps, 2 * shift));
    }
    const float rstd = row_rstd(var, shift);
    const float mean = gn * (1.0f / sqrtf(var)) * a.inv_d; // of g n
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int e = (u * TPR + at) * 8, left = a.D - e, k = AGAIN ? 0 : u;
      if constexpr (AGAIN) held(u);
      if (left <= 0) continue;
      float g[8];
      load8((const T*)a.gain + e, left, g);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float n = s[k][i] * rstd;
        sums[u][i] = fmaf(d[k][i], n, sums[u][i]);
        o[k][i] = fmaf(rstd, fmaf(-n, mean, d[k][i] * g[i]), o[k][i]);
      }
      if (a.dx) store8((T*)a.dx + row * a.ld_dx + e, left, o[k]);
      if (a.dr) store8((R*)a.dr + row * a.ld_dr + e, left, o[k]);
    }
  }
  if (!a.parts) return;
  if constexpr (RPB > 1) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < 8; ++i) if (group) lds[((group - 1) * U * 8 + u * 8 + i) * TPR + at] = sums[u][i];
    __syncthreads();
    if (group) return;
#pragma unroll
    for (int g = 1; g < RPB; ++g)
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < 8; ++i) sums[u][i] += lds[((g - 1) * U * 8 + u * 8 + i) * TPR + at];
  }
  float* const to = a.parts + (int64_t)blockIdx.x * a.D;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int e = (u * TPR + at) * 8, left = a.D - e;
    if (left > 0) store8(to + e, left, sums[u]);
  }
}

// gain's gradient: the sums of the blocks, 32 columns (whole lines of memory) a block of 32 groups, in fixed orders: 512 blocks of 8000 columns
// 5.0 us, by 16 columns 9.0; 784 of 1024 4.0 either way, the time to launch and read once.
struct GainArgs { const float* parts; void* out; int n, D; };
constexpr int kGainCols = 32;
template <typename T> __global__ __launch_bounds__(1024) void gain_kernel(GainArgs a) {
  constexpr int G = 1024 / kGainCols;
  __shared__ float part[G][kGainCols];
  const int l = threadIdx.x % kGainCols, c = blockIdx.x * kGainCols + l, g = threadIdx.x / kGainCols;
  float v = 0.f;
  if (c < a.D) {
#pragma unroll 4
    for (int p = g; p < a.n; p += G) v += a.parts[(int64_t)p * a.D + c];
  }
  part[g][l] = v;
  for (int n = G / 2; n > 0; n >>= 1) {
    __syncthreads();
    if (g < n) part[g][l] += part[g + n][l];
  }
  if (g == 0 && c < a.D) ((T*)a.out)[c] = (T)part[0][l];
}

// values = q * scale.  Bound: HBM; 32 768 x 3200 into bf16 53 us, 6.0 TB/s; 12 800 x 3200 19.2 (20.8 without writing through).
struct DequantArgs { const int8_t* q; const float* scale; void* out; int64_t ld_q, ld_out; int rows, D; bool through; };
template <typename T> __global__ __launch_bounds__(256) void dequant_kernel(DequantArgs a) {
  const int chunks = (a.D + 7) / 8;
  const int64_t all = (int64_t)a.rows * chunks;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / chunks;
    const int e = (int)(i - row * chunks) * 8, left = a.D - e;
    const int8_t* const q = a.q + row * a.ld_q + e;
    const float s = a.scale[row];
    float v[8];
    if (left >= 8) {
      const pair1 u = *(const pair1*)q;
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = (float)(int8_t)(u[j / 4] >> (8 * (j & 3))) * s;
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = j < left ? (float)q[j] * s : 0.f;
    }
    store8((T*)a.out + row * a.ld_out + e, left, v, a.through);
  }
}

// f(threads per row, chunks per thread) as integral constants.  Few chunks a thread keep more rows in flight: 32 768 x 3200 with its sum and
// 8 bits 210 us by 512 threads of one chunk, 221 by 256 of two, 243 by a wave of seven; 6000 x 8192 bf16 forward 74 by 512 of two, 79 by 256 of
// four; backward (measured without loads ahead) 10 000 x 2048 42 us by 256 of one, 67 by a wave of four, but 6272 x 1024 13.9 by a wave of two, 18.8
// by 256 of one; with them 6000 x 8000 89 by 512 of two, 96 by 1024 of one.  Rows that are only rounded (NORM = false) have half the loads: 12 800 x
// 3200 24.3 us by 256 of two, 29.6 by 512 of one, 32 768 x 1152 28.1 by a wave of three, 33.0 by 256 of one.  (Fewer blocks that load the next
// row ahead are no faster: 24.8 and 32.1.)
template <bool NORM, class F> hipError_t by_width(int D, F&& f) {
  using std::integral_constant;
#define EPD_WIDTH(tpr, u) return f(integral_constant<int, tpr>{}, integral_constant<int, u>{})
  if (D <= 64) EPD_WIDTH(8, 1);
  if (D <= 512) EPD_WIDTH(64, 1);
  if (D <= 1024) EPD_WIDTH(64, 2);
  if constexpr (!NORM) { if (D <= 1536) EPD_WIDTH(64, 3); }
  if (D <= 2048) EPD_WIDTH(256, 1);
  if constexpr (NORM) { if (D <= 4096) EPD_WIDTH(512, 1); }
  else if (D <= 4096) EPD_WIDTH(256, 2);
  if (D <= 8192) EPD_WIDTH(512, 2);
  if (D <= 16384) EPD_WIDTH(1024, 2);
  if (D <= 32768) EPD_WIDTH(1024, 4);
  EPD_WIDTH(1024, 8);
#undef EPD_WIDTH
}

template <typename T, typename R, bool NORM> hipError_t launch_norm_rows(const NormArgs& all, hipStream_t s) {
  return by_width<NORM>(all.D, [&](auto TPR, auto U) {
    constexpr int tpr = decltype(TPR)::value, rpb = tpr < 256 ? 256 / tpr : 1;
    constexpr int64_t most = (int64_t)kMaxGrid * rpb / (tpr > 512 ? 2 : 1);      // rows of a launch
    for (int64_t r = 0; r < all.rows; r += most) {
      NormArgs a = all;
      a.rows = (int)std::min<int64_t>(all.rows - r, most);
      if (a.x) a.x = (const T*)a.x + r * a.ld_x;
      if (a.r) a.r = (const R*)a.r + r * a.ld_r;
      if (a.sum) a.sum = (R*)a.sum + r * a.ld_sum;
      if (a.y) a.y = (T*)a.y + r * a.ld_y;
      if (a.q) { a.q += r * a.ld_q; a.scale += r; }
      void* args[] = {(void*)&a};
      if (hipError_t e = hipLaunchKernel((const void*)norm_kernel<T, R, tpr, decltype(U)::value, NORM>, dim3((a.rows + rpb - 1) / rpb), dim3(tpr < 256 ? 256 : tpr), args, 0, s)) return e;
    }
    return hipSuccess;
  });
}

// Blocks of the backward pass: the chip filled, then more rows for each group of threads, whose sums it keeps.  As many as stay resident (16 384 x
// 3200 with 512 blocks 102 us and 4.8 for gain's kernel, with 1024 106 and 6.2; 20 000 x 400 with 1024 26.8, with 512 32.2; 1500 x 65 536, whose
// blocks fill a unit each, with 256 422 and 28, with 512 436 and 53).
int grad_rows_per_block(int D) { return D <= 64 ? 32 : D <= 1024 ? 4 : 1; }      // as by_width has it
int grad_most_blocks(int D) { return D > 8192 ? 256 : D > 2048 ? 512 : 1024; }
int grad_rows(int rows, int D) {         // of a group
  const int64_t groups = (int64_t)grad_most_blocks(D) * grad_rows_per_block(D);
  return (int)((rows + groups - 1) / groups);
}
int grad_blocks(int rows, int D) {
  const int64_t per = (int64_t)grad_rows(rows, D) * grad_rows_per_block(D);
  return (int)((rows + per - 1) / per);
}

template <typename T, typename R> hipError_t launch_norm_grad(NormGradArgs a, void* dgain, hipStream_t s) {
  const int blocks = grad_blocks(a.rows, a.D);
  a.per = grad_rows(a.rows, a.D);
  void* args[] = {(void*)&a};
  hipError_t e = by_width<true>(a.D, [&](auto TPR, auto U) {
    constexpr int tpr = decltype(TPR)::value;
    return hipLaunchKernel((const void*)norm_grad_kernel<T, R, tpr, decltype(U)::value>, dim3(blocks), dim3(tpr < 256 ? 256 : tpr), args, 0, s);
  });
  if (e != hipSuccess || !dgain) return e;
  GainArgs g{a.parts, dgain, blocks, a.D};
  void* gargs[] = {(void*)&g};
  return hipLaunchKernel((const void*)gain_kernel<T>, dim3((a.D + kGainCols - 1) / kGainCols), dim3(1024), gargs, 0, s);
}

epd_status check_cfg(const char* who, const epd_add_norm_cfg* c) {
  if (!c) return op_fail(EPD_ERR_INVALID_ARG, "%s: cfg is NULL", who);
  if (c->struct_size != sizeof(epd_add_norm_cfg)) return op_fail(EPD_ERR_INVALID_ARG, "%s: cfg.struct_size %u != %zu", who, c->struct_size, sizeof(epd_add_norm_cfg));
  if (!known_dtype(c->dtype) || !known_dtype(c->residual_dtype)) return op_fail(EPD_ERR_INVALID_ARG, "%s: dtype or residual_dtype invalid", who);
  if (c->dtype == EPD_F32 && c->residual_dtype != EPD_F32) return op_fail(EPD_ERR_UNSUPPORTED, "%s: an fp32 norm has an fp32 residual stream", who);
  if (c->hidden < 1 || c->hidden > kNormDim) return op_fail(EPD_ERR_UNSUPPORTED, "%s: hidden %d: 1 .. %d", who, c->hidden, kNormDim);
  if (c->max_tokens < 1) return op_fail(EPD_ERR_INVALID_ARG, "%s: max_tokens %d", who, c->max_tokens);
  if (!(c->eps >= 0.f) || !std::isfinite(c->eps)) return op_fail(EPD_ERR_INVALID_ARG, "%s: eps must be finite and not negative", who);
  return EPD_OK;
}

uint64_t workspace_bytes(const epd_add_norm_cfg& c) {
  // (fewer tokens may take as many blocks)
  const int64_t per = grad_rows_per_block(c.hidden), blocks = std::min<int64_t>(grad_most_blocks(c.hidden), (c.max_tokens + per - 1) / per);
  return ((uint64_t)blocks * c.hidden * 4 + 255) / 256 * 256;
}

template <class F> hipError_t by_types(const epd_add_norm_cfg& c, F&& f) {
  if (c.dtype == EPD_F32) return f(0.f, 0.f);
  return c.residual_dtype == EPD_F32 ? f((__bf16)0.f, 0.f) : f((__bf16)0.f, (__bf16)0.f);
}

}  // namespace
}  // namespace epd

using namespace epd;

extern "C" {

uint64_t epd_add_norm_workspace_bytes(const epd_add_norm_cfg* cfg) {
  if (check_cfg("epd_add_norm_workspace_bytes", cfg) != EPD_OK) return 0;
  return workspace_bytes(*cfg);
}

epd_status epd_add_norm(const epd_add_norm_cfg* cfg, const epd_add_norm_rows* rows, const void* gain, int32_t tokens, void* stream) {
  const char* const who = "epd_add_norm";
  if (epd_status s = check_cfg(who, cfg)) return s;
  if (!rows) return op_fail(EPD_ERR_INVALID_ARG, "%s: rows is NULL", who);
  if (tokens < 0 || tokens > cfg->max_tokens) return op_fail(EPD_ERR_SHAPE, "%s: tokens %d: 0 .. max_tokens %d", who, tokens, cfg->max_tokens);
  const int D = cfg->hidden, es = cfg->dtype == EPD_F32 ? 4 : 2, rs = cfg->residual_dtype == EPD_F32 ? 4 : 2;
  if (!rows->x && !rows->residual && tokens) return op_fail(EPD_ERR_INVALID_ARG, "%s: neither x nor residual", who);
  if (!rows->sum && !rows->y && !rows->q) return op_fail(EPD_ERR_INVALID_ARG, "%s: no output", who);
  epd_add_norm_rows r = *rows;
  if (tokens == 0) return EPD_OK;
  if (r.x) if (epd_status s = check_rows(who, "x", r.x, r.ld_x, tokens, D, es)) return s;
  if (r.residual) if (epd_status s = check_rows(who, "residual", r.residual, r.ld_residual, tokens, D, rs)) return s;
  if (r.sum) if (epd_status s = check_rows(who, "sum", r.sum, r.ld_sum, tokens, D, rs)) return s;
  if (r.y) if (epd_status s = check_rows(who, "y", r.y, r.ld_y, tokens, D, es)) return s;
  if (r.q) if (epd_status s = check_rows(who, "q", r.q, r.ld_q, tokens, D, 1)) return s;
  if (r.q && (!r.scale || (uintptr_t)r.scale % 4)) return op_fail(EPD_ERR_INVALID_ARG, "%s: q without a scale, or it is not aligned", who);
  if ((r.y || r.q) && (!gain || (uintptr_t)gain % es)) return op_fail(EPD_ERR_INVALID_ARG, "%s: gain is NULL or not aligned to its elements", who);
  if (r.sum && r.sum == r.residual && r.ld_sum != r.ld_residual) return op_fail(EPD_ERR_SHAPE, "%s: sum in place of residual, the rows must be as far apart", who);
  if (r.y && r.y == r.x && r.ld_y != r.ld_x) return op_fail(EPD_ERR_SHAPE, "%s: y in place of x, the rows must be as far apart", who);
  const NormArgs a{r.x, r.residual, gain, r.sum, r.y, (int8_t*)r.q, r.scale, r.ld_x, r.ld_residual, r.ld_sum, r.ld_y, r.ld_q, tokens, D, cfg->eps, 1.0f / (float)D};
  const hipError_t e = by_types(*cfg, [&](auto t, auto u) { return launch_norm_rows<decltype(t), decltype(u), true>(a, (hipStream_t)stream); });
  return e == hipSuccess ? EPD_OK : op_launch_failed(who, e);
}

epd_status epd_add_norm_backward(const epd_add_norm_cfg* cfg, const epd_add_norm_grads* grads, const void* gain, int32_t tokens, void* workspace,
                                 uint64_t bytes, void* stream) {
  const char* const who = "epd_add_norm_backward";
  if (epd_status s = check_cfg(who, cfg)) return s;
  if (!grads) return op_fail(EPD_ERR_INVALID_ARG, "%s: grads is NULL", who);
  if (tokens < 0 || tokens > cfg->max_tokens) return op_fail(EPD_ERR_SHAPE, "%s: tokens %d: 0 .. max_tokens %d", who, tokens, cfg->max_tokens);
  const int D = cfg->hidden, es = cfg->dtype == EPD_F32 ? 4 : 2, rs = cfg->residual_dtype == EPD_F32 ? 4 : 2;
  epd_add_norm_grads g = *grads;
  if ((uintptr_t)g.gain % es) return op_fail(EPD_ERR_INVALID_ARG, "%s: the gradient of gain is not aligned to its elements", who);
  if (g.gain) {
    if (!workspace || (uintptr_t)workspace % 256) return op_fail(EPD_ERR_WORKSPACE, "%s: workspace is NULL or not 256-byte aligned", who);
    if (bytes < workspace_bytes(*cfg)) return op_fail(EPD_ERR_WORKSPACE, "%s: workspace_bytes %llu < required %llu", who, (unsigned long long)bytes, (unsigned long long)workspace_bytes(*cfg));
  }
  hipError_t e = hipSuccess;
  if (tokens == 0) {                     // a sum over no rows
    if (!g.gain) return EPD_OK;
    GainArgs a{(const float*)workspace, g.gain, 0, D};
    void* args[] = {(void*)&a};
    e = hipLaunchKernel(es == 4 ? (const void*)gain_kernel<float> : (const void*)gain_kernel<__bf16>, dim3((D + kGainCols - 1) / kGainCols), dim3(1024), args, 0, (hipStream_t)stream);
    return e == hipSuccess ? EPD_OK : op_launch_failed(who, e);
  }
  if (epd_status s = check_rows(who, "sum", g.sum, g.ld_sum, tokens, D, rs)) return s;
  if (epd_status s = check_rows(who, "dy", g.dy, g.ld_dy, tokens, D, es)) return s;
  if (g.dsum) if (epd_status s = check_rows(who, "dsum", g.dsum, g.ld_dsum, tokens, D, rs)) return s;
  if (g.dx) if (epd_status s = check_rows(who, "dx", g.dx, g.ld_dx, tokens, D, es)) return s;
  if (g.dresidual) if (epd_status s = check_rows(who, "dresidual", g.dresidual, g.ld_dresidual, tokens, D, rs)) return s;
  if (!gain || (uintptr_t)gain % es) return op_fail(EPD_ERR_INVALID_ARG, "%s: gain is NULL or not aligned to its elements", who);
  if (g.dx && g.dx == g.dy && g.ld_dx != g.ld_dy) return op_fail(EPD_ERR_SHAPE, "%s: dx in place of dy, the rows must be as far apart", who);
  if (g.dresidual && g.dresidual == g.dsum && g.ld_dresidual != g.ld_dsum) return op_fail(EPD_ERR_SHAPE, "%s: dresidual in place of dsum, the rows must be as far apart", who);
  if (!g.dx && !g.dresidual && !g.gain) return EPD_OK;
  const NormGradArgs a{g.sum, g.dy, g.dsum, gain, g.dx, g.dresidual, g.gain ? (float*)workspace : nullptr, g.ld_sum, g.ld_dy, g.ld_dsum, g.ld_dx, g.ld_dresidual,
                       tokens, D, 0, cfg->eps, 1.0f / (float)D};
  e = by_types(*cfg, [&](auto t, auto u) { return launch_norm_grad<decltype(t), decltype(u)>(a, g.gain, (hipStream_t)stream); });
  return e == hipSuccess ? EPD_OK : op_launch_failed(who, e);
}

epd_status epd_quant_rows(int32_t dtype, const void* x, int64_t ld_x, int32_t rows, int32_t cols, void* q, int64_t ld_q, float* scale, void* stream) {
  const char* const who = "epd_quant_rows";
  if (!known_dtype(dtype)) return op_fail(EPD_ERR_INVALID_ARG, "%s: dtype %d", who, dtype);
  if (rows < 0) return op_fail(EPD_ERR_SHAPE, "%s: rows %d", who, rows);
  if (cols < 1 || cols > kNormDim) return op_fail(EPD_ERR_UNSUPPORTED, "%s: cols %d: 1 .. %d", who, cols, kNormDim);
  if (rows == 0) return EPD_OK;
  if (epd_status s = check_rows(who, "x", x, ld_x, rows, cols, dtype == EPD_F32 ? 4 : 2)) return s;
  if (epd_status s = check_rows(who, "q", q, ld_q, rows, cols, 1)) return s;
  if (!scale || (uintptr_t)scale % 4) return op_fail(EPD_ERR_INVALID_ARG, "%s: scale is NULL or not aligned", who);
  NormArgs a{};
  a.x = x; a.q = (int8_t*)q; a.scale = scale; a.ld_x = ld_x; a.ld_q = ld_q; a.rows = rows; a.D = cols;
  const hipError_t e = dtype == EPD_F32 ? launch_norm_rows<float, float, false>(a, (hipStream_t)stream) : launch_norm_rows<__bf16, __bf16, false>(a, (hipStream_t)stream);
  return e == hipSuccess ? EPD_OK : op_launch_failed(who, e);
}

epd_status epd_dequant_rows(const void* q, int64_t ld_q, const float* scale, int32_t rows, int32_t cols, int32_t dtype, void* out, int64_t ld_out, void* stream) {
  const char* const who = "epd_dequant_rows";
  if (!known_dtype(dtype)) return op_fail(EPD_ERR_INVALID_ARG, "%s: dtype %d", who, dtype);
  if (rows < 0) return op_fail(EPD_ERR_SHAPE, "%s: rows %d", who, rows);
  if (cols < 1 || cols > kNormDim) return op_fail(EPD_ERR_UNSUPPORTED, "%s: cols %d: 1 .. %d", who, cols, kNormDim);
  if (rows == 0) return EPD_OK;
  if (epd_status s = check_rows(who, "q", q, ld_q, rows, cols, 1)) return s;
  if (epd_status s = check_rows(who, "out", out, ld_out, rows, cols, dtype == EPD_F32 ? 4 : 2)) return s;
  if (!scale || (uintptr_t)scale % 4) return op_fail(EPD_ERR_INVALID_ARG, "%s: scale is NULL or not aligned", who);
  DequantArgs a{(const int8_t*)q, scale, out, ld_q, ld_out, rows, cols, writes_through(out, ld_out, dtype == EPD_F32 ? 4 : 2)};
  const int64_t threads = (int64_t)rows * ((cols + 7) / 8);
  void* args[] = {(void*)&a};
  const hipError_t e = hipLaunchKernel(dtype == EPD_F32 ? (const void*)dequant_kernel<float> : (const void*)dequant_kernel<__bf16>,
                                       dim3((int)std::min<int64_t>((threads + 255) / 256, 65536)), dim3(256), args, 0, (hipStream_t)stream);
  return e == hipSuccess ? EPD_OK : op_launch_failed(who, e);
}

}  // extern "C"
