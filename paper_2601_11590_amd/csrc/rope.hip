// Rotary positions with several axes, as operators of their own: rotation of q / k rows by positions
// that the caller gives (the encoder's rotary table only knows raster grids), its inverse, which is also its
// gradient, and the (t, h, w) positions of sequences of text and visual tokens: what the
// consumer of V_m = E(I_m) computes on V_m || V_t next (paper section 3.1, Eq. 1 and 2).
//
// Rotation.  Pair p = (x, y) of a head at position pos[axis(p)] turns by a = pos * f_p:
//   (x, y) -> (x cos a - y sin a, x sin a + y cos a);   the inverse turns by -a.
// Bound: HBM, every value is read and written once.  So that the angles cost nothing beside that, a block
// first makes the cos / sin of its few tokens' pairs in LDS, one each, and then turns all heads of all
// tensors with them, 16 bytes per access where rows allow.  (They are made again in every call: at 50 heads
// of 128 a table in memory would save one double multiplication and a dozen fp32 ones per 100 values.)
//
// Angles.  In turns, r = pos * (f_p / 2 pi) in fp64, so that an int32 position far into a long context
// keeps its phase (f_p, its quotient and the product are off by 2^-52 together or so, and 2^31 positions at f_p = 1 are 3.4e8
// turns: 1e-7 of a turn; 4e-11 within a million tokens).  The quarter
// turns are taken off in fp64; what is left, |x| <= pi / 4, goes through the Taylor sums of sine and
// cosine in fp32 (next terms 1.8e-9 and 1.2e-10, below half a step of fp32).
#include "op_error.h"

#include <algorithm>
#include <climits>
#include <cmath>

namespace epd {

constexpr int kRopePairs = 128;      // rotary pairs of a head
constexpr int kRopeTensors = 4;      // tensors per call (q and k, or their gradients)
constexpr int kRopeHeads = 256;      // heads of one tensor: a token's chunks stay below 65536

struct RopeTensor {
  const void* in;
  void* out;
  int64_t in_token, in_head, out_token, out_head;   // strides, elements
  int32_t heads;
  int32_t per_token;                 // chunks per token: heads * chunks
  uint32_t inv_per_token, inv_chunks;                // ceil(2^32 / .): quotients of numbers below 65536
  int32_t chunks;                    // of a head: turned, then copied
};

struct RopeArgs {
  RopeTensor t[kRopeTensors];
  const int32_t* positions;
  int64_t pos_stride;
  int32_t n, tokens, pairs, turned;  // tensors; tokens; pairs per head; chunks of a head that are turned
  int32_t block_tokens, inverse;
  uint32_t inv_pairs;
  double turns[kRopePairs];          // f_p / 2 pi
  uint8_t axis[kRopePairs];
};

template <typename T, int N> struct alignas(sizeof(T) * N) Pack { T v[N]; };

// x / d for x, d < 65536, inv = ceil(2^32 / d) (d = 1: inv wraps to 0)
__device__ __forceinline__ uint32_t quotient(uint32_t x, uint32_t inv) { return inv ? __umulhi(x, inv) : x; }

__device__ __forceinline__ float2 turn_cos_sin(double r) {
  const double q = rint(4.0 * r);
  const float x = (float)((r - 0.25 * q) * 6.283185307179586476925);
  const float z = x * x;
  float s = fmaf(z, 2.7557319224e-6f, -1.9841269841e-4f), c = fmaf(z, -2.7557319224e-7f, 2.4801587302e-5f);
  s = fmaf(z, s, 8.3333333333e-3f); c = fmaf(z, c, -1.3888888889e-3f);
  s = fmaf(z, s, -1.6666666667e-1f); c = fmaf(z, c, 4.1666666667e-2f);
  s = fmaf(x * z, s, x); c = fmaf(z * z, c, fmaf(z, -0.5f, 1.0f));
  const int k = (int)((long long)q & 3);           // quarter turns
  const float a = k & 1 ? s : c, b = k & 1 ? c : s;
  return make_float2((k == 1 || k == 2) ? -a : a, k >= 2 ? -b : b);
}

// VEC elements per access.  ADJACENT: pair p = elements (2p, 2p + 1) of a head; otherwise (p, p + pairs).
// A chunk is VEC pairs (halves), VEC / 2 (adjacent; 1 where VEC = 1), or VEC elements that are copied.
template <typename T, int VEC, bool ADJACENT>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
  constexpr int NP = ADJACENT ? (VEC > 1 ? VEC / 2 : 1) : VEC;
  __shared__ float2 table[256];                    // [token of the block][pair]: block_tokens * pairs <= 256
  const int tid = threadIdx.x;
  const int tok0 = blockIdx.x * a.block_tokens, toks = min(a.block_tokens, a.tokens - tok0);
  if (tid < toks * a.pairs) {
    const int t = quotient(tid, a.inv_pairs), p = tid - t * a.pairs;
    const int pos = a.positions[(int64_t)a.axis[p] * a.pos_stride + tok0 + t];
    float2 cs = turn_cos_sin((double)pos * a.turns[p]);
    if (a.inverse) cs.y = -cs.y;
    table[tid] = cs;
  }
  __syncthreads();
  for (int n = 0; n < a.n; ++n) {
    const RopeTensor& x = a.t[n];
    const int all = toks * x.per_token;
    for (int i = blockIdx.y * 256 + tid; i < all; i += 256 * gridDim.y) {
      const int t = quotient(i, x.inv_per_token), r = i - t * x.per_token;
      const int h = quotient(r, x.inv_chunks), c = r - h * x.chunks;
      const T* const in = (const T*)x.in + (int64_t)(tok0 + t) * x.in_token + (int64_t)h * x.in_head;
      T* const out = (T*)x.out + (int64_t)(tok0 + t) * x.out_token + (int64_t)h * x.out_head;
      if (c >= a.turned) {                         // elements beyond the pairs (only where out is not in)
        const int e = 2 * a.pairs + (c - a.turned) * VEC;
        *(Pack<T, VEC>*)(out + e) = *(const Pack<T, VEC>*)(in + e);
        continue;
      }
      const float2* const cs = table + t * a.pairs + c * NP;
      if constexpr (ADJACENT && VEC > 1) {
        Pack<T, VEC> v = *(const Pack<T, VEC>*)(in + c * VEC);
#pragma unroll
        for (int j = 0; j < NP; ++j) {
          const float u = (float)v.v[2 * j], w = (float)v.v[2 * j + 1];
          v.v[2 * j] = (T)fmaf(u, cs[j].x, -w * cs[j].y);
          v.v[2 * j + 1] = (T)fmaf(u, cs[j].y, w * cs[j].x);
        }
        *(Pack<T, VEC>*)(out + c * VEC) = v;
      } else {
        const int lo = ADJACENT ? 2 * c : c * VEC, hi = ADJACENT ? 2 * c + 1 : a.pairs + c * VEC;
        Pack<T, VEC> v = *(const Pack<T, VEC>*)(in + lo), w = *(const Pack<T, VEC>*)(in + hi);
#pragma unroll
        for (int j = 0; j < NP; ++j) {
          const float x0 = (float)v.v[j], y0 = (float)w.v[j];
          v.v[j] = (T)fmaf(x0, cs[j].x, -y0 * cs[j].y);
          w.v[j] = (T)fmaf(x0, cs[j].y, y0 * cs[j].x);
        }
        *(Pack<T, VEC>*)(out + lo) = v;
        *(Pack<T, VEC>*)(out + hi) = w;
      }
    }
  }
}

template <typename T, int VEC> static hipError_t launch_rope_vec(const RopeArgs& a, bool adjacent, dim3 grid, hipStream_t s) {
  void* args[] = {(void*)&a};
  return hipLaunchKernel(adjacent ? (const void*)rope_kernel<T, VEC, true> : (const void*)rope_kernel<T, VEC, false>, grid, dim3(256), args, 0, s);
}

static hipError_t launch_rope(const RopeArgs& a, bool bf16, int vec, bool adjacent, dim3 grid, hipStream_t s) {
  if (bf16) {
    switch (vec) {
      case 8: return launch_rope_vec<__bf16, 8>(a, adjacent, grid, s);
      case 4: return launch_rope_vec<__bf16, 4>(a, adjacent, grid, s);
      case 2: return launch_rope_vec<__bf16, 2>(a, adjacent, grid, s);
      default: return launch_rope_vec<__bf16, 1>(a, adjacent, grid, s);
    }
  }
  switch (vec) {
    case 4: return launch_rope_vec<float, 4>(a, adjacent, grid, s);
    case 2: return launch_rope_vec<float, 2>(a, adjacent, grid, s);
    default: return launch_rope_vec<float, 1>(a, adjacent, grid, s);
  }
}

// ------------------------------------------------------------------------------ positions
constexpr int kPosSpans = 240;       // spans per launch: they travel as kernel arguments, which end at 4 KB
struct PosSpan { int32_t tok, pos, h, w; };        // first token (of the launch), its position; h = 0: text
struct PosArgs {
  int32_t* out;                      // [3, stride], from the first token of the launch on
  int64_t stride;
  int32_t n, tokens, t_step, pad;
  PosSpan span[kPosSpans];
};
static_assert(sizeof(PosArgs) <= 4096 && sizeof(RopeArgs) <= 4096, "kernel arguments");

// A thread per token, which finds its span by bisection in LDS.  Bound: latency; 12 bytes a token.
__global__ __launch_bounds__(256) void rope_positions_kernel(PosArgs a) {
  __shared__ PosSpan span[kPosSpans];
  for (int i = threadIdx.x; i < a.n; i += 256) span[i] = a.span[i];
  __syncthreads();
  const int tok = blockIdx.x * 256 + threadIdx.x;
  if (tok >= a.tokens) return;
  int lo = 0, hi = a.n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (span[mid].tok <= tok) lo = mid; else hi = mid;
  }
  const PosSpan s = span[lo];
  const int i = tok - s.tok;
  int t = i, r = i, c = i;
  if (s.h > 0) {
    const int hw = s.h * s.w, in_frame = i % hw;
    t = i / hw * a.t_step; r = in_frame / s.w; c = in_frame - r * s.w;
  }
  a.out[tok] = s.pos + t;
  a.out[a.stride + tok] = s.pos + r;
  a.out[2 * a.stride + tok] = s.pos + c;
}

// Tokens of a span: -1 where its sizes are inconsistent, -2 where they pass 2^31 - 1.
static int64_t span_tokens(const int32_t* thw) {
  const int64_t t = thw[0], h = thw[1], w = thw[2];
  if (h == 0 && w == 0) return t < 0 ? -1 : t;
  if (t <= 0 || h <= 0 || w <= 0) return -1;
  return h * w > INT_MAX || t * (h * w) > INT_MAX ? -2 : t * h * w;
}

// Axis and turns per position of every pair.  A pure function of the configuration, which a program keeps from call to
// call: the last table of the thread is kept with it (64 powers are 2.5 us of a call for one token).
static void pair_table(const epd_rope_cfg& c, int pairs, RopeArgs& a) {
  struct Table { epd_rope_cfg of; double turns[kRopePairs]; uint8_t axis[kRopePairs]; };
  static thread_local Table t = {};
  bool same = t.of.struct_size == c.struct_size && t.of.axes == c.axes && t.of.layout == c.layout && t.of.ladder == c.ladder && t.of.base == c.base;
  for (int x = 0; same && x < c.axes; ++x) same = t.of.pairs[x] == c.pairs[x];
  if (!same) {
    int p = 0;
    auto put = [&](int x, int j) {
      const double f = std::pow(c.base, c.ladder == EPD_ROPE_LADDER_AXIS ? -(double)j / c.pairs[x] : -(double)p / pairs);
      t.axis[p] = (uint8_t)x;
      t.turns[p++] = f / 6.283185307179586476925;
    };
    if (c.layout == EPD_ROPE_SECTIONS) {
      for (int x = 0; x < c.axes; ++x)
        for (int j = 0; j < c.pairs[x]; ++j) put(x, j);
    } else {
      for (int j = 0; p < pairs; ++j)
        for (int x = 0; x < c.axes; ++x)
          if (j < c.pairs[x]) put(x, j);
    }
    t.of = c;
  }
  std::copy(t.turns, t.turns + pairs, a.turns);
  std::copy(t.axis, t.axis + pairs, a.axis);
}

}  // namespace epd

using namespace epd;

extern "C" {

epd_status epd_rope_apply(const epd_rope_cfg* c, const epd_rope_tensor* tensors, int32_t num_tensors, const int32_t* positions,
                          int64_t position_stride, int32_t tokens, int32_t inverse, void* stream) {
  if (!c || !tensors || !positions) return op_fail(EPD_ERR_INVALID_ARG, "epd_rope_apply: a required pointer is NULL");
  if (c->struct_size != sizeof(epd_rope_cfg)) return op_fail(EPD_ERR_INVALID_ARG, "epd_rope_apply: cfg.struct_size %u != %zu", c->struct_size, sizeof(epd_rope_cfg));
  if ((c->dtype != EPD_F32 && c->dtype != EPD_BF16) || (c->layout != EPD_ROPE_SECTIONS && c->layout != EPD_ROPE_INTERLEAVED) ||
      (c->ladder != EPD_ROPE_LADDER_AXIS && c->ladder != EPD_ROPE_LADDER_HEAD) || (c->pairing != EPD_ROPE_HALF && c->pairing != EPD_ROPE_ADJACENT))
    return op_fail(EPD_ERR_INVALID_ARG, "epd_rope_apply: dtype, layout, ladder or pairing invalid");
  if (c->axes < 1 || c->axes > 4) return op_fail(EPD_ERR_INVALID_ARG, "epd_rope_apply: axes %d: 1 .. 4", c->axes);
  if (c->head_dim < 2 || c->head_dim > 2 * kRopePairs) return op_fail(EPD_ERR_UNSUPPORTED, "epd_rope_apply: head_dim %d: 2 .. %d", c->head_dim, 2 * kRopePairs);
  if (!(c->base > 0.0) || !std::isfinite(c->base)) return op_fail(EPD_ERR_INVALID_ARG, "epd_rope_apply: base must be positive and finite");
  int pairs = 0;
  for (int x = 0; x < c->axes; ++x) {
    if (c->pairs[x] < 0 || c->pairs[x] > kRopePairs) return op_fail(EPD_ERR_INVALID_ARG, "epd_rope_apply: pairs[%d] = %d", x, c->pairs[x]);
    pairs += c->pairs[x];
  }
  if (pairs < 1 || 2 * pairs > c->head_dim) return op_fail(EPD_ERR_UNSUPPORTED, "epd_rope_apply: %d pairs: 1 .. head_dim / 2 = %d", pairs, c->head_dim / 2);
  if (tokens < 0) return op_fail(EPD_ERR_SHAPE, "epd_rope_apply: tokens %d", tokens);
  if (position_stride < (c->axes > 1 ? tokens : 0)) return op_fail(EPD_ERR_SHAPE, "epd_rope_apply: position_stride %lld < tokens %d", (long long)position_stride, tokens);
  if (num_tensors < 1 || num_tensors > kRopeTensors) return op_fail(EPD_ERR_INVALID_ARG, "epd_rope_apply: num_tensors %d: 1 .. %d", num_tensors, kRopeTensors);
  if (inverse != 0 && inverse != 1) return op_fail(EPD_ERR_INVALID_ARG, "epd_rope_apply: inverse %d: 0 or 1", inverse);

  RopeArgs a{};
  const bool bf = c->dtype == EPD_BF16, adjacent = c->pairing == EPD_ROPE_ADJACENT;
  const size_t es = bf ? 2 : 4;
  pair_table(*c, pairs, a);
  // elements per access: what every pointer, stride and the pairs allow, 16 bytes at most
  int vec = bf ? 8 : 4, heads = 0;
  auto fits = [&](int64_t v) { while (vec > 1 && v % vec) vec /= 2; };
  fits(c->head_dim);
  fits(adjacent ? 2 * pairs : pairs);
  epd_rope_tensor of[kRopeTensors];
  for (int i = 0; i < num_tensors; ++i) {
    epd_rope_tensor& x = of[i];
    x = tensors[i];
    if (x.heads < 0 || x.heads > kRopeHeads) return op_fail(EPD_ERR_UNSUPPORTED, "epd_rope_apply: tensor %d has %d heads: 0 .. %d", i, x.heads, kRopeHeads);
    if (x.heads == 0 || tokens == 0) continue;
    if (!x.in || !x.out) return op_fail(EPD_ERR_INVALID_ARG, "epd_rope_apply: tensor %d: a required pointer is NULL", i);
    if (((uintptr_t)x.in | (uintptr_t)x.out) % es) return op_fail(EPD_ERR_INVALID_ARG, "epd_rope_apply: tensor %d is not aligned to its elements", i);
    if (tokens == 1) x.in_token = x.out_token = 0;         // there is no next row
    if (x.heads == 1) x.in_head = x.out_head = 0;
    constexpr int64_t kMaxStride = 1ll << 40;
    for (int64_t v : {x.in_token, x.in_head, x.out_token, x.out_head})
      if (v < 0 || v > kMaxStride) return op_fail(EPD_ERR_SHAPE, "epd_rope_apply: tensor %d has a stride of %lld", i, (long long)v);
    // rows of the output must be apart: tokens of heads, or heads of tokens
    const bool token_major = (x.heads == 1 || x.out_head >= c->head_dim) && (tokens == 1 || (__int128)x.out_token >= (__int128)(x.heads - 1) * x.out_head + c->head_dim);
    const bool head_major = (tokens == 1 || x.out_token >= c->head_dim) && (x.heads == 1 || (__int128)x.out_head >= (__int128)(tokens - 1) * x.out_token + c->head_dim);
    if (!token_major && !head_major) return op_fail(EPD_ERR_SHAPE, "epd_rope_apply: the output rows of tensor %d overlap", i);
    if (x.in == x.out && (x.in_token != x.out_token || x.in_head != x.out_head)) return op_fail(EPD_ERR_SHAPE, "epd_rope_apply: tensor %d: in place, the strides must be the same", i);
    for (int64_t v : {x.in_token, x.in_head, x.out_token, x.out_head}) fits(v);
    while (vec > 1 && ((uintptr_t)x.in | (uintptr_t)x.out) % (vec * es)) vec /= 2;
    heads += x.heads;
  }
  if (!heads) return EPD_OK;
  const int np = adjacent ? std::max(vec / 2, 1) : vec;
  a.pairs = pairs; a.turned = pairs / np; a.inverse = inverse; a.pos_stride = position_stride;
  auto inv = [](uint32_t d) { return (uint32_t)(((1ull << 32) + d - 1) / d); };
  a.inv_pairs = inv(pairs);
  int most = 1;
  for (int i = 0; i < num_tensors; ++i) {
    const epd_rope_tensor& x = of[i];
    if (!x.heads) continue;
    RopeTensor& d = a.t[a.n++];
    d.in = x.in; d.out = x.out; d.heads = x.heads;
    d.in_token = x.in_token; d.in_head = x.in_head; d.out_token = x.out_token; d.out_head = x.out_head;
    d.chunks = a.turned + (x.in == x.out ? 0 : (c->head_dim - 2 * pairs) / vec);
    d.per_token = x.heads * d.chunks;
    d.inv_chunks = inv(d.chunks); d.inv_per_token = inv(d.per_token);
    most = std::max(most, d.per_token);
  }
  // tokens per block: a cos / sin for every thread, while there are blocks for the whole chip; few tokens get several
  // blocks each, down to one round of threads
  a.block_tokens = std::max(1, std::min(256 / pairs, 65536 / most));
  while (a.block_tokens > 1 && tokens / a.block_tokens < 1024) a.block_tokens /= 2;
  const int blocks = (int)(((int64_t)tokens + a.block_tokens - 1) / a.block_tokens);
  const int shares = blocks >= 512 ? 1 : std::max(1, std::min((most * a.block_tokens + 255) / 256, 512 / blocks));
  for (int b = 0; b < blocks; b += kMaxGrid) {
    const int n = std::min(kMaxGrid, blocks - b);
    const int64_t tok0 = (int64_t)b * a.block_tokens;
    RopeArgs part = a;
    part.positions = positions + tok0;
    part.tokens = (int)std::min<int64_t>(tokens - tok0, (int64_t)n * a.block_tokens);
    for (int i = 0; i < a.n; ++i) {
      part.t[i].in = (const char*)a.t[i].in + tok0 * a.t[i].in_token * (int64_t)es;
      part.t[i].out = (char*)a.t[i].out + tok0 * a.t[i].out_token * (int64_t)es;
    }
    if (hipError_t e = launch_rope(part, bf, vec, adjacent, dim3(n, shares), (hipStream_t)stream))
      return op_launch_failed("epd_rope_apply", e);
  }
  return EPD_OK;
}

int64_t epd_rope_tokens(const int32_t* span_thw, int32_t num_spans) {
  if (!span_thw || num_spans < 0) { op_fail(EPD_ERR_INVALID_ARG, "epd_rope_tokens: span_thw is NULL or num_spans %d", num_spans); return -1; }
  int64_t tokens = 0;
  for (int64_t i = 0; i < num_spans; ++i) {
    const int64_t n = span_tokens(span_thw + 3 * i);
    if (n < 0 || (tokens += n) > INT_MAX) { op_fail(EPD_ERR_SHAPE, "epd_rope_tokens: span %lld is inconsistent or passes %d tokens", (long long)i, INT_MAX); return -1; }
  }
  return tokens;
}

epd_status epd_rope_positions(const int32_t* span_thw, const int32_t* cu_spans, int32_t num_sequences, const int32_t* start, int32_t t_step,
                              int32_t* positions, int64_t position_stride, int32_t* next_out, void* stream) {
  if (!span_thw || !cu_spans || !positions) return op_fail(EPD_ERR_INVALID_ARG, "epd_rope_positions: a required pointer is NULL");
  if (num_sequences < 0) return op_fail(EPD_ERR_SHAPE, "epd_rope_positions: num_sequences %d", num_sequences);
  if (t_step < 0) return op_fail(EPD_ERR_INVALID_ARG, "epd_rope_positions: t_step %d", t_step);
  if (cu_spans[0] != 0) return op_fail(EPD_ERR_SHAPE, "epd_rope_positions: cu_spans must start at 0");
  for (int s = 0; s < num_sequences; ++s)                  // first: the spans end at the last of cu_spans
    if (cu_spans[s + 1] < cu_spans[s]) return op_fail(EPD_ERR_SHAPE, "epd_rope_positions: cu_spans decreases at %d", s);
  // everything is checked before the first launch: two walks over the spans
  for (int pass = 0; pass < 2; ++pass) {
    int64_t tok = 0, sent = 0;
    PosArgs a;
    a.n = 0; a.stride = position_stride; a.t_step = t_step; a.pad = 0;
    auto flush = [&]() {
      hipError_t e = hipSuccess;
      if (a.n && tok > sent) {
        a.out = positions + sent; a.tokens = (int)(tok - sent);
        void* args[] = {(void*)&a};
        e = hipLaunchKernel((const void*)rope_positions_kernel, dim3((a.tokens - 1) / 256 + 1), dim3(256), args, 0, (hipStream_t)stream);
      }
      a.n = 0; sent = tok;
      return e;
    };
    for (int s = 0; s < num_sequences; ++s) {
      int64_t pos = start ? start[s] : 0;
      for (int i = cu_spans[s]; i < cu_spans[s + 1]; ++i) {
        const int64_t t = span_thw[3 * (int64_t)i], h = span_thw[3 * (int64_t)i + 1], w = span_thw[3 * (int64_t)i + 2];
        const bool text = h == 0 && w == 0;
        const int64_t count = span_tokens(span_thw + 3 * (int64_t)i);
        if (!pass && count == -1)
          return op_fail(EPD_ERR_SHAPE, "epd_rope_positions: span %d = (%lld, %lld, %lld): a text is (n, 0, 0), an item has positive sizes", i, (long long)t, (long long)h, (long long)w);
        if (!pass && count < 0) return op_fail(EPD_ERR_SHAPE, "epd_rope_positions: span %d has too many tokens", i);
        const int64_t ahead = text ? t : std::max((int64_t)t_step * (t - 1) + 1, std::max(h, w));
        if (pass && count) {
          if (a.n == kPosSpans)
            if (hipError_t e = flush()) return op_launch_failed("epd_rope_positions", e);
          a.span[a.n++] = PosSpan{(int32_t)(tok - sent), (int32_t)pos, (int32_t)h, (int32_t)w};
        }
        tok += count;
        pos += ahead;
        if (!pass && tok > INT_MAX) return op_fail(EPD_ERR_SHAPE, "epd_rope_positions: more than %d tokens", INT_MAX);
        if (!pass && pos > INT_MAX) return op_fail(EPD_ERR_SHAPE, "epd_rope_positions: sequence %d runs past position %d", s, INT_MAX);
      }
      if (pass && next_out) next_out[s] = (int32_t)pos;
    }
    if (!pass) {
      if (position_stride < tok) return op_fail(EPD_ERR_SHAPE, "epd_rope_positions: position_stride %lld < %lld tokens", (long long)position_stride, (long long)tok);
    } else if (hipError_t e = flush()) {
      return op_launch_failed("epd_rope_positions", e);
    }
  }
  return EPD_OK;
}

}  // extern "C"
