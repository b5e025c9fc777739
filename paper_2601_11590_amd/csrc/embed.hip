// Embeddings of sequences of text and visual tokens, V_m || V_t (paper section 3.1 "Prefill Stage", Eq. 1 and 2), as an operator: a
// token's row comes from the table, scaled, or is a row of V_m as it is; and the gradients of both.
// Bound: HBM (few tokens: latency).
//
// Backward.  Text and visual rows are one range of keys, the table's rows and behind them those of V_m:
//   grad[key] = sum of dout over the tokens of that key (* scale)
// The tokens are sorted by key, which puts those of a row side by side; blocks then add runs of equal keys.  Nothing is added
// atomically, so a gradient's bits depend on the ids alone.
//   1. sort_kernel: up to 8192 tokens a block, sorted in LDS by their keys' digits, from the lowest up, keeping the order of equal ones;
//      meanwhile the other blocks clear the gradients, which is most of what is written where the table is large
//   2. merge_kernel (more than 8192 tokens): eight sorted lists into one at a time: an element's place is its own plus the numbers of
//      smaller ones in the other lists
//   3. sums_kernel: pieces of 16 or 32 sorted tokens; runs within a piece are written, the ends of others left as partial sums
//   4. runs_kernel: runs over several pieces, so that a token that takes every other place costs no more than others
#include "op_error.h"
#include "rows.h"

#include <algorithm>
#include <cmath>

namespace epd {

namespace {

constexpr int kEmbedDim = 65536, kEmbedRows = 1 << 30, kEmbedTokens = 1 << 24;

struct EmbedArgs {
  const void *table, *rows;
  const int32_t* ids;
  void* out;
  int64_t ld_out;
  int tokens, D, vocab, num_rows;
  float scale;
};

// A wave takes U * 512 elements of a token's row.
template <typename T, typename O, int U> __global__ __launch_bounds__(256) void embed_kernel(EmbedArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t token = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (token >= a.tokens) return;
  const int id = a.ids[token];
  const bool text = id >= 0 && id < a.vocab, visual = id < 0 && id >= -a.num_rows;
  const T* const from = text ? (const T*)a.table + (int64_t)id * a.D : visual ? (const T*)a.rows + (int64_t)(-1 - id) * a.D : nullptr;
  O* const out = (O*)a.out + token * a.ld_out;
  const float scale = text ? a.scale : 1.0f;
  const int e0 = (int)blockIdx.y * U * 512 + lane * 8;
  float v[U][8];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int e = e0 + u * 512, left = a.D - e;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[u][i] = 0.f;
    if (from && left > 0) load8(from + e, left, v[u]);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int e = e0 + u * 512, left = a.D - e;
    if (left <= 0) continue;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[u][i] *= scale;
    store8(out + e, left, v[u]);
  }
}

// ------------------------------------------------------------------------------ sorted tokens
constexpr int kSortList = 8192, kSortWaves = 16, kMaxDigit = 9;

struct SortArgs {
  const int32_t* ids;
  uint32_t *key, *at;                // sorted lists of kSortList
  int tokens, vocab, num_rows;
  uint32_t none;                     // the key of tokens without a gradient, behind all others: vocab + num_rows
  int passes, bits;                  // digits of a key, and their bits
  int sort_blocks;
  void* clear[2];                    // gradients to clear, and their 16-byte pieces and bytes behind these
  int64_t pieces[2];
  int tail[2];
};

__global__ __launch_bounds__(1024) void sort_kernel(SortArgs a) {
  __shared__ uint32_t keys[2][kSortList];
  __shared__ uint16_t ats[2][kSortList];
  __shared__ uint32_t count[kSortWaves << kMaxDigit];
  __shared__ uint32_t wave_sum[kSortWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if ((int)blockIdx.x >= a.sort_blocks) {
    const int64_t t0 = ((int64_t)blockIdx.x - a.sort_blocks) * 1024 + tid, n = ((int64_t)gridDim.x - a.sort_blocks) * 1024;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      quad2* const to = (quad2*)a.clear[j];
      for (int64_t i = t0; i < a.pieces[j]; i += n) to[i] = quad2{0u, 0u, 0u, 0u};
      if (t0 < a.tail[j]) ((uint8_t*)(to + a.pieces[j]))[t0] = 0;
    }
    return;
  }
  const int first = (int)blockIdx.x * kSortList, n = min(kSortList, a.tokens - first);
  const int rounds = (n + 1023) / 1024, base = wave * rounds * 64;       // a wave's elements: side by side, 64 a round
  for (int r = 0; r < rounds; ++r) {
    const int i = base + r * 64 + lane;
    uint32_t k = a.none;                                   // elements past the last one stay behind it: equal keys keep their order
    if (i < n) {
      const int id = a.ids[first + i];
      if (id >= 0) { if (id < a.vocab) k = (uint32_t)id; }
      else if (id >= -a.num_rows) k = (uint32_t)a.vocab + (uint32_t)(-1 - id);
    }
    keys[0][i] = k;
    ats[0][i] = (uint16_t)i;
  }
  __syncthreads();
  const int digits = 1 << a.bits, per = digits * kSortWaves / 1024;      // counters per thread in the scan (bits >= 6: one or more)
  for (int p = 0; p < a.passes; ++p) {
    const int from = p & 1, shift = p * a.bits;
    for (int c = tid; c < digits * kSortWaves; c += 1024) count[c] = 0;
    __syncthreads();
    uint32_t place[kSortList / 1024];                      // among the wave's elements of the same digit
#pragma unroll
    for (int r = 0; r < kSortList / 1024; ++r) {
      if (r >= rounds) break;
      const uint32_t d = keys[from][base + r * 64 + lane] >> shift & (digits - 1);
      uint64_t same = ~0ull;
      for (int b = 0; b < a.bits; ++b) {
        const uint64_t set = __ballot(d >> b & 1);
        same &= d >> b & 1 ? set : ~set;
      }
      uint32_t* const c = &count[d * kSortWaves + wave];
      const uint32_t before = *(volatile uint32_t*)c;
      place[r] = before + (uint32_t)__popcll(same & ((1ull << lane) - 1));
      // (LDS takes a wave's accesses in order: all lanes have read before the first of each digit writes)
      if (__ffsll((unsigned long long)same) - 1 == lane) *(volatile uint32_t*)c = before + (uint32_t)__popcll(same);
    }
    __syncthreads();
    // exclusive sums over [digit][wave]
    uint32_t mine = 0;
    for (int j = 0; j < per; ++j) mine += count[tid * per + j];
    uint32_t upto = mine;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) { const uint32_t v = __shfl_up(upto, o); if (lane >= o) upto += v; }
    if (lane == 63) wave_sum[wave] = upto;
    __syncthreads();
    uint32_t sum = upto - mine;
    for (int w = 0; w < wave; ++w) sum += wave_sum[w];
    for (int j = 0; j < per; ++j) { const uint32_t c = count[tid * per + j]; count[tid * per + j] = sum; sum += c; }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSortList / 1024; ++r) {
      if (r >= rounds) break;
      const int i = base + r * 64 + lane;
      const uint32_t k = keys[from][i], to = count[(k >> shift & (digits - 1)) * kSortWaves + wave] + place[r];
      keys[from ^ 1][to] = k;
      ats[from ^ 1][to] = ats[from][i];
    }
    __syncthreads();
  }
  const int last = a.passes & 1;
  for (int i = tid; i < n; i += 1024) {
    a.key[first + i] = keys[last][i];
    a.at[first + i] = (uint32_t)first + ats[last][i];
  }
}

// Groups of up to eight sorted lists of `len` into one each; lists stand in the order of their tokens, so of equal keys those of an
// earlier list come first.
constexpr int kMergeLists = 8;
struct MergeArgs { const uint32_t *key, *at; uint32_t *key_out, *at_out; int tokens, len, steps; };      // steps: 2^steps > len
__global__ __launch_bounds__(256) void merge_kernel(MergeArgs a) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= a.tokens) return;
  const int list = i / a.len, first = list / kMergeLists * kMergeLists;
  const uint32_t k = a.key[i];
  int below[kMergeLists], size[kMergeLists];
#pragma unroll
  for (int j = 0; j < kMergeLists; ++j) {
    const int64_t start = (int64_t)(first + j) * a.len;
    below[j] = 0;
    size[j] = first + j == list ? 0 : (int)max((int64_t)0, min((int64_t)a.len, a.tokens - start));
  }
  for (int s = a.steps - 1; s >= 0; --s) {
    uint32_t probe[kMergeLists];
#pragma unroll
    for (int j = 0; j < kMergeLists; ++j) {
      const int next = below[j] + (1 << s);
      probe[j] = next <= size[j] ? a.key[(int64_t)(first + j) * a.len + next - 1] : 0xffffffffu;
    }
#pragma unroll
    for (int j = 0; j < kMergeLists; ++j) {
      const int next = below[j] + (1 << s);
      if (next <= size[j] && (first + j < list ? probe[j] <= k : probe[j] < k)) below[j] = next;
    }
  }
  int64_t to = (int64_t)first * a.len + (i - (int64_t)list * a.len);
#pragma unroll
  for (int j = 0; j < kMergeLists; ++j) to += below[j];
  a.key_out[to] = k;
  a.at_out[to] = a.at[i];
}

// ------------------------------------------------------------------------------ sums of runs
constexpr int kPiece = 32, kFewPieces = 1024;      // tokens of a piece; half of that while the pieces are fewer than the second
int piece_of(int tokens) { return tokens <= kFewPieces * kPiece / 2 ? kPiece / 2 : kPiece; }
int pieces_of(int tokens) { return (tokens + piece_of(tokens) - 1) / piece_of(tokens); }
int most_pieces(int max_tokens) { return std::max(pieces_of(max_tokens), pieces_of(std::min(max_tokens, kFewPieces * kPiece / 2))); }

struct SumsArgs {
  const uint32_t *key, *at;
  const void* dout;
  float* parts;                      // [piece][2][D]: the run that comes from the piece before, and the one that starts here and goes on
  void *table, *rows;
  int64_t ld;
  int tokens, D, vocab, piece;
  uint32_t none;
  float scale;
};

template <typename T> __device__ __forceinline__ T* row_of(const SumsArgs& a, uint32_t key, float& scale) {
  const bool text = key < (uint32_t)a.vocab;
  scale = text ? a.scale : 1.0f;
  return text ? (T*)a.table + (int64_t)key * a.D : (T*)a.rows + (int64_t)(key - (uint32_t)a.vocab) * a.D;
}

// (tokens whose gradient is not wanted keep their places, so that the others' sums have the same bits in every call)
__device__ __forceinline__ bool wanted(const SumsArgs& a, uint32_t key) { return key < (uint32_t)a.vocab ? a.table != nullptr : key < a.none && a.rows != nullptr; }

template <typename T, typename O> __global__ __launch_bounds__(256) void sums_kernel(SumsArgs a) {
  __shared__ uint32_t key[kPiece + 2], at[kPiece];         // key[0]: that of the token ahead
  const int p0 = blockIdx.x * a.piece, n = min(a.piece, a.tokens - p0);
  if ((int)threadIdx.x < n + 2) {
    const int p = p0 - 1 + (int)threadIdx.x;
    key[threadIdx.x] = p >= 0 && p < a.tokens ? a.key[p] : 0xffffffffu;
    if (threadIdx.x < n) at[threadIdx.x] = a.at[p0 + (int)threadIdx.x];
  }
  __syncthreads();
  const int e = ((int)blockIdx.y * 256 + (int)threadIdx.x) * 8, left = a.D - e;
  if (left <= 0) return;
  float sum[8];
  bool from_before = key[0] == key[1];
#pragma unroll
  for (int i = 0; i < 8; ++i) sum[i] = 0.f;
  constexpr int BATCH = 8;
  for (int b = 0; b < n; b += BATCH) {
    float v[BATCH][8];
#pragma unroll
    for (int j = 0; j < BATCH; ++j)
      if (b + j < n && wanted(a, key[b + j + 1])) load8((const O*)a.dout + (int64_t)at[b + j] * a.ld + e, left, v[j]);
#pragma unroll
    for (int j = 0; j < BATCH; ++j) {
      if (b + j >= n) break;
      const uint32_t k = key[b + j + 1];
      if (k >= a.none) return;                             // and all behind it
      const bool ends = key[b + j + 2] != k;
      if (!wanted(a, k)) { from_before = !ends; continue; }
#pragma unroll
      for (int i = 0; i < 8; ++i) sum[i] += v[j][i];
      if (!ends && b + j + 1 < n) continue;
      if (ends && !from_before) {
        float scale;
        T* const row = row_of<T>(a, k, scale);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] *= scale;
        store8(row + e, left, sum);
      } else {
        store8(a.parts + ((int64_t)blockIdx.x * 2 + (from_before ? 0 : 1)) * a.D + e, left, sum);
      }
      from_before = false;
#pragma unroll
      for (int i = 0; i < 8; ++i) sum[i] = 0.f;
    }
  }
}

// Runs that start in piece blockIdx.x and go on: their partial sums, 256 columns a block, sixteen groups of threads in turn.
template <typename T> __global__ __launch_bounds__(1024) void runs_kernel(SumsArgs a) {
  __shared__ float part[16][256];
  const int piece = blockIdx.x;
  const int64_t next = (int64_t)(piece + 1) * a.piece;     // < tokens
  const uint32_t k = a.key[next];
  if (!wanted(a, k) || a.key[next - 1] != k || (piece > 0 && a.key[next - a.piece - 1] == k)) return;
  int64_t last = next, step = 1;                           // the last token of the run
  while (last + step < a.tokens && a.key[last + step] == k) { last += step; step *= 2; }
  for (; step > 0; step /= 2)
    if (last + step < a.tokens && a.key[last + step] == k) last += step;
  const int n = (int)(last / a.piece) - piece + 1;
  const int g = threadIdx.x >> 6, e = (int)blockIdx.y * 256 + (int)(threadIdx.x & 63) * 4;
  float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int p = g; p < n; p += 16) {
    const float* const from = a.parts + ((int64_t)(piece + p) * 2 + (p ? 0 : 1)) * a.D + e;
    if (e + 4 <= a.D) {
      const quad4 u = *(const quad4*)from;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] += u[i];
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) if (e + i < a.D) v[i] += from[i];
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) part[g][(threadIdx.x & 63) * 4 + i] = v[i];
  __syncthreads();
  const int c = (int)blockIdx.y * 256 + (int)threadIdx.x;
  if (threadIdx.x >= 256 || c >= a.D) return;
  float sum = part[0][threadIdx.x], scale;
#pragma unroll
  for (int i = 1; i < 16; ++i) sum += part[i][threadIdx.x];
  T* const row = row_of<T>(a, k, scale);
  row[c] = (T)(sum * scale);
}

epd_status check_cfg(const char* who, const epd_embed_cfg* c) {
  if (!c) return op_fail(EPD_ERR_INVALID_ARG, "%s: cfg is NULL", who);
  if (c->struct_size != sizeof(epd_embed_cfg)) return op_fail(EPD_ERR_INVALID_ARG, "%s: cfg.struct_size %u != %zu", who, c->struct_size, sizeof(epd_embed_cfg));
  if (!known_dtype(c->dtype) || !known_dtype(c->out_dtype)) return op_fail(EPD_ERR_INVALID_ARG, "%s: dtype or out_dtype invalid", who);
  if (c->dtype == EPD_F32 && c->out_dtype != EPD_F32) return op_fail(EPD_ERR_UNSUPPORTED, "%s: an fp32 table has fp32 rows", who);
  if (c->vocab < 1 || c->vocab > kEmbedRows) return op_fail(EPD_ERR_UNSUPPORTED, "%s: vocab %d: 1 .. 2^30", who, c->vocab);
  if (c->hidden < 1 || c->hidden > kEmbedDim) return op_fail(EPD_ERR_UNSUPPORTED, "%s: hidden %d: 1 .. %d", who, c->hidden, kEmbedDim);
  if (c->max_tokens < 1 || c->max_tokens > kEmbedTokens) return op_fail(EPD_ERR_UNSUPPORTED, "%s: max_tokens %d: 1 .. 2^24", who, c->max_tokens);
  if (!std::isfinite(c->scale)) return op_fail(EPD_ERR_INVALID_ARG, "%s: scale must be finite", who);
  return EPD_OK;
}

epd_status check_call(const char* who, const epd_embed_cfg* c, int32_t num_rows, const int32_t* ids, int32_t tokens) {
  if (epd_status s = check_cfg(who, c)) return s;
  if (tokens < 0 || tokens > c->max_tokens) return op_fail(EPD_ERR_SHAPE, "%s: tokens %d: 0 .. max_tokens %d", who, tokens, c->max_tokens);
  if (num_rows < 0 || num_rows > kEmbedRows) return op_fail(EPD_ERR_UNSUPPORTED, "%s: num_rows %d: 0 .. 2^30", who, num_rows);
  if (tokens && (!ids || (uintptr_t)ids % 4)) return op_fail(EPD_ERR_INVALID_ARG, "%s: ids is NULL or not aligned", who);
  return EPD_OK;
}

struct EmbedLayout { size_t list, parts, total; };         // bytes: key and at, twice, and the partial sums
EmbedLayout embed_layout(const epd_embed_cfg& c) {
  EmbedLayout L;
  auto up = [](size_t v) { return (v + 255) / 256 * 256; };
  L.list = up((size_t)c.max_tokens * 4);
  L.parts = 4 * L.list;
  L.total = up(L.parts + (size_t)most_pieces(c.max_tokens) * 2 * c.hidden * 4);
  return L;
}

template <class F> hipError_t by_types(const epd_embed_cfg& c, F&& f) {
  if (c.dtype == EPD_F32) return f(0.f, 0.f);
  return c.out_dtype == EPD_F32 ? f((__bf16)0.f, 0.f) : f((__bf16)0.f, (__bf16)0.f);
}

}  // namespace
}  // namespace epd

using namespace epd;

extern "C" {

uint64_t epd_embed_workspace_bytes(const epd_embed_cfg* cfg) {
  if (check_cfg("epd_embed_workspace_bytes", cfg) != EPD_OK) return 0;
  return embed_layout(*cfg).total;
}

epd_status epd_embed(const epd_embed_cfg* cfg, const void* table, const void* rows, int32_t num_rows, const int32_t* ids, int32_t tokens, void* out,
                     int64_t ld_out, void* stream) {
  const char* const who = "epd_embed";
  if (epd_status s = check_call(who, cfg, num_rows, ids, tokens)) return s;
  const epd_embed_cfg& c = *cfg;
  const int es = c.dtype == EPD_F32 ? 4 : 2;
  if (!table || (num_rows && !rows)) return op_fail(EPD_ERR_INVALID_ARG, "%s: a required pointer is NULL", who);
  if (((uintptr_t)table | (num_rows ? (uintptr_t)rows : 0)) % es) return op_fail(EPD_ERR_INVALID_ARG, "%s: table or rows are not aligned to their elements", who);
  if (tokens == 0) return EPD_OK;
  if (epd_status s = check_rows(who, "out", out, ld_out, tokens, c.hidden, c.out_dtype == EPD_F32 ? 4 : 2)) return s;
  EmbedArgs a{table, rows, ids, out, ld_out, tokens, c.hidden, c.vocab, num_rows, c.scale};
  void* args[] = {(void*)&a};
  // few tokens: a row over as many waves as it has pieces of 512 (32 rows of 3200: 7 waves each, not 2)
  const bool few = (int64_t)tokens * ((c.hidden + 2047) / 2048) < 4096;
  const dim3 grid((tokens + 3) / 4, few ? (c.hidden + 511) / 512 : (c.hidden + 2047) / 2048);
  const hipError_t e = by_types(c, [&](auto t, auto o) {
    typedef decltype(t) T;
    typedef decltype(o) O;
    return hipLaunchKernel(few ? (const void*)embed_kernel<T, O, 1> : (const void*)embed_kernel<T, O, 4>, grid, dim3(256), args, 0, (hipStream_t)stream);
  });
  return e == hipSuccess ? EPD_OK : op_launch_failed(who, e);
}

epd_status epd_embed_backward(const epd_embed_cfg* cfg, const int32_t* ids, int32_t tokens, const void* dout, int64_t ld_dout, int32_t num_rows,
                              void* dtable, void* drows, void* workspace, uint64_t workspace_bytes, void* stream) {
  const char* const who = "epd_embed_backward";
  if (epd_status s = check_call(who, cfg, num_rows, ids, tokens)) return s;
  const epd_embed_cfg& c = *cfg;
  const int es = c.dtype == EPD_F32 ? 4 : 2;
  if (((uintptr_t)dtable | (uintptr_t)drows) % es) return op_fail(EPD_ERR_INVALID_ARG, "%s: gradients are not aligned to their elements", who);
  if (tokens) if (epd_status s = check_rows(who, "dout", dout, ld_dout, tokens, c.hidden, c.out_dtype == EPD_F32 ? 4 : 2)) return s;
  if (!workspace || (uintptr_t)workspace % 256) return op_fail(EPD_ERR_WORKSPACE, "%s: workspace is NULL or not 256-byte aligned", who);
  const EmbedLayout L = embed_layout(c);
  if (workspace_bytes < L.total) return op_fail(EPD_ERR_WORKSPACE, "%s: workspace_bytes %llu < required %zu", who, (unsigned long long)workspace_bytes, L.total);
  if (num_rows == 0) drows = nullptr;
  if (!dtable && !drows) return EPD_OK;
  char* const ws = (char*)workspace;
  uint32_t *key = (uint32_t*)ws, *at = (uint32_t*)(ws + L.list), *key2 = (uint32_t*)(ws + 2 * L.list), *at2 = (uint32_t*)(ws + 3 * L.list);
  hipStream_t st = (hipStream_t)stream;

  SortArgs s{};
  s.ids = ids; s.key = key; s.at = at; s.tokens = tokens; s.vocab = c.vocab; s.num_rows = num_rows;
  s.none = (uint32_t)c.vocab + (uint32_t)num_rows;
  int bits = 1;
  while ((uint64_t)s.none >> bits) ++bits;
  s.passes = (bits + kMaxDigit - 1) / kMaxDigit;
  s.bits = std::max(6, (bits + s.passes - 1) / s.passes);
  s.sort_blocks = (tokens + kSortList - 1) / kSortList;
  auto clears = [&](int j, void* p, int64_t n) { if (p) { s.clear[j] = p; s.pieces[j] = n * es / 16; s.tail[j] = (int)(n * es % 16); } };
  clears(0, dtable, (int64_t)c.vocab * c.hidden);
  clears(1, drows, (int64_t)num_rows * c.hidden);
  const int clear_blocks = (int)std::max<int64_t>(1, std::min<int64_t>(1024, (s.pieces[0] + s.pieces[1]) / 8192));
  void* sargs[] = {(void*)&s};
  hipError_t e = hipLaunchKernel((const void*)sort_kernel, dim3(s.sort_blocks + clear_blocks), dim3(1024), sargs, 0, st);
  int64_t len = kSortList;
  for (; e == hipSuccess && len < tokens; len *= kMergeLists) {
    MergeArgs m{key, at, key2, at2, tokens, (int)len, 1};
    while ((1ll << m.steps) <= len) ++m.steps;
    void* margs[] = {(void*)&m};
    e = hipLaunchKernel((const void*)merge_kernel, dim3((tokens + 255) / 256), dim3(256), margs, 0, st);
    std::swap(key, key2);
    std::swap(at, at2);
  }
  if (e == hipSuccess && tokens) {
    const int pieces = pieces_of(tokens);
    SumsArgs a{key, at, dout, (float*)(ws + L.parts), dtable, drows, ld_dout, tokens, c.hidden, c.vocab, piece_of(tokens), s.none, c.scale};
    void* args[] = {(void*)&a};
    e = by_types(c, [&](auto t, auto o) {
      return hipLaunchKernel((const void*)sums_kernel<decltype(t), decltype(o)>, dim3(pieces, (c.hidden + 2047) / 2048), dim3(256), args, 0, st);
    });
    if (e == hipSuccess && pieces > 1)
      e = hipLaunchKernel(es == 4 ? (const void*)runs_kernel<float> : (const void*)runs_kernel<__bf16>, dim3(pieces - 1, (c.hidden + 255) / 256), dim3(1024), args, 0, st);
  }
  return e == hipSuccess ? EPD_OK : op_launch_failed(who, e);
}

}  // extern "C"
