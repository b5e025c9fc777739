// Embeddings of sequences of text and visual tokens, V_m || V_t (paper section 3.1 "Prefill Stage", Eq. 1 and 2), as an operator: a
// token's row comes from the table, scaled, or is a row of V_m as it is; and the gradients of both.
// Bound: HBM (few tokens: latency).
//
// Backward.  Text and visual rows are one range of keys, the table's rows and behind them those of V_m:
//   grad[key] = sum of dout over the tokens of that key (* scale)
// The tokens are sorted by key, which puts those of a row side by side; blocks then add runs of equal keys (up to 128 tokens: few_kernel).  Nothing is added
// atomically (an atomic counter only gives long runs their places in a list), so a gradient's bits depend on ids and values alone.
//   1. sort_kernel: up to 4096 tokens a block, sorted in LDS by their keys' digits, from the lowest up, keeping the order of equal ones;
//      meanwhile other blocks clear the gradients, or as much of them as the sort hides (4096 keys of 18 bits 11 us; 65 MB beside 2049 tokens 10)
//   2. merge_kernel (more than 4096 tokens): eight sorted lists into one at a time: an element's place is its own plus the numbers of
//      smaller ones in the other lists
//   3. sums_kernel: pieces of 8 to 32 sorted tokens; runs within a piece and the next are written, longer ones left as partial sums; where the
//      tokens' rows are many, its other blocks clear the rest of the rows of no token (32 768 fp32 rows of 3200 into 131 072 in bf16: 257 us, 4.5 TB/s)
//   4. runs_kernel: those, so that a token that takes every other place costs no more than others
#include "op_error.h"
#include "rows.h"

#include <algorithm>
#include <cmath>

namespace epd {

namespace {

constexpr int kEmbedDim = 65536, kEmbedRows = 1 << 30, kEmbedTokens = 1 << 24;
constexpr int64_t kEmbedElements = 1ll << 38;              // of all tokens: a launch has fewer than 2^32 threads along each axis of its grid

struct EmbedArgs {
  const void *table, *rows;
  const int32_t* ids;
  void* out;
  int64_t ld_out;
  int tokens, D, vocab, num_rows;
  float scale;
  bool through;                      // see writes_through
};

// A wave takes U * 512 elements of a token's row.  16 384 rows of 3584, bf16: 47.2 us, 5.0 TB/s (48.6 ... 49.3 without writing through).
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
    store8(out + e, left, v[u], a.through);
  }
}

// ------------------------------------------------------------------------------ sorted tokens
constexpr int kSortList = 4096, kSortWaves = 16, kMaxDigit = 9;

struct SortArgs {
  const int32_t* ids;
  uint32_t *key, *at;                // sorted lists of kSortList
  int tokens, vocab, num_rows;
  uint32_t none;                     // the key of tokens without a gradient, behind all others: vocab + num_rows
  int passes, bits;                  // digits of a key, and their bits
  int sort_blocks;
  uint32_t* counts;                  // two counters to clear
  void* clear[2];                    // gradients to clear, and their 16-byte pieces and bytes behind these
  int64_t pieces[2];
  int tail[2];
};

__device__ __forceinline__ uint32_t key_of(int id, int vocab, int num_rows, uint32_t none) {
  if (id >= 0) return id < vocab ? (uint32_t)id : none;
  return id >= -num_rows ? (uint32_t)vocab + (uint32_t)(-1 - id) : none;
}

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
      if ((uintptr_t)to % 16 == 0) {                       // (65 MB beside 2049 tokens 10.0 us, not written through 11.3 ... 12.8)
        for (int64_t i = t0; i < a.pieces[j]; i += n) store16_through(to + i, quad2{0u, 0u, 0u, 0u});
      } else {
        for (int64_t i = t0; i < a.pieces[j]; i += n) to[i] = quad2{0u, 0u, 0u, 0u};
      }
      if (t0 < a.tail[j]) ((uint8_t*)(to + a.pieces[j]))[t0] = 0;
    }
    return;
  }
  if (blockIdx.x == 0 && tid < 2) a.counts[tid] = 0;
  const int first = (int)blockIdx.x * kSortList, n = min(kSortList, a.tokens - first);
  const int rounds = (n + 1023) / 1024, base = wave * rounds * 64;       // a wave's elements: side by side, 64 a round
  for (int r = 0; r < rounds; ++r) {
    const int i = base + r * 64 + lane;
    // elements past the last one stay behind it: equal keys keep their order
    const uint32_t k = i < n ? key_of(a.ids[first + i], a.vocab, a.num_rows, a.none) : a.none;
    keys[0][i] = k;
    ats[0][i] = (uint16_t)i;
  }
  __syncthreads();
  const int digits = 1 << a.bits;
  for (int p = 0; p < a.passes; ++p) {
    const int from = p & 1, shift = p * a.bits;
    for (int c = tid; c < digits * kSortWaves; c += 1024) count[c] = 0;
    __syncthreads();
    // place among the wave's elements of the same digit.  The lanes of a digit find each other by ballots; LDS takes a wave's accesses in
    // order, so all of them have read its counter before the first of them writes it
    uint32_t place[kSortList / 1024], digit[kSortList / 1024];
    uint32_t* const mine = count + wave * digits;
#pragma unroll
    for (int r = 0; r < kSortList / 1024; ++r) {
      if (r >= rounds) break;
      const uint32_t d = keys[from][base + r * 64 + lane] >> shift & (digits - 1);
      uint32_t lo = ~0u, hi = ~0u;                         // lanes of the same digit
#pragma unroll
      for (int b = 0; b < kMaxDigit; ++b) {                // (bits that no digit has change nothing)
        const uint64_t set = __ballot(d >> b & 1);
        const uint32_t mask = (uint32_t)((int)(d << (31 - b)) >> 31);
        lo &= ~((uint32_t)set ^ mask);
        hi &= ~((uint32_t)(set >> 32) ^ mask);
      }
      const uint32_t before = mine[d], ahead = __builtin_amdgcn_mbcnt_hi(hi, __builtin_amdgcn_mbcnt_lo(lo, 0u));
      asm volatile("" ::: "memory");
      digit[r] = d;
      place[r] = before + ahead;
      if (ahead == 0) mine[d] = before + (uint32_t)(__popc(lo) + __popc(hi));
      asm volatile("" ::: "memory");
    }
    __syncthreads();
    // exclusive sums, digits first, waves of a digit after that: a thread per digit
    uint32_t of[kSortWaves], all = 0;
    if (tid < digits) {
#pragma unroll
      for (int w = 0; w < kSortWaves; ++w) { of[w] = all; all += count[w * digits + tid]; }
    }
    uint32_t upto = all;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) { const uint32_t v = __shfl_up(upto, o); if (lane >= o) upto += v; }
    if (lane == 63) wave_sum[wave] = upto;
    __syncthreads();
    if (tid < digits) {
      uint32_t sum = upto - all;
#pragma unroll
      for (int w = 0; w < (1 << kMaxDigit) / 64; ++w) if (w < wave) sum += wave_sum[w];
#pragma unroll
      for (int w = 0; w < kSortWaves; ++w) count[w * digits + tid] = sum + of[w];
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSortList / 1024; ++r) {
      if (r >= rounds) break;
      const int i = base + r * 64 + lane;
      const uint32_t to = mine[digit[r]] + place[r];
      keys[from ^ 1][to] = keys[from][i];
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

// Groups of up to eight sorted lists of `len` (a multiple of 4096) into one each; lists stand in the order of their tokens, so of equal keys
// those of an earlier list come first.  A thread per element; every 1/128th key of the lists comes to LDS, so that only the last steps of
// its searches wait for memory.
constexpr int kMergeLists = 8, kSamples = 128;
struct MergeArgs { const uint32_t *key, *at; uint32_t *key_out, *at_out; int tokens, len; };
__global__ __launch_bounds__(256) void merge_kernel(MergeArgs a) {
  __shared__ uint32_t sample[kMergeLists][kSamples];
  const int64_t i0 = (int64_t)blockIdx.x * 256;            // a block's elements are of one list
  const int list = (int)(i0 / a.len), first = list / kMergeLists * kMergeLists, stride = a.len / kSamples;
  for (int s = threadIdx.x; s < kMergeLists * kSamples; s += 256) {
    const int64_t p = (int64_t)(first + s / kSamples) * a.len + (int64_t)(s % kSamples + 1) * stride - 1;
    sample[s / kSamples][s % kSamples] = p < a.tokens ? a.key[p] : 0xffffffffu;
  }
  __syncthreads();
  const int64_t i = i0 + threadIdx.x;
  if (i >= a.tokens) return;
  const uint32_t k = a.key[i];
  int below[kMergeLists], size[kMergeLists];
#pragma unroll
  for (int j = 0; j < kMergeLists; ++j) {
    const int64_t start = (int64_t)(first + j) * a.len;
    below[j] = 0;
    size[j] = first + j == list ? 0 : (int)max((int64_t)0, min((int64_t)a.len, a.tokens - start));
  }
  auto under = [&](int j, uint32_t key) { return first + j < list ? key <= k : key < k; };
#pragma unroll
  for (int s = kSamples; s > 0; s /= 2)                    // in samples
#pragma unroll
    for (int j = 0; j < kMergeLists; ++j) {
      const int next = below[j] + s;
      if (next * stride <= size[j] && under(j, sample[j][next - 1])) below[j] = next;
    }
#pragma unroll
  for (int j = 0; j < kMergeLists; ++j) below[j] *= stride;
  for (int s = stride / 2; s > 0; s /= 2) {
    uint32_t probe[kMergeLists];
#pragma unroll
    for (int j = 0; j < kMergeLists; ++j) {
      const int next = below[j] + s;
      probe[j] = next <= size[j] ? a.key[(int64_t)(first + j) * a.len + next - 1] : 0xffffffffu;
    }
#pragma unroll
    for (int j = 0; j < kMergeLists; ++j)
      if (below[j] + s <= size[j] && under(j, probe[j])) below[j] += s;
  }
  int64_t to = (int64_t)first * a.len + (i - (int64_t)list * a.len);
#pragma unroll
  for (int j = 0; j < kMergeLists; ++j) to += below[j];
  a.key_out[to] = k;
  a.at_out[to] = a.at[i];
}

// ------------------------------------------------------------------------------ sums of runs
constexpr int64_t kClearAll = 48 << 20;              // bytes of the tokens' rows up to which all rows are cleared first
constexpr int64_t kClearBesideSort = 96 << 20;       // bytes
constexpr int kPiece = 32, kLeastPiece = 8, kFewPieces = 1024;      // tokens of a piece, fewer while that gives no more pieces than this
int piece_of(int tokens) {
  int piece = kLeastPiece;
  while (piece < kPiece && tokens > kFewPieces * piece) piece *= 2;
  return piece;
}
int pieces_of(int tokens) { return (tokens + piece_of(tokens) - 1) / piece_of(tokens); }
int most_pieces(int max_tokens) { return std::max(pieces_of(max_tokens), std::min(kFewPieces, (max_tokens + kLeastPiece - 1) / kLeastPiece)); }

// Runs of kManyParts pieces or more stand from the end of the list on.  Their order there is that in which blocks came by; no sum depends on it.
constexpr int kManyParts = 33;
struct Run { uint32_t key; int piece, parts, pad; };
struct Runs { uint32_t count[4]; Run list[1]; };

struct SumsArgs {
  const uint32_t *key, *at;
  const void* dout;
  float* parts;                      // [piece][2][D]: the run that comes from the piece before, and the one that starts here and goes on
  void *table, *rows;
  int64_t ld;
  int tokens, D, vocab, piece;
  uint32_t none;
  float scale;
  Runs* runs;
  int most_runs;                     // that the list holds
  const int32_t* ids;                // few_kernel
  int num_rows;
  int cut, skip;                     // rows [cut, cut + skip) are clear already
  int slices, sum_blocks, clear_blocks, clear_rows;        // sums_kernel: blocks per piece, of sums, and those that clear `clear_rows` rows a wave
};

template <typename T> __device__ __forceinline__ T* row_of(const SumsArgs& a, uint32_t key, float& scale) {
  const bool text = key < (uint32_t)a.vocab;
  scale = text ? a.scale : 1.0f;
  return text ? (T*)a.table + (int64_t)key * a.D : (T*)a.rows + (int64_t)(key - (uint32_t)a.vocab) * a.D;
}

// (tokens whose gradient is not wanted keep their places, so that the others' sums have the same bits in every call)
__device__ __forceinline__ bool wanted(const SumsArgs& a, uint32_t key) { return key < (uint32_t)a.vocab ? a.table != nullptr : key < a.none && a.rows != nullptr; }

// Rows of no token, by a wave, `clear_rows` (up to 64) at a time: its lanes look for as many rows among the sorted keys.
template <typename T> __device__ __forceinline__ void clear_rows(const SumsArgs& a, const uint32_t* sorted, int64_t wave) {
  const int lane = threadIdx.x & 63;
  for (int64_t r0 = wave * a.clear_rows; r0 < (int64_t)a.none - a.skip; r0 += 4ll * a.clear_blocks * a.clear_rows) {
    const int64_t r = r0 + lane;                           // without the rows [cut, cut + skip)
    const uint32_t key = (uint32_t)min(r < a.cut ? r : r + a.skip, (int64_t)a.none);
    int lo = 0, hi = a.tokens;                             // the first token of this key or a later one
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (sorted[mid] < key) lo = mid + 1; else hi = mid;
    }
    uint64_t absent = __ballot(lane < a.clear_rows && key < a.none && wanted(a, key) && (lo >= a.tokens || sorted[min(lo, a.tokens - 1)] != key));
    float zero[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, scale;
    for (; absent; absent &= absent - 1) {
      T* const row = row_of<T>(a, (uint32_t)__builtin_amdgcn_readlane((int)key, __ffsll((unsigned long long)absent) - 1), scale);
      for (int e = lane * 8; e < a.D; e += 512) store8(row + e, a.D - e, zero);
    }
  }
}

// The runs of sorted tokens [first, last), whose last one ends there or leaves a part: rows of the gradient, or partial sums.  e: the
// thread's first column; all lanes of a wave come here, those past the row's end with it.  What decides about a token -- whether its run ends,
// whether it counts -- is made for all of a batch at once by its lanes: read from LDS token by token it took longer than the rows
// (230 rows of one token: 56 us).
//   TINY: rows of fewer than eight elements.  Otherwise the last eight of a row stand in for the ones that would run past it, which two
// threads then write alike, so that no load waits behind a branch: a batch's loads go out together.
template <typename T, typename O, bool TINY, int BATCH>
__device__ __forceinline__ void add_runs(const SumsArgs& a, const uint32_t* key, const uint32_t* at, int first, int last, bool from_before, int piece, int e) {
  const int lane = threadIdx.x & 63;
  if (e - lane * 8 >= a.D || first >= last || (!a.table && key[last - 1] < (uint32_t)a.vocab) || (!a.rows && key[first] >= (uint32_t)a.vocab)) return;
  const bool live = e < a.D;
  const int left = TINY ? a.D : 8;
  e = TINY ? 0 : min(e, a.D - 8);
  float sum[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) sum[i] = 0.f;
  for (int b = first; b < last; b += BATCH) {
    const uint32_t held = key[min(b + lane, last - 1)];
    const uint32_t next = key[min(b + lane, last - 1) + 1];
    const uint64_t ends = __ballot(held != next), counts = __ballot(held < a.none);        // (sorted: those that count stand first)
    const uint32_t row_at = at[min(b + lane, last - 1)];
    float v[BATCH][8];
#pragma unroll
    for (int j = 0; j < BATCH; ++j) {
      const O* const from = (const O*)a.dout + (int64_t)(uint32_t)__builtin_amdgcn_readlane((int)row_at, j) * a.ld + e;
      if constexpr (TINY) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[j][i] = (float)from[min(i, left - 1)];
      } else {
        load8(from, 8, v[j]);
      }
    }
#pragma unroll
    for (int j = 0; j < BATCH; ++j) {
      if (b + j >= last || !(counts >> j & 1)) break;
#pragma unroll
      for (int i = 0; i < 8; ++i) sum[i] += v[j][i];
      if (!(ends >> j & 1) && b + j + 1 < last) continue;
      const uint32_t k = (uint32_t)__builtin_amdgcn_readlane((int)held, j);
      if (wanted(a, k) && live) {
        if ((ends >> j & 1) && !from_before) {
          float scale;
          T* const row = row_of<T>(a, k, scale);
#pragma unroll
          for (int i = 0; i < 8; ++i) sum[i] *= scale;
          store8(row + e, left, sum);
        } else {
          store8(a.parts + ((int64_t)piece * 2 + (from_before ? 0 : 1)) * a.D + e, left, sum);
        }
      }
      from_before = false;
#pragma unroll
      for (int i = 0; i < 8; ++i) sum[i] = 0.f;
    }
    if (!(counts >> (BATCH - 1) & 1)) return;              // what is left has no row
  }
}

// A block's runs are those that start in its piece.  One that ends in the next piece is finished here, beyond the piece's end, and
// passed over there; one that goes on further is `long`: every block adds its own part, for runs_kernel.
template <typename T, typename O, bool TINY> __global__ __launch_bounds__(256) void sums_kernel(SumsArgs a) {
  __shared__ uint32_t keys[3 * kPiece + 2], at[2 * kPiece];            // from the token ahead of the piece before on
  // blocks that clear stand evenly between the others, so that reads and writes go on together
  const int64_t all = gridDim.x;
  const int clear = (int)((int64_t)blockIdx.x * a.clear_blocks / all);
  if ((int)(((int64_t)blockIdx.x + 1) * a.clear_blocks / all) > clear) {
    clear_rows<T>(a, a.key, (int64_t)clear * 4 + (threadIdx.x >> 6));
    return;
  }
  const int block = (int)blockIdx.x - clear, piece = block / a.slices, slice = block - piece * a.slices;
  const int S = a.piece, p0 = piece * S, mine = min(S, a.tokens - p0), more = min(2 * S, a.tokens - p0);
  for (int i = threadIdx.x; i < 3 * S + 2; i += 256) {
    const int p = p0 - S - 1 + i;
    keys[i] = p >= 0 && p < a.tokens ? a.key[p] : 0xffffffffu;
  }
  if ((int)threadIdx.x < more) at[threadIdx.x] = a.at[p0 + (int)threadIdx.x];
  __syncthreads();
  const uint32_t* const key = keys + S + 1;                // of the piece's first token; [-S - 1, 2 S] are there
  const int lane = threadIdx.x & 63;
  const uint32_t here = lane < 2 * S ? key[lane] : 0xffffffffu;
  const bool begun = key[-1] == key[0], goes_on = key[mine - 1] == key[mine], whole = key[mine - 1] == key[0];
  // a run that started before: a part of a long one, or finished by the block before
  bool from_before = begun && (key[-S - 1] == key[0] || (whole && goes_on));
  const int first = begun && !from_before ? min(mine, __ffsll((unsigned long long)~__ballot(here == key[0])) - 1) : 0;
  // one past the last token to add
  int last = mine;
  if (goes_on && !(begun && whole) && key[2 * S] != key[mine - 1]) last += __ffsll((unsigned long long)~(__ballot(here == key[mine - 1]) >> mine)) - 1;
  // a long run that starts here is listed by one wave, which finds its last piece: every lane looks at one of 64 places
  if (goes_on && !(begun && whole) && key[2 * S] == key[mine - 1] && slice == 0 && threadIdx.x < 64) {
    const uint32_t k = key[mine - 1];
    const int pieces = (a.tokens + S - 1) / S;
    int to = piece + 2, end = pieces;
    while (end - to > 1) {
      const int step = (end - to + 63) / 64, p = to + lane * step;
      to += (__popcll(__ballot(p < end && a.key[(int64_t)min(p, end - 1) * S] == k)) - 1) * step;
      end = min(end, to + step);
    }
    if (lane == 0 && wanted(a, k)) {
      const bool many = to - piece + 1 >= kManyParts;
      const int i = (int)atomicAdd(&a.runs->count[many], 1u);
      a.runs->list[many ? a.most_runs - 1 - i : i] = Run{k, piece, to - piece + 1, 0};
    }
  }
  add_runs<T, O, TINY, 8>(a, key, at, first, last, from_before, piece, (slice * 256 + (int)threadIdx.x) * 8);          // (the ballots above need every lane)
}

// Up to kFewTokens tokens: every block sorts them for itself, by how many go before each, so that one launch does for all (100 rows of 382
// 8.2 us, by three launches 15).  Runs are added whole by the wave whose piece they start in, 2.8 us for 16 rows, which is why more tokens
// take the other way: a token that takes most of 256 places, 43 us.
constexpr int kFewTokens = 128;
template <typename T, typename O, bool TINY> __global__ __launch_bounds__(256) void few_kernel(SumsArgs a) {
  __shared__ __attribute__((aligned(16))) uint32_t given[kFewTokens], key[kFewTokens + 1], at[kFewTokens];
  const int tid = threadIdx.x, lane = tid & 63;
  uint32_t mine = 0xffffffffu;
  if (tid < a.tokens) mine = key_of(a.ids[tid], a.vocab, a.num_rows, a.none);
  if (tid < kFewTokens) given[tid] = mine;
  key[a.tokens] = 0xffffffffu;
  __syncthreads();
  int place = 0;
#pragma unroll 8
  for (int i = 0; i < a.tokens; i += 4) {                  // (what stands past the last token goes before nothing)
    const uint4 k = *(const uint4*)(given + i);
    place += (k.x < mine || (k.x == mine && i < tid)) + (k.y < mine || (k.y == mine && i + 1 < tid)) + (k.z < mine || (k.z == mine && i + 2 < tid)) +
             (k.w < mine || (k.w == mine && i + 3 < tid));
  }
  if (tid < a.tokens) { key[place] = mine; at[place] = (uint32_t)tid; }
  __syncthreads();
  const int clear = (int)((int64_t)blockIdx.x * a.clear_blocks / gridDim.x);
  if ((int)(((int64_t)blockIdx.x + 1) * a.clear_blocks / gridDim.x) > clear) {
    clear_rows<T>(a, key, (int64_t)clear * 4 + (tid >> 6));
    return;
  }
  // 512 columns of a piece a wave (2048 a block leave a token that takes most places to two units of the chip: 54 us for 230 rows of 3200)
  const int item = ((int)blockIdx.x - clear) * 4 + (tid >> 6), piece = item / a.slices, slice = item - piece * a.slices;
  if (piece * a.piece >= a.tokens) return;
  auto end_of = [&](int p) {                               // of the run that holds sorted token p; every lane looks at one of 64 tokens
    const uint32_t k = key[p];
    for (;;) {
      const uint64_t other = __ballot(key[min(p + lane, a.tokens)] != k);
      if (other) return p + __ffsll((unsigned long long)other) - 1;
      p += 64;
    }
  };
  int first = piece * a.piece, last = min(first + a.piece, a.tokens);
  const bool begun = first > 0 && key[first - 1] == key[first];
  last = end_of(last - 1);
  if (begun) first = end_of(first);
  // (a run over the whole piece that started before leaves first = last)
  add_runs<T, O, TINY, TINY ? 8 : 16>(a, key, at, first, last, false, piece, (slice * 64 + lane) * 8);
}

// Long runs, those over three pieces or more, as sums_kernel listed them: the parts of one, some columns a block, groups of threads in
// turn.  Most have a few parts: eight groups for 512 columns; from kManyParts on 64 for 64, so that a token that takes most places is spread
// over the chip (29 500 of 32 768 tokens, 3200 columns: 56 us by eight groups).
template <typename T, bool TINY> __global__ __launch_bounds__(512) void runs_kernel(SumsArgs a) {
  __shared__ float part[512 * 8];
  const int few = (int)a.runs->count[0], many = (int)a.runs->count[1];
  const int few_cols = (a.D + 511) / 512, many_cols = (a.D + 63) / 64;
  const int64_t items = (int64_t)few * few_cols + (int64_t)many * many_cols;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const bool is_few = item < (int64_t)few * few_cols;
    const int64_t i = is_few ? item : item - (int64_t)few * few_cols;
    const int cols = is_few ? few_cols : many_cols, run = (int)(i / cols), slice = (int)(i - (int64_t)run * cols);
    const Run r = is_few ? a.runs->list[run] : a.runs->list[a.most_runs - 1 - run];
    const int lanes = is_few ? 64 : 8, G = 512 / lanes, lane = threadIdx.x & (lanes - 1), g = threadIdx.x / lanes;
    const int c0 = slice * lanes * 8, at = c0 + lane * 8, e = TINY ? at : min(at, a.D - 8), left = TINY ? a.D - at : 8;      // see sums_kernel
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = 0.f;
    if (at < a.D) {
      constexpr int BATCH = 4;
      for (int p = g; p < r.parts; p += G * BATCH) {
        float u[BATCH][8];
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
          const int q = min(p + G * b, r.parts - 1);
          load8(a.parts + ((int64_t)(r.piece + q) * 2 + (q ? 0 : 1)) * a.D + e, left, u[b]);
        }
#pragma unroll
        for (int b = 0; b < BATCH; ++b)
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] += p + G * b < r.parts ? u[b][j] : 0.f;
      }
      // (the shifted window of a row's last threads writes the columns that they share alike)
#pragma unroll
      for (int j = 0; j < 8; ++j) if (e + j - c0 >= 0 && j < left) part[g * lanes * 8 + e + j - c0] = v[j];
    }
    __syncthreads();
    const int c = c0 + (int)threadIdx.x;
    if ((int)threadIdx.x < lanes * 8 && c < a.D) {
      float sum = part[threadIdx.x], scale;
      for (int j = 1; j < G; ++j) sum += part[j * lanes * 8 + threadIdx.x];
      T* const row = row_of<T>(a, r.key, scale);
      row[c] = (T)(sum * scale);
    }
    __syncthreads();
  }
}

epd_status check_cfg(const char* who, const epd_embed_cfg* c) {
  if (!c) return op_fail(EPD_ERR_INVALID_ARG, "%s: cfg is NULL", who);
  if (c->struct_size != sizeof(epd_embed_cfg)) return op_fail(EPD_ERR_INVALID_ARG, "%s: cfg.struct_size %u != %zu", who, c->struct_size, sizeof(epd_embed_cfg));
  if (!known_dtype(c->dtype) || !known_dtype(c->out_dtype)) return op_fail(EPD_ERR_INVALID_ARG, "%s: dtype or out_dtype invalid", who);
  if (c->dtype == EPD_F32 && c->out_dtype != EPD_F32) return op_fail(EPD_ERR_UNSUPPORTED, "%s: an fp32 table has fp32 rows", who);
  if (c->vocab < 1 || c->vocab > kEmbedRows) return op_fail(EPD_ERR_UNSUPPORTED, "%s: vocab %d: 1 .. 2^30", who, c->vocab);
  if (c->hidden < 1 || c->hidden > kEmbedDim) return op_fail(EPD_ERR_UNSUPPORTED, "%s: hidden %d: 1 .. %d", who, c->hidden, kEmbedDim);
  if (c->max_tokens < 1 || c->max_tokens > kEmbedTokens) return op_fail(EPD_ERR_UNSUPPORTED, "%s: max_tokens %d: 1 .. 2^24", who, c->max_tokens);
  if ((int64_t)c->max_tokens * c->hidden > kEmbedElements) return op_fail(EPD_ERR_UNSUPPORTED, "%s: max_tokens * hidden %lld: up to 2^38", who, (long long)c->max_tokens * c->hidden);
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

struct EmbedLayout { size_t list, parts, runs, total; };   // bytes: key and at, twice, the partial sums, and the long runs
int most_runs(int pieces) { return pieces / 2 + 1; }       // a long run covers the piece behind its first one
EmbedLayout embed_layout(const epd_embed_cfg& c) {
  EmbedLayout L;
  auto up = [](size_t v) { return (v + 255) / 256 * 256; };
  L.list = up((size_t)c.max_tokens * 4);
  L.parts = 4 * L.list;
  L.runs = up(L.parts + (size_t)most_pieces(c.max_tokens) * 2 * c.hidden * 4);
  L.total = up(L.runs + sizeof(Runs) + (size_t)most_runs(most_pieces(c.max_tokens)) * sizeof(Run));
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
  EmbedArgs a{table, rows, ids, out, ld_out, tokens, c.hidden, c.vocab, num_rows, c.scale, writes_through(out, ld_out, c.out_dtype == EPD_F32 ? 4 : 2)};
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

  const uint32_t none = (uint32_t)c.vocab + (uint32_t)num_rows;
  const int pieces = tokens ? pieces_of(tokens) : 0;
  Runs* const runs = (Runs*)(ws + L.runs);
  SumsArgs a{key, at, dout, (float*)(ws + L.parts), dtable, drows, ld_dout, tokens, c.hidden, c.vocab, tokens ? piece_of(tokens) : 0, none, c.scale};
  a.runs = runs; a.most_runs = most_runs(pieces);
  a.ids = ids; a.num_rows = num_rows;
  a.slices = (c.hidden + 2047) / 2048;
  a.sum_blocks = pieces * a.slices;
  // rows a wave clears: 64 KB, fewer while that leaves waves of the chip idle
  a.clear_rows = (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(64, 65536 / ((int64_t)c.hidden * es)), none / 1024));
  a.clear_blocks = (int)std::min<int64_t>(kMaxGrid, ((int64_t)none + 4 * a.clear_rows - 1) / (4 * a.clear_rows));
  void* args[] = {(void*)&a};
  if (tokens && tokens <= kFewTokens) {
    a.slices = (c.hidden + 511) / 512;
    a.sum_blocks = (pieces * a.slices + 3) / 4;
    const hipError_t e = by_types(c, [&](auto t, auto o) {
      typedef decltype(t) T;
      typedef decltype(o) O;
      return hipLaunchKernel(c.hidden < 8 ? (const void*)few_kernel<T, O, true> : (const void*)few_kernel<T, O, false>, dim3(a.sum_blocks + a.clear_blocks), dim3(256), args, 0, st);
    });
    return e == hipSuccess ? EPD_OK : op_launch_failed(who, e);
  }
  // Which launch clears the gradients: rows beside the sort, which leaves most of the chip idle, or the rows of no token beside the sums.
  // The former writes rows of tokens twice.  All rows where the tokens' are few; otherwise as many of the table's last rows as the sort
  // hides (32 768 tokens, 131 072 x 3200: 298 us without these, 288 with).
  const bool clear_all = (int64_t)tokens * c.hidden * es <= kClearAll;
  SortArgs s{};
  s.counts = runs->count;
  s.ids = ids; s.key = key; s.at = at; s.tokens = tokens; s.vocab = c.vocab; s.num_rows = num_rows; s.none = none;
  int bits = 1;
  while ((uint64_t)none >> bits) ++bits;
  s.passes = (bits + kMaxDigit - 1) / kMaxDigit;
  s.bits = std::max(6, (bits + s.passes - 1) / s.passes);
  s.sort_blocks = (tokens + kSortList - 1) / kSortList;
  auto clears = [&](int j, void* p, int64_t n) { if (p) { s.clear[j] = p; s.pieces[j] = n * es / 16; s.tail[j] = (int)(n * es % 16); } };
  if (clear_all) {
    clears(0, dtable, (int64_t)c.vocab * c.hidden);
    clears(1, drows, (int64_t)num_rows * c.hidden);
    a.clear_blocks = 0;
  } else if (dtable) {
    a.skip = (int)std::min<int64_t>(c.vocab, kClearBesideSort / ((int64_t)c.hidden * es));
    a.cut = c.vocab - a.skip;
    clears(0, (char*)dtable + (int64_t)a.cut * c.hidden * es, (int64_t)a.skip * c.hidden);
  }
  const int clear_blocks = !s.pieces[0] && !s.pieces[1] && !s.tail[0] && !s.tail[1] ? 0 : (int)std::max<int64_t>(1, std::min<int64_t>(1024, (s.pieces[0] + s.pieces[1]) / 8192));
  void* sargs[] = {(void*)&s};
  hipError_t e = hipLaunchKernel((const void*)sort_kernel, dim3(s.sort_blocks + clear_blocks), dim3(1024), sargs, 0, st);
  for (int64_t len = kSortList; e == hipSuccess && len < tokens; len *= kMergeLists) {
    MergeArgs m{key, at, key2, at2, tokens, (int)len};
    void* margs[] = {(void*)&m};
    e = hipLaunchKernel((const void*)merge_kernel, dim3((tokens + 255) / 256), dim3(256), margs, 0, st);
    std::swap(key, key2);
    std::swap(at, at2);
  }
  a.key = key; a.at = at;
  if (e == hipSuccess && tokens)
    e = by_types(c, [&](auto t, auto o) {
      typedef decltype(t) T;
      typedef decltype(o) O;
      return hipLaunchKernel(c.hidden < 8 ? (const void*)sums_kernel<T, O, true> : (const void*)sums_kernel<T, O, false>, dim3(a.sum_blocks + a.clear_blocks), dim3(256), args, 0, st);
    });
  if (e == hipSuccess && pieces > 2)
    e = by_types(c, [&](auto t, auto) {
      typedef decltype(t) T;
      return hipLaunchKernel(c.hidden < 8 ? (const void*)runs_kernel<T, true> : (const void*)runs_kernel<T, false>,
                             dim3((int)std::min<int64_t>(1024, (int64_t)a.most_runs * ((c.hidden + 63) / 64))), dim3(512), args, 0, st);
    });
  return e == hipSuccess ? EPD_OK : op_launch_failed(who, e);
}

}  // extern "C"
