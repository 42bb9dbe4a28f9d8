// Embedding lookup with scaling, and its gradient by sorted tokens.
//
//   out_t = scale E[id_t];  dE_v = scale sum over t with id_t = v of dx_t
//
// Both are bound by memory: the lookup reads a row and writes one for each
// token, the gradient reads each token's row once and writes every row of the
// table once, zeros for words that do not occur (no separate clearing pass).
// An id outside [0, vocab) is padding: its row is zero and it gives no gradient.
//
// The gradient first sorts the tokens by id, stably, so that a word's tokens
// stand together in the order of the batch, and then gives each table row to
// one wave (of each slice of columns), which adds its tokens in 32 bits in that
// order: no atomics, the same bits every time.  Words follow Zipf's law, so one may
// have a tenth of all tokens: every kChunk tokens of a word are summed beforehand
// by a wave of their own, and the row adds these sums and what is left.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "cel_internal.h"

namespace cel {
namespace {

constexpr int kChunk = 32;       // sorted tokens of one partial sum
constexpr int kDigit = 9;        // bits of an id sorted at once: two passes up to 262,143 words
constexpr int kBins = 1 << kDigit;
constexpr int kSortB = 1024, kSortW = kSortB / 64;
constexpr int kRankMost = 8192;  // tokens that are ranked against each other, at most
constexpr int kRankB = 256, kRankEach = 16, kRankTokens = kRankB / kRankEach;  // threads, threads a token, tokens
constexpr int kSlice = 512;      // columns a wave handles
constexpr int kTogether = 4;     // rows of the lookup that a wave has on their way at once
constexpr int kRowsAt = 4;       // table rows a wave writes one behind the other,
constexpr int64_t kFewRows = 16384;  // unless there are at most this many pieces of rows, see k_embed_grad

// A launch has fewer than 2^32 threads along x: workgroups beyond kGridX stand in further rows of
// the grid.  The last row's surplus has nothing to do.
constexpr int64_t kGridX = 1 << 23;
__device__ inline int64_t block_number() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

// BYTES at any address of the element type, as one access.
template <int BYTES>
struct __attribute__((packed, aligned(2))) Raw {
  uint32_t w[BYTES / 4];
};
// A wave's kSlice columns are S chunks of 64 lanes with E values each; E values
// of the rows written are 16 bytes.
template <class O>
struct Shape {
  static constexpr int E = 16 / sizeof(O), S = kSlice / 64 / E;
};
template <class T, int E>
__device__ inline Raw<E * sizeof(T)> load_raw(const T *p, int64_t left) {
  Raw<E * sizeof(T)> r{};
  if (left >= E) {
    r = *reinterpret_cast<const Raw<E * sizeof(T)> *>(p);
  } else {
    T x[E];
#pragma unroll
    for (int e = 0; e < E; e++) x[e] = e < left ? p[e] : (T)0.f;
    __builtin_memcpy(&r, x, sizeof r);
  }
  return r;
}
template <class T, int E>
__device__ inline void values(float (&f)[E], const Raw<E * sizeof(T)> &r) {
  T x[E];
  __builtin_memcpy(x, &r, sizeof r);
#pragma unroll
  for (int e = 0; e < E; e++) f[e] = (float)x[e];
}
// NT: past the caches.  An output larger than the memory-side cache (256 MiB)
// would only push out what is read again (lookup of 32,768 rows of 8,192: 126 us
// against 221); a smaller one is still there when it is used next (gradient of
// 50,001 rows of 1,024 in 32 bits: 55 us against 65).
constexpr int64_t kCached = int64_t(256) << 20;
template <class O, int E, bool NT>
__device__ inline void store_values(O *p, const float (&f)[E], float by, int64_t left) {
  O x[E];
#pragma unroll
  for (int e = 0; e < E; e++) x[e] = (O)(f[e] * by);
  if (left >= E) {
    Raw<E * sizeof(O)> r;
    __builtin_memcpy(&r, x, sizeof r);
    if constexpr (NT) {
      typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
      typedef __attribute__((ext_vector_type(4), aligned(2))) uint32_t any_u32x4;
      static_assert(sizeof r == 16, "whole stores");
      __builtin_nontemporal_store(__builtin_bit_cast(u32x4, r), reinterpret_cast<any_u32x4 *>(p));
    } else {
      *reinterpret_cast<Raw<E * sizeof(O)> *>(p) = r;
    }
  } else {
#pragma unroll
    for (int e = 0; e < E; e++)
      if (e < left) p[e] = x[e];
  }
}

// A wave takes kTogether tokens and kSlice columns of their rows: every load is
// on its way before the first store.  Bound by memory: 32,768 rows of 8,192 from
// a table of 131,072 words, 16 bits: 118 us, 537 MB written at 4.6 TB/s, with the
// reads of frequent words answered by the caches.  512 rows of 1,024: 4 us, a launch.
template <class T, class I, bool NT>
__global__ void __launch_bounds__(256) k_embed(const T *table, int64_t stride, int64_t vocab, const I *ids, int64_t tokens,
                                               int64_t h, int slices, float scale, T *out) {
  constexpr int E = Shape<T>::E, S = Shape<T>::S;
  const int64_t task = block_number() * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t t0 = task / slices * kTogether, c0 = (task % slices) * kSlice + (threadIdx.x & 63) * E;
  if (t0 >= tokens) return;
  Raw<16> r[kTogether][S];
#pragma unroll
  for (int k = 0; k < kTogether; k++) {
    const int64_t id = t0 + k < tokens ? (int64_t)ids[t0 + k] : -1;
    const bool in = id >= 0 && id < vocab;
#pragma unroll
    for (int u = 0; u < S; u++) {
      const int64_t c = c0 + u * 64 * E;
      r[k][u] = in && c < h ? load_raw<T, E>(table + id * stride + c, h - c) : Raw<16>{};
    }
  }
#pragma unroll
  for (int k = 0; k < kTogether; k++) {
    if (t0 + k >= tokens) break;
#pragma unroll
    for (int u = 0; u < S; u++) {
      const int64_t c = c0 + u * 64 * E;
      float f[E];
      values<T, E>(f, r[k][u]);
      if (c < h) store_values<T, E, NT>(out + (t0 + k) * h + c, f, scale, h - c);
    }
  }
}

// ---------------------------------------------------------- sort by token id
__device__ inline uint32_t digit_of(uint32_t key, int shift) { return (key >> shift) & (kBins - 1); }
template <class I>
__device__ inline uint32_t key_of(const I *ids, int64_t t, int64_t vocab) {
  const int64_t id = ids[t];
  return id >= 0 && id < vocab ? (uint32_t)id : (uint32_t)vocab;
}

// The lanes whose digit equals this lane's, among those that take part.
__device__ inline uint64_t same_digit(uint32_t digit, bool in) {
  uint64_t m = __ballot(in);
#pragma unroll
  for (int b = 0; b < kDigit; b++) {
    const bool bit = (digit >> b) & 1;
    const uint64_t v = __ballot(bit);
    m &= bit ? v : ~v;
  }
  return m;
}
// Counts this lane's digit in its wave's column of counters and returns how
// many tokens before it, in the wave's order, had the same.
__device__ inline uint32_t rank_in_wave(uint32_t (*count)[kSortW + 1], int wave, int lane, uint32_t digit, bool in) {
  const uint64_t m = same_digit(digit, in);
  uint32_t before = 0;
  if (in) before = count[digit][wave];
  lds_order();
  if (in && __builtin_ctzll(m) == lane) count[digit][wave] = before + (uint32_t)__builtin_popcountll(m);
  lds_order();
  return before + (uint32_t)__builtin_popcountll(m & ((uint64_t(1) << lane) - 1));
}
// Turns every digit's counts into where each wave's tokens of it begin: base, and the waves before.
__device__ inline void start_counts(uint32_t (*count)[kSortW + 1], const uint32_t *base, int tid) {
  if (tid < kBins) {
    uint32_t at = base[tid];
#pragma unroll
    for (int w = 0; w < kSortW; w++) {
      const uint32_t x = count[tid][w];
      count[tid][w] = at;
      at += x;
    }
  }
  __syncthreads();
}

// Few tokens: every token's place is the number of tokens that come before it,
// counted against all of them, kRankEach threads a token.  Tokens squared
// comparisons, but one launch and no dependent passes: 4,096 tokens in 11 us and 8,192
// in 21, where the sort below takes 25 and 26 us; 8,193 in 33 and 16,384 in 69, where it
// takes 28 and 29 us.  Bound by the reads of LDS.
template <class I>
__global__ void __launch_bounds__(kRankB) k_embed_rank(const I *ids, int tokens, int64_t vocab, uint32_t *keys,
                                                       uint32_t *order) {
  __shared__ __align__(16) uint32_t s_key[kRankMost];
  const int tid = threadIdx.x;
  for (int t0 = tid; t0 < (tokens + 3) / 4 * 4; t0 += 8 * kRankB) {
    uint32_t k[8];
#pragma unroll
    for (int u = 0; u < 8; u++) k[u] = t0 + u * kRankB < tokens ? key_of(ids, t0 + u * kRankB, vocab) : ~0u;
#pragma unroll
    for (int u = 0; u < 8; u++)
      if (t0 + u * kRankB < kRankMost) s_key[t0 + u * kRankB] = k[u];
  }
  __syncthreads();
  const int t = blockIdx.x * kRankTokens + tid / kRankEach, part = tid % kRankEach;
  const uint32_t key = t < tokens ? s_key[t] : 0;
  uint32_t before = 0;
  // up to three entries behind the last token are read, larger than any key
#pragma unroll 8
  for (int i = 4 * part; i < tokens; i += 4 * kRankEach) {
    const uint4 k = *reinterpret_cast<const uint4 *>(&s_key[i]);
    before += (k.x < key + (i < t)) + (k.y < key + (i + 1 < t)) + (k.z < key + (i + 2 < t)) + (k.w < key + (i + 3 < t));
  }
#pragma unroll
  for (int o = 1; o < kRankEach; o <<= 1) before += __shfl_xor(before, o);
  if (t < tokens && part == 0) {
    keys[before] = key;
    order[before] = t;
  }
}

// Many tokens: a radix sort by several workgroups, each of which holds `tile`
// tokens (a multiple of 2 kSortB): a pass counts digits per tile (table [tiles][kBins]),
// and then puts every token in its place.  first: from ids, else from keys.
// Bound by latency: 32,768 tokens, 4.6 and 10.6 us a pass.
template <class I>
__global__ void __launch_bounds__(kSortB) k_embed_count(const I *ids, const uint32_t *keys, bool first, int64_t tokens,
                                                        int64_t vocab, int64_t tile, int shift, uint32_t *table) {
  __shared__ uint32_t count[kBins];
  const int tid = threadIdx.x;
  if (tid < kBins) count[tid] = 0;
  __syncthreads();
  const int64_t t0 = blockIdx.x * tile, t1 = min(tokens, t0 + tile);
  for (int64_t t = t0 + tid; t < t1; t += kSortB)
    atomicAdd(&count[digit_of(first ? key_of(ids, t, vocab) : keys[t], shift)], 1u);
  __syncthreads();
  if (tid < kBins) table[(int64_t)blockIdx.x * kBins + tid] = count[tid];
}
template <class I>
__global__ void __launch_bounds__(kSortB) k_embed_move(const I *ids, const uint32_t *keys, const uint32_t *order, bool first,
                                                       int64_t tokens, int64_t vocab, int64_t tile, int shift,
                                                       const uint32_t *table, uint32_t *keys_to, uint32_t *order_to) {
  __shared__ uint32_t count[kBins][kSortW + 1];  // one more: a digit's counters start in different banks
  __shared__ uint32_t s_base[kBins], s_sum[kSortW];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint32_t all = 0, before = 0;
  if (tid < kBins) {
    for (int b = 0; b < (int)gridDim.x; b++) {
      const uint32_t x = table[(int64_t)b * kBins + tid];
      if (b < (int)blockIdx.x) before += x;
      all += x;
    }
  }
  uint32_t up = all;
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t y = __shfl_up(up, o);
    if (lane >= o) up += y;
  }
  if (lane == 63) s_sum[wave] = up;
  __syncthreads();
  if (tid < kBins) {
    for (int w = 0; w < wave; w++) up += s_sum[w];
    s_base[tid] = up - all + before;
  }
  const int64_t t0 = blockIdx.x * tile, t1 = min(tokens, t0 + tile);
  for (int64_t at = t0; at < t1; at += 2 * kSortB) {  // two tokens a thread at once, in the waves' order
    for (int i = tid; i < kBins * (kSortW + 1); i += kSortB) (&count[0][0])[i] = 0;
    __syncthreads();
    uint32_t key[2] = {0, 0}, pos[2] = {0, 0}, rank[2];
#pragma unroll
    for (int u = 0; u < 2; u++) {
      const int64_t t = at + wave * 128 + u * 64 + lane;
      if (t < t1) {
        key[u] = first ? key_of(ids, t, vocab) : keys[t];
        pos[u] = first ? (uint32_t)t : order[t];
      }
    }
#pragma unroll
    for (int u = 0; u < 2; u++)
      rank[u] = rank_in_wave(count, wave, lane, digit_of(key[u], shift), at + wave * 128 + u * 64 + lane < t1);
    __syncthreads();
    uint32_t sum = 0;
    if (tid < kBins) {
#pragma unroll
      for (int w = 0; w < kSortW; w++) sum += count[tid][w];
    }
    start_counts(count, s_base, tid);
#pragma unroll
    for (int u = 0; u < 2; u++) {
      if (at + wave * 128 + u * 64 + lane >= t1) continue;
      const uint32_t to = count[digit_of(key[u], shift)][wave] + rank[u];
      keys_to[to] = key[u];
      order_to[to] = pos[u];
    }
    __syncthreads();
    if (tid < kBins) s_base[tid] += sum;
  }
}

// ------------------------------------------------------------ sums by word
// Rows row_of(t) of dx for t in [a, b), added in order to the lane's columns,
// kAtOnce of them on their way at a time.
template <class T, int E, int S, class Row>
__device__ inline void add_rows(float (&f)[S][E], const T *dx, int64_t stride, int64_t a, int64_t b, int64_t c0, int64_t h,
                                Row row_of) {
  constexpr int kAtOnce = 4;
  for (int64_t t = a; t < b; t += kAtOnce) {
    Raw<E * sizeof(T)> r[kAtOnce][S];
#pragma unroll
    for (int k = 0; k < kAtOnce; k++) {
      const T *row = dx + row_of(t + k < b ? t + k : b - 1) * stride;
#pragma unroll
      for (int u = 0; u < S; u++) {
        const int64_t c = c0 + u * 64 * E;
        if (t + k < b && c < h) r[k][u] = load_raw<T, E>(row + c, h - c);
      }
    }
#pragma unroll
    for (int k = 0; k < kAtOnce; k++)
#pragma unroll
      for (int u = 0; u < S; u++) {
        if (t + k >= b || c0 + u * 64 * E >= h) continue;
        float x[E];
        values<T, E>(x, r[k][u]);
#pragma unroll
        for (int e = 0; e < E; e++) f[u][e] += x[e];
      }
  }
}

// Blocks below `searches`: where each word's tokens begin (start [vocab + 1]).
// The others: the sums of the words' full chunks (part [tokens / kChunk][h]; a
// word's chunks are counted from its first token, so that its sum depends on no
// other word, and chunk p of a word that begins at a lies at a / kChunk + p).
// A wave's chain is one chunk's reads and two short searches: 32,768 tokens of
// 8,192 values in 47 us, 190 MB (4.1 TB/s); 4,096 of 1,024 in 13 us, by latency.
template <class T>
__global__ void __launch_bounds__(256) k_embed_parts(const uint32_t *__restrict__ keys, const uint32_t *__restrict__ order,
                                                     int64_t tokens, int64_t vocab, int searches, uint32_t *start, const T *dx,
                                                     int64_t stride, int64_t h, int slices, float *part) {
  const int64_t block = block_number();
  if (block < searches) {
    const int64_t v = block * 256 + threadIdx.x;
    if (v > vocab) return;
    int64_t lo = 0, hi = tokens;
    while (lo < hi) {
      const int64_t mid = (lo + hi) >> 1;
      if (keys[mid] < (uint32_t)v) lo = mid + 1;
      else hi = mid;
    }
    start[v] = (uint32_t)lo;
    return;
  }
  constexpr int E = Shape<float>::E, S = Shape<float>::S;
  const int64_t task = (block - searches) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // The chunk that begins among the kChunk tokens from w on, if there is one,
  // reaches past the last of them, and holds one kChunk / 2 further or nearer too.
  const int64_t chunk = task / slices, w = chunk * kChunk;
  if (w + kChunk > tokens) return;
  const uint32_t key = keys[w + kChunk - 1];
  if (key >= (uint32_t)vocab || (keys[w + kChunk / 2 - 1] != key &&
                                 (w + kChunk * 3 / 2 > tokens || keys[w + kChunk * 3 / 2 - 1] != key)))
    return;
  int64_t a = 0, hi = w + kChunk - 1;  // where the word begins
  while (a < hi) {
    const int64_t mid = (a + hi) >> 1;
    if (keys[mid] < key) a = mid + 1;
    else hi = mid;
  }
  const int64_t t0 = a >= w ? a : w + (a - w) % kChunk + (((a - w) % kChunk) ? kChunk : 0);
  if (t0 + kChunk > tokens || keys[t0 + kChunk - 1] != key) return;
  const int64_t c0 = (task % slices) * kSlice + (threadIdx.x & 63) * E;
  float f[S][E] = {};
  add_rows<T, E, S>(f, dx, stride, t0, t0 + kChunk, c0, h, [&](int64_t t) { return (int64_t)order[t]; });
#pragma unroll
  for (int u = 0; u < S; u++) {
    const int64_t c = c0 + u * 64 * E;
    if (c < h) store_values<float, E, false>(part + chunk * h + c, f[u], 1.f, h - c);
  }
}

// A wave takes `rows` rows of the table and kSlice of their columns: one where the
// pieces are few, so that no wave adds several frequent words while others are done (1,000
// rows of 64, 8,192 tokens: 24 -> 14 us, 32,768 tokens 50 -> 35; at 16,000 pieces the two are within
// 7 % of each other), else kRowsAt (131,072 rows of 8,192: 607 us one by one, 480 so).  Bound by memory:
// 131,072 rows of 8,192 from 32,768 tokens, 16 bits: 480 us, 2.5 GB at 5.2 TB/s; 50,001 rows
// of 1,024 in 32 bits from 4,096: 32 us into memory that was written just before, 10 us more
// into other (205 MB, of which the memory-side cache may hold the one).  Eight rows of dx on their way
// instead of four take more registers and leave fewer waves: 724 us for the first.
template <class T, class O, bool NT>
__global__ void __launch_bounds__(256) k_embed_grad(const uint32_t *start, const uint32_t *__restrict__ order, int64_t vocab,
                                                    const T *dx, int64_t stride, int64_t h, int slices,
                                                    const float *__restrict__ part, float scale, int rows, O *grad) {
  constexpr int E = Shape<O>::E, S = Shape<O>::S;
  const int lane = threadIdx.x & 63;
  const int64_t task = block_number() * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t v0 = task / slices * rows;
  if (v0 >= vocab) return;
  const int64_t c0 = (task % slices) * kSlice + lane * E;
  const uint32_t at = lane <= rows && v0 + lane <= vocab ? start[v0 + lane] : 0;
#pragma unroll 1
  for (int r = 0; r < rows && v0 + r < vocab; r++) {
    const int64_t a = (uint32_t)__builtin_amdgcn_readlane(at, r), b = (uint32_t)__builtin_amdgcn_readlane(at, r + 1);
    float f[S][E] = {};
    if (a < b) {
      const int64_t chunks = (b - a) / kChunk;
      add_rows<float, E, S>(f, part, h, a / kChunk, a / kChunk + chunks, c0, h, [](int64_t p) { return p; });
      add_rows<T, E, S>(f, dx, stride, a + chunks * kChunk, b, c0, h, [&](int64_t t) { return (int64_t)order[t]; });
    }
#pragma unroll
    for (int u = 0; u < S; u++) {
      const int64_t c = c0 + u * 64 * E;
      if (c < h) store_values<O, E, NT>(grad + (v0 + r) * h + c, f[u], scale, h - c);
    }
  }
}

// ------------------------------------------------------------- entry points
// Scratch of cel_embed_grad: start [vocab + 1], keys and order twice, the
// digit table, and the chunks' sums.
constexpr int64_t kTiles = 128;  // workgroups of a sort, at most
struct Plan {
  int64_t tiles, tile;
  int bits;
  int64_t start, keys[2], order[2], table, part, bytes;
};
Plan plan_of(int64_t tokens, int64_t vocab, int64_t h) {
  Plan p{};
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    const int64_t x = at;
    at += (bytes + 255) / 256 * 256;
    return x;
  };
  while (p.bits < 32 && (vocab >> p.bits) != 0) p.bits++;
  p.tile = (std::max((tokens + kTiles - 1) / kTiles, (int64_t)1) + 2 * kSortB - 1) / (2 * kSortB) * (2 * kSortB);
  p.tiles = (tokens + p.tile - 1) / p.tile;
  p.start = take(4 * (vocab + 1));
  for (int i = 0; i < 2; i++) p.keys[i] = take(4 * tokens), p.order[i] = take(4 * tokens);
  p.table = take(4 * kBins * p.tiles);
  p.part = take(4 * (tokens / kChunk) * h);
  p.bytes = at;
  return p;
}
int check_embed(const cel_embed_args *a, const char *fn) {
  if (!a) return set_error(CEL_E_ARG, "%s: NULL descriptor", fn);
  if (a->type < CEL_BF16 || a->type > CEL_F32) return set_error(CEL_E_ARG, "%s: type %d", fn, a->type);
  if (a->id_bytes != 4 && a->id_bytes != 8) return set_error(CEL_E_ARG, "%s: ids of %d bytes", fn, a->id_bytes);
  if (a->tokens < 0 || a->tokens > INT32_MAX || a->vocab < 1 || a->vocab > INT32_MAX - 1 || a->hidden < 1 ||
      a->hidden > (1 << 24))
    return set_error(CEL_E_ARG, "%s: %lld tokens, %lld words, rows of %lld", fn, (long long)a->tokens, (long long)a->vocab,
                     (long long)a->hidden);
  if (a->stride < a->hidden || a->stride > (int64_t(1) << 40))
    return set_error(CEL_E_ARG, "%s: rows of %lld values %lld apart", fn, (long long)a->hidden, (long long)a->stride);
  if (a->tokens && !a->ids) return set_error(CEL_E_ARG, "%s: ids is NULL", fn);
  if (!std::isfinite(a->scale)) return set_error(CEL_E_ARG, "%s: scale %g", fn, (double)a->scale);
  return CEL_OK;
}
int slices_of(const cel_embed_args *a) {
  return (int)((a->hidden + kSlice - 1) / kSlice);
}
int grid_of(int64_t waves, const char *fn, dim3 *grid) {
  const int64_t b = (waves + 3) / 4, rows = (b + kGridX - 1) / kGridX;
  if (rows > 65535) return set_error(CEL_E_ARG, "%s: too large a call", fn);
  *grid = dim3((unsigned)std::min(b, kGridX), (unsigned)rows);
  return CEL_OK;
}

template <class T>
int embed(const cel_embed_args *a, const void *table, void *out, hipStream_t s) {
  const int slices = slices_of(a);
  dim3 grid;
  CEL_TRY(grid_of((a->tokens + kTogether - 1) / kTogether * slices, "cel_embed", &grid));
  KTimer kt(s, "k_embed");
  auto go = [&](auto id, auto nt) {
    typedef decltype(id) I;
    k_embed<T, I, decltype(nt)::value><<<grid, 256, 0, s>>>((const T *)table, a->stride, a->vocab, (const I *)a->ids,
                                                            a->tokens, a->hidden, slices, a->scale, (T *)out);
  };
  const bool nt = a->tokens * a->hidden * (int64_t)sizeof(T) > kCached;
  if (a->id_bytes == 4) nt ? go(int32_t{}, std::true_type{}) : go(int32_t{}, std::false_type{});
  else nt ? go(int64_t{}, std::true_type{}) : go(int64_t{}, std::false_type{});
  CEL_HIP(hipGetLastError());
  return CEL_OK;
}

template <class I>
int sort_tokens(const cel_embed_args *a, const Plan &p, char *w, int *in, hipStream_t s) {
  const I *ids = (const I *)a->ids;
  auto u32 = [&](int64_t at) { return reinterpret_cast<uint32_t *>(w + at); };
  *in = 0;
  if (a->tokens == 0) return CEL_OK;
  if (a->tokens <= kRankMost) {
    KTimer kt(s, "k_embed_rank");
    k_embed_rank<I><<<(unsigned)((a->tokens + kRankTokens - 1) / kRankTokens), kRankB, 0, s>>>(
        ids, (int)a->tokens, a->vocab, u32(p.keys[0]), u32(p.order[0]));
    CEL_HIP(hipGetLastError());
    return CEL_OK;
  }
  for (int shift = 0; shift < p.bits; shift += kDigit) {
    const int from = *in, to = from ^ 1;
    KTimer kt(s, "k_embed_sort");
    k_embed_count<I><<<(unsigned)p.tiles, kSortB, 0, s>>>(ids, u32(p.keys[from]), shift == 0, a->tokens, a->vocab, p.tile,
                                                          shift, u32(p.table));
    k_embed_move<I><<<(unsigned)p.tiles, kSortB, 0, s>>>(ids, u32(p.keys[from]), u32(p.order[from]), shift == 0, a->tokens,
                                                         a->vocab, p.tile, shift, u32(p.table), u32(p.keys[to]),
                                                         u32(p.order[to]));
    CEL_HIP(hipGetLastError());
    *in = to;
  }
  return CEL_OK;
}

template <class T>
int embed_grad(const cel_embed_args *a, const void *dx, void *work, int grad_type, void *grad, hipStream_t s) {
  const Plan p = plan_of(a->tokens, a->vocab, a->hidden);
  const int slices = slices_of(a), searches = (int)((a->vocab + 1 + 255) / 256);
  const int rows = a->vocab * slices <= kFewRows ? 1 : kRowsAt;
  dim3 parts, sums;
  CEL_TRY(grid_of((a->tokens / kChunk) * slices + 4 * (int64_t)searches, "cel_embed_grad", &parts));
  CEL_TRY(grid_of((a->vocab + rows - 1) / rows * slices, "cel_embed_grad", &sums));
  char *w = static_cast<char *>(work);
  int in = 0;
  CEL_TRY(a->id_bytes == 4 ? sort_tokens<int32_t>(a, p, w, &in, s) : sort_tokens<int64_t>(a, p, w, &in, s));
  const uint32_t *keys = reinterpret_cast<uint32_t *>(w + p.keys[in]), *order = reinterpret_cast<uint32_t *>(w + p.order[in]);
  uint32_t *start = reinterpret_cast<uint32_t *>(w + p.start);
  float *part = reinterpret_cast<float *>(w + p.part);
  {
    KTimer kt(s, "k_embed_parts");
    k_embed_parts<T><<<parts, 256, 0, s>>>(keys, order, a->tokens, a->vocab, searches, start, (const T *)dx, a->stride,
                                           a->hidden, slices, part);
    CEL_HIP(hipGetLastError());
  }
  KTimer kt(s, "k_embed_grad");
  auto go = [&](auto out, auto nt) {
    typedef decltype(out) O;
    k_embed_grad<T, O, decltype(nt)::value><<<sums, 256, 0, s>>>(start, order, a->vocab, (const T *)dx, a->stride, a->hidden,
                                                                 slices, part, a->scale, rows, (O *)grad);
  };
  const bool f32 = grad_type == CEL_F32, nt = a->vocab * a->hidden * (f32 ? 4 : (int64_t)sizeof(T)) > kCached;
  if (f32) nt ? go(float{}, std::true_type{}) : go(float{}, std::false_type{});
  else nt ? go(T{}, std::true_type{}) : go(T{}, std::false_type{});
  CEL_HIP(hipGetLastError());
  return CEL_OK;
}

}  // namespace
}  // namespace cel

using namespace cel;

extern "C" int cel_embed(const cel_embed_args *a, const void *table, void *out, hipStream_t s) {
  CEL_TRY(check_embed(a, "cel_embed"));
  if (a->tokens == 0) return CEL_OK;
  if (!table || !out) return set_error(CEL_E_ARG, "cel_embed: table or out is NULL");
  return a->type == CEL_BF16  ? embed<__bf16>(a, table, out, s)
         : a->type == CEL_F16 ? embed<_Float16>(a, table, out, s)
                              : embed<float>(a, table, out, s);
}

extern "C" int64_t cel_embed_grad_scratch(int64_t tokens, int64_t vocab, int64_t hidden) {
  if (tokens < 0 || tokens > INT32_MAX || vocab < 1 || vocab > INT32_MAX - 1 || hidden < 1 || hidden > (1 << 24))
    return set_error(CEL_E_ARG, "cel_embed_grad_scratch: %lld tokens, %lld words, rows of %lld", (long long)tokens,
                     (long long)vocab, (long long)hidden);
  return plan_of(tokens, vocab, hidden).bytes;
}

extern "C" int cel_embed_grad(const cel_embed_args *a, const void *dx, void *scratch, int32_t grad_type, void *grad,
                              hipStream_t s) {
  CEL_TRY(check_embed(a, "cel_embed_grad"));
  if (grad_type != a->type && grad_type != CEL_F32)
    return set_error(CEL_E_ARG, "cel_embed_grad: a gradient of type %d of rows of type %d", grad_type, a->type);
  if (!grad || !scratch || (a->tokens && !dx)) return set_error(CEL_E_ARG, "cel_embed_grad: NULL array");
  return a->type == CEL_BF16  ? embed_grad<__bf16>(a, dx, scratch, grad_type, grad, s)
         : a->type == CEL_F16 ? embed_grad<_Float16>(a, dx, scratch, grad_type, grad, s)
                              : embed_grad<float>(a, dx, scratch, grad_type, grad, s);
}
