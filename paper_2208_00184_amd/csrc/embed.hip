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
// have a tenth of all tokens: every aligned chunk of kChunk sorted tokens that
// is one word through and through is summed beforehand by a wave of its own,
// and the row adds the chunks' sums.
#include <algorithm>
#include <cmath>

#include "cel_internal.h"

namespace cel {
namespace {

constexpr int kChunk = 64;       // sorted tokens of one partial sum
constexpr int kDigit = 9;        // bits of an id sorted at once: two passes up to 262,143 words
constexpr int kBins = 1 << kDigit;
constexpr int kSortB = 1024, kSortW = kSortB / 64;
constexpr int kOne = 8;          // tokens a thread holds in the sort by one workgroup
constexpr int kSegs = 4;         // 16-byte chunks a lane handles of a row slice
constexpr int kRowsAt = 4;       // table rows a wave writes one behind the other

// 16 bytes at any address of the element type.
struct __attribute__((packed, aligned(2))) Raw16 {
  uint32_t w[4];
};
template <class T>
struct Vec {
  static constexpr int N = 16 / sizeof(T);
};
template <class T>
__device__ inline void load_vec(float (&f)[Vec<T>::N], const T *p, int count) {
  if (count == Vec<T>::N) {
    const Raw16 r = *reinterpret_cast<const Raw16 *>(p);
    T x[Vec<T>::N];
    __builtin_memcpy(x, &r, 16);
#pragma unroll
    for (int e = 0; e < Vec<T>::N; e++) f[e] = (float)x[e];
  } else {
#pragma unroll
    for (int e = 0; e < Vec<T>::N; e++) f[e] = e < count ? (float)p[e] : 0.f;
  }
}
// N values rounded to O, 16 bytes at a time.
template <class O, int N>
__device__ inline void store_vec(O *p, const float (&f)[N], int count) {
  O x[N];
#pragma unroll
  for (int e = 0; e < N; e++) x[e] = (O)f[e];
  if (count == N) {
#pragma unroll
    for (int b = 0; b < (int)(N * sizeof(O)) / 16; b++) {
      Raw16 r;
      __builtin_memcpy(&r, x + b * Vec<O>::N, 16);
      *reinterpret_cast<Raw16 *>(p + b * Vec<O>::N) = r;
    }
    if constexpr (N * sizeof(O) % 16 != 0) {
#pragma unroll
      for (int e = N * sizeof(O) / 16 * Vec<O>::N; e < N; e++) p[e] = x[e];
    }
  } else {
#pragma unroll
    for (int e = 0; e < N; e++)
      if (e < count) p[e] = x[e];
  }
}

// A wave takes one token and kSegs * 64 chunks of its row.
template <class T, class I>
__global__ void __launch_bounds__(256) k_embed(const T *table, int64_t stride, int64_t vocab, const I *ids, int64_t tokens,
                                               int64_t h, int slices, float scale, T *out) {
  constexpr int N = Vec<T>::N;
  const int lane = threadIdx.x & 63;
  const int64_t task = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t t = task / slices;
  if (t >= tokens) return;
  const int64_t id = ids[t], c0 = (task % slices) * (kSegs * 64 * N) + lane * N;
  const bool in = id >= 0 && id < vocab;
  float f[kSegs][N];
#pragma unroll
  for (int u = 0; u < kSegs; u++) {
    const int64_t c = c0 + u * 64 * N;
#pragma unroll
    for (int e = 0; e < N; e++) f[u][e] = 0.f;
    if (in && c < h) load_vec<T>(f[u], table + id * stride + c, (int)min((int64_t)N, h - c));
  }
#pragma unroll
  for (int u = 0; u < kSegs; u++) {
    const int64_t c = c0 + u * 64 * N;
#pragma unroll
    for (int e = 0; e < N; e++) f[u][e] *= scale;
    if (c < h) store_vec<T, N>(out + t * h + c, f[u], (int)min((int64_t)N, h - c));
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
__device__ inline uint32_t rank_in_wave(uint32_t (*count)[kSortW], int wave, int lane, uint32_t digit, bool in) {
  const uint64_t m = same_digit(digit, in);
  uint32_t before = 0;
  if (in) before = count[digit][wave];
  lds_order();
  if (in && __builtin_ctzll(m) == lane) count[digit][wave] = before + (uint32_t)__builtin_popcountll(m);
  lds_order();
  return before + (uint32_t)__builtin_popcountll(m & ((uint64_t(1) << lane) - 1));
}
// Exclusive sums over the digits, and inside a digit over the waves; base:
// what each digit starts from besides, or NULL.  Called by the whole workgroup.
__device__ inline void start_counts(uint32_t (*count)[kSortW], uint32_t *s_sum, const uint32_t *base, int tid) {
  const int lane = tid & 63, wave = tid >> 6;
  uint32_t all = 0;
  if (tid < kBins) {
#pragma unroll
    for (int w = 0; w < kSortW; w++) {
      const uint32_t x = count[tid][w];
      count[tid][w] = all;
      all += x;
    }
  }
  if (!base) {
    uint32_t up = all;
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t y = __shfl_up(up, o);
      if (lane >= o) up += y;
    }
    if (tid < kBins && lane == 63) s_sum[wave] = up;
    __syncthreads();
    if (tid < kBins) {
      uint32_t b = up - all;
      for (int w = 0; w < wave; w++) b += s_sum[w];
      all = b;
    }
  } else if (tid < kBins) {
    all = base[tid];
  }
  if (tid < kBins) {
#pragma unroll
    for (int w = 0; w < kSortW; w++) count[tid][w] += all;
  }
  __syncthreads();
}

// Up to kOne * kSortB tokens by one workgroup, every pass through LDS.
template <class I>
__global__ void __launch_bounds__(kSortB) k_embed_sort_one(const I *ids, int tokens, int64_t vocab, int bits, uint32_t *keys,
                                                           uint32_t *order) {
  __shared__ uint32_t count[kBins][kSortW];
  __shared__ uint32_t s_key[kOne * kSortB], s_pos[kOne * kSortB], s_sum[kSortW];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint32_t key[kOne], pos[kOne];
  const int mine = wave * kOne * 64 + lane;  // a wave's tokens stand together
#pragma unroll
  for (int u = 0; u < kOne; u++) {
    pos[u] = mine + u * 64;
    key[u] = (int)pos[u] < tokens ? key_of(ids, pos[u], vocab) : 0;
  }
  for (int shift = 0; shift < bits; shift += kDigit) {
    for (int i = tid; i < kBins * kSortW; i += kSortB) (&count[0][0])[i] = 0;
    __syncthreads();
    uint32_t rank[kOne];
#pragma unroll
    for (int u = 0; u < kOne; u++) rank[u] = rank_in_wave(count, wave, lane, digit_of(key[u], shift), mine + u * 64 < tokens);
    __syncthreads();
    start_counts(count, s_sum, nullptr, tid);
#pragma unroll
    for (int u = 0; u < kOne; u++) {
      if (mine + u * 64 >= tokens) continue;
      const uint32_t to = count[digit_of(key[u], shift)][wave] + rank[u];
      s_key[to] = key[u];
      s_pos[to] = pos[u];
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kOne; u++) {
      if (mine + u * 64 >= tokens) continue;
      key[u] = s_key[mine + u * 64];
      pos[u] = s_pos[mine + u * 64];
    }
  }
#pragma unroll
  for (int u = 0; u < kOne; u++) {
    if (mine + u * 64 >= tokens) continue;
    keys[mine + u * 64] = key[u];
    order[mine + u * 64] = pos[u];
  }
}

// The same by several workgroups, each of which holds `tile` tokens (a
// multiple of kSortB): a pass counts digits per tile (table [tiles][kBins]),
// and then puts every token in its place.  first: from ids, else from keys.
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
  __shared__ uint32_t count[kBins][kSortW];
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
    for (int i = tid; i < kBins * kSortW; i += kSortB) (&count[0][0])[i] = 0;
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
    start_counts(count, s_sum, s_base, tid);
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
// Sorted tokens [a, b), added in order to the lane's columns; a row or a
// partial sum alike.
template <class T>
__device__ inline void add_tokens(float (&f)[kSegs][Vec<T>::N], const T *dx, int64_t stride, const uint32_t *order, int64_t a,
                                  int64_t b, int64_t c0, int64_t h) {
  constexpr int N = Vec<T>::N;
  for (int64_t t = a; t < b; t++) {
    const T *row = dx + (int64_t)order[t] * stride;
#pragma unroll
    for (int u = 0; u < kSegs; u++) {
      const int64_t c = c0 + u * 64 * N;
      if (c >= h) continue;
      float x[N];
      load_vec<T>(x, row + c, (int)min((int64_t)N, h - c));
#pragma unroll
      for (int e = 0; e < N; e++) f[u][e] += x[e];
    }
  }
}

// Blocks below `searches`: where each word's tokens begin (start [vocab + 1]).
// The others: the sums of the chunks that hold one word only (part [chunks][h]).
template <class T>
__global__ void __launch_bounds__(256) k_embed_parts(const uint32_t *keys, const uint32_t *order, int64_t tokens, int64_t vocab,
                                                     int searches, uint32_t *start, const T *dx, int64_t stride, int64_t h,
                                                     int slices, float *part) {
  if ((int)blockIdx.x < searches) {
    const int64_t v = (int64_t)blockIdx.x * 256 + threadIdx.x;
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
  constexpr int N = Vec<T>::N;
  const int lane = threadIdx.x & 63;
  const int64_t task = (int64_t)(blockIdx.x - searches) * 4 + (threadIdx.x >> 6);
  const int64_t chunk = task / slices, t0 = chunk * kChunk;
  if (t0 + kChunk > tokens) return;
  const uint32_t key = keys[t0];
  if (key != keys[t0 + kChunk - 1] || key >= (uint32_t)vocab) return;
  const int64_t c0 = (task % slices) * (kSegs * 64 * N) + lane * N;
  float f[kSegs][N] = {};
  add_tokens<T>(f, dx, stride, order, t0, t0 + kChunk, c0, h);
#pragma unroll
  for (int u = 0; u < kSegs; u++) {
    const int64_t c = c0 + u * 64 * N;
    if (c < h) store_vec<float, N>(part + chunk * h + c, f[u], (int)min((int64_t)N, h - c));
  }
}

// A wave takes kRowsAt rows of the table and kSegs * 64 chunks of their columns.
template <class T, class O>
__global__ void __launch_bounds__(256) k_embed_grad(const uint32_t *start, const uint32_t *order, int64_t vocab, const T *dx,
                                                    int64_t stride, int64_t h, int slices, const float *part, float scale,
                                                    O *grad) {
  constexpr int N = Vec<T>::N;
  const int lane = threadIdx.x & 63;
  const int64_t task = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t v0 = task / slices * kRowsAt;
  if (v0 >= vocab) return;
  const int64_t c0 = (task % slices) * (kSegs * 64 * N) + lane * N;
  const uint32_t at = lane <= kRowsAt && v0 + lane <= vocab ? start[v0 + lane] : 0;
  for (int r = 0; r < kRowsAt && v0 + r < vocab; r++) {
    const int64_t a = (uint32_t)__builtin_amdgcn_readlane(at, r), b = (uint32_t)__builtin_amdgcn_readlane(at, r + 1);
    float f[kSegs][N] = {};
    if (a < b) {
      const int64_t first = (a + kChunk - 1) / kChunk, last = b / kChunk;  // chunks inside [a, b)
      if (first < last) {
        add_tokens<T>(f, dx, stride, order, a, first * kChunk, c0, h);
        for (int64_t p = first; p < last; p++)
#pragma unroll
          for (int u = 0; u < kSegs; u++) {
            const int64_t c = c0 + u * 64 * N;
#pragma unroll
            for (int e = 0; e < N; e++)
              if (c + e < h) f[u][e] += part[p * h + c + e];
          }
        add_tokens<T>(f, dx, stride, order, last * kChunk, b, c0, h);
      } else {
        add_tokens<T>(f, dx, stride, order, a, b, c0, h);
      }
    }
#pragma unroll
    for (int u = 0; u < kSegs; u++) {
      const int64_t c = c0 + u * 64 * N;
#pragma unroll
      for (int e = 0; e < N; e++) f[u][e] *= scale;
      if (c < h) store_vec<O, N>(grad + (v0 + r) * h + c, f[u], (int)min((int64_t)N, h - c));
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
  const int64_t per = kSegs * 64 * (a->type == CEL_F32 ? 4 : 8);
  return (int)((a->hidden + per - 1) / per);
}
int blocks_of(int64_t waves, const char *fn, unsigned *blocks) {
  const int64_t b = (waves + 3) / 4;
  if (b > INT32_MAX) return set_error(CEL_E_ARG, "%s: too large a call", fn);
  *blocks = (unsigned)b;
  return CEL_OK;
}

template <class T>
int embed(const cel_embed_args *a, const void *table, void *out, hipStream_t s) {
  const int slices = slices_of(a);
  unsigned blocks;
  CEL_TRY(blocks_of(a->tokens * slices, "cel_embed", &blocks));
  KTimer kt(s, "k_embed");
  if (a->id_bytes == 4)
    k_embed<T, int32_t><<<blocks, 256, 0, s>>>((const T *)table, a->stride, a->vocab, (const int32_t *)a->ids, a->tokens,
                                               a->hidden, slices, a->scale, (T *)out);
  else
    k_embed<T, int64_t><<<blocks, 256, 0, s>>>((const T *)table, a->stride, a->vocab, (const int64_t *)a->ids, a->tokens,
                                               a->hidden, slices, a->scale, (T *)out);
  CEL_HIP(hipGetLastError());
  return CEL_OK;
}

template <class I>
int sort_tokens(const cel_embed_args *a, const Plan &p, char *w, int *in, hipStream_t s) {
  const I *ids = (const I *)a->ids;
  auto u32 = [&](int64_t at) { return reinterpret_cast<uint32_t *>(w + at); };
  *in = 0;
  if (a->tokens <= kOne * kSortB) {
    KTimer kt(s, "k_embed_sort_one");
    k_embed_sort_one<I><<<1, kSortB, 0, s>>>(ids, (int)a->tokens, a->vocab, p.bits, u32(p.keys[0]), u32(p.order[0]));
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
  char *w = static_cast<char *>(work);
  int in = 0;
  CEL_TRY(a->id_bytes == 4 ? sort_tokens<int32_t>(a, p, w, &in, s) : sort_tokens<int64_t>(a, p, w, &in, s));
  const int slices = slices_of(a);
  const uint32_t *keys = reinterpret_cast<uint32_t *>(w + p.keys[in]), *order = reinterpret_cast<uint32_t *>(w + p.order[in]);
  uint32_t *start = reinterpret_cast<uint32_t *>(w + p.start);
  float *part = reinterpret_cast<float *>(w + p.part);
  const int searches = (int)((a->vocab + 1 + 255) / 256);
  unsigned blocks;
  CEL_TRY(blocks_of((a->tokens / kChunk) * slices + 4 * (int64_t)searches, "cel_embed_grad", &blocks));
  {
    KTimer kt(s, "k_embed_parts");
    k_embed_parts<T><<<blocks, 256, 0, s>>>(keys, order, a->tokens, a->vocab, searches, start, (const T *)dx, a->stride,
                                            a->hidden, slices, part);
    CEL_HIP(hipGetLastError());
  }
  CEL_TRY(blocks_of((a->vocab + kRowsAt - 1) / kRowsAt * slices, "cel_embed_grad", &blocks));
  KTimer kt(s, "k_embed_grad");
  if (grad_type == CEL_F32)
    k_embed_grad<T, float><<<blocks, 256, 0, s>>>(start, order, a->vocab, (const T *)dx, a->stride, a->hidden, slices, part,
                                                  a->scale, (float *)grad);
  else
    k_embed_grad<T, T><<<blocks, 256, 0, s>>>(start, order, a->vocab, (const T *)dx, a->stride, a->hidden, slices, part,
                                              a->scale, (T *)grad);
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
