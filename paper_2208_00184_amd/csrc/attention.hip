// Attention over a packed batch with grouped heads, and its gradient: causal over
// the batch itself, or (CROSS) to the states of an encoder, packed alike.
//
// Token i of a sequence sees the tokens j <= i of the same sequence, or all of
// the states that belong to its sequence:
//   s_ij = scale <q_i, k_j>,  lse_i = log sum_j exp s_ij,  p_ij = exp(s_ij - lse_i)
//   o_i = sum_j p_ij v_j
// and backwards, with D_i = <do_i, o_i>:
//   dv_j = sum p_ij do_i,  ds_ij = p_ij (<do_i, v_j> - D_i)
//   dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum_i ds_ij q_i
// dv and dk also sum over the query heads that share the key/value head.
//
// Tiles are cut from the token axis whatever the sequences' borders, and each
// row (or column) carries the borders of its own sequence, so many short
// sequences fill tiles as well as one long one.  The products run on
// 32x32x16 matrix instructions in orientations that let one product's result
// be the next one's operand without leaving its registers:
//   a result tile D[m][n] puts column n = lane % 32 and rows 8 (r / 4) + 4
//   (lane / 32) + r % 4 in register r; registers 8 j .. 8 j + 7, rounded to
//   16 bits, are a right operand B[k][n] for 16 values of k, in that order of k.
//   The left operand takes its k in the same order: two transposed 8-byte
//   reads of LDS, four rows each.
// Scores, running maxima and sums, and all accumulators are 32 bit.  p and ds
// are rounded to the inputs' 16-bit type as operands, since the matrix cores
// take 16-bit operands only at their full rate; the sum under p's quotient
// adds the unrounded values.  float16's narrow range gets a scale for them, see kScaled.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "cel_internal.h"

namespace cel {
namespace {

constexpr int kWaves = 4;            // waves of a workgroup
constexpr int kRows = 32;            // tile rows a wave owns
constexpr int kBlock = kWaves * kRows;
constexpr int kStep = 64;            // rows of the other side staged at once
constexpr int kAhead = 4;             // reads of LDS stand this many matrix instructions before their use
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

typedef __attribute__((ext_vector_type(16))) float acc16;
typedef __attribute__((ext_vector_type(4))) float acc4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;

template <class T>
struct Half;
template <>
struct Half<__bf16> {
  typedef __attribute__((ext_vector_type(8))) __bf16 v8;
  typedef __attribute__((ext_vector_type(2))) __bf16 v2;
  static __device__ acc16 mma(u32x4 a, u32x4 b, acc16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
  }
};
template <>
struct Half<_Float16> {
  typedef __attribute__((ext_vector_type(8))) _Float16 v8;
  typedef __attribute__((ext_vector_type(2))) _Float16 v2;
  static __device__ acc16 mma(u32x4 a, u32x4 b, acc16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
  }
};
template <class T>
__device__ inline uint32_t pack2(float lo, float hi) {
  const typename Half<T>::v2 x = __builtin_convertvector(f32x2{lo, hi}, typename Half<T>::v2);
  return __builtin_bit_cast(uint32_t, x);
}
// Registers 8 j .. 8 j + 7 of a result tile as a 16-bit operand.
template <class T>
__device__ inline u32x4 operand(const acc16 &x, int j) {
  u32x4 b;
#pragma unroll
  for (int e = 0; e < 4; e++) b[e] = pack2<T>(x[8 * j + 2 * e], x[8 * j + 2 * e + 1]);
  return b;
}
// float16 has 2^-14 .. 2^16 (and 2^-24 with fewer bits), while ds is as large or small as the loss and
// its scale make dout, and 1 / length besides.  A column's (one row's for dq, one key's for dk)
// entries of ds are therefore rounded times a power of two of that column's own, 2^up, taken
// out of its sums where they are stored.  up begins so high that the first entry that is not
// 0 brings it down: when one passes kTop, up falls to where that one is near 2^8, and
// the sums so far with it.  Entries 2^22 below a column's largest so keep all their bits, and what is lost
// of smaller ones is 2^-33 of the largest.  p of dv takes a constant 2^kPUp: at most 1, it
// leaves room for what lse's own rounding makes it too large where scores are in the millions.
// The largest entry is looked for in every step, 4 % of the gradient's time (9,973 tokens in 37
// sequences, 24 heads of 80 over 4: dk and dv 156 -> 164 us, dq 123 -> 126).  Without all this
// dq of one sequence of 4,096 at a dout of 2^-12 was off by 6.8e-3 where its results' own rounding is 1.2e-3.
template <class T>
constexpr bool kScaled = __is_same(T, _Float16);
template <class T>
constexpr int kUp = kScaled<T> ? 64 : 0;
template <class T>
constexpr int kPUp = kScaled<T> ? 8 : 0;
constexpr float kTop = 32768.f;
__device__ inline float power(int e) { return ldexpf(1.f, e); }
// The exponent by which a column whose largest entry is `top` comes down.  An infinity stays
// one whatever the power; up stays.
__device__ inline int down_by(float top) {
  return top > kTop && top < INFINITY ? 9 - __builtin_amdgcn_frexp_expf(top) : 0;
}
__device__ inline float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
// The sum or maximum of lane l's and lane l ^ 32's values, in both.
__device__ inline float half_sum(float x) {
  const u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ inline float half_max(float x) {
  const u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

struct Rows {  // a [tokens][heads][dim] view, strides in elements
  char *p;
  int64_t row, head;
};
struct AttnArgs {
  Rows q, k, v, out, dout, dq, dk, dv;
  const int32_t *ptr, *k_ptr;  // of the rows; of the keys where they are others
  int32_t S, T, U, H, K, d, tiles;  // U: keys
  float *lse;
  float *rows;  // the backward pass's scratch: lse in units of log 2 less kPUp, D, each [heads][tokens]
  float *part;  // and behind it, where a key/value head's query heads are dealt out to `parts` workgroups, dk
                // and dv of each part, [parts][2][keys][kv_heads][dim]
  int32_t parts;
  int32_t *order, *k_order;  // CROSS: the tiles of rows and of keys with the longest first, or NULL: as they come
  int32_t splits;            // CROSS: workgroups that share a tile's keys, one behind the other
  float *split;              // where these leave their sums, [splits][heads][tokens][dim], and behind them each
                             // row's maximum and sum of the forward pass, [splits][heads][tokens][2]
  float scale;
};

// A staged tile: kStep rows of DP 16-bit values, in 16-byte chunks.  Chunk c
// of row r lies at position c ^ Swz::of(r) of its row: the 16 rows that a wave's
// plain 16-byte reads touch at once, and the four rows of a transposed read,
// then lie in different banks.
template <int DP>
struct Swz {
  static __device__ int of(int r) {
    return DP == 128 ? ((r & 3) << 2) | ((r >> 2) & 3) : (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
  }
};
template <int DP>
__device__ inline int chunk_at(int r, int c) {  // byte offset
  return r * (DP * 2) + ((c ^ Swz<DP>::of(r)) << 4);
}
// x, as far as the compiler knows made from the loop's variable `by`: what is
// made from it inside the loop is not kept in registers across the loop.
__device__ __forceinline__ int fresh(int x, int by) {
  asm("" : "+v"(x) : "s"(by));
  return x;
}
// Copies rows [r0, r0 + kStep) of one head of a view straight into LDS, 16
// bytes a lane; rows at or past `end`, and values past d, become zeros: they
// lie beyond the buffer descriptor's size.  The copy is in order with the
// wave's other loads and done once vmcnt says so.
template <int DP, class Order = Swz<DP>>
struct Stager {
  static constexpr int C = DP / 8, kLoads = kStep * C / (kWaves * 64), kRowsApart = kWaves * 64 / C;
  static_assert(kLoads >= 1 && kRowsApart % 16 == 0, "whole loads, and the order repeats after 16 rows");
  const char *base;
  uint32_t at, row;  // this lane's offset in a tile; bytes between rows
  __device__ Stager(const Rows &x, int d, int tid) : base(x.p), row((uint32_t)(2 * x.row)) {
    const int r = tid / C, c = (tid % C) ^ Order::of(r);
    at = c * 8 < d ? (uint32_t)r * row + 16 * c : 0x80000000u;
  }
  __device__ void load(char *lds, int64_t head_bytes, int r0, int end, int wave) const {
    const int rows = min(end - r0, kStep);
    const __amdgpu_buffer_rsrc_t buf = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<char *>(base + head_bytes + (int64_t)r0 * row), 0, rows > 0 ? (uint32_t)rows * row : 0u, 0x00020000);
#pragma unroll
    for (int i = 0; i < kLoads; i++)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          buf, (__attribute__((address_space(3))) void *)(lds + (i * kWaves + wave) * 1024), 16,
          at + (uint32_t)i * kRowsApart * row, 0, 0, 0);
  }
};
// Between tiles: this wave's copies have landed and its reads of LDS are
// done; after it, every wave's are.
__device__ inline void next_tile() {
  __builtin_amdgcn_s_waitcnt(0x0070);  // vmcnt(0), lgkmcnt(0)
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// Where a lane reads a staged tile: byte offsets of its first chunk, by rows
// and by columns.  The others follow by flipping bits of the chunk's position.
template <int DP>
struct Lane {
  static constexpr int RB = 2 * DP;
  int rows, cols;
  __device__ explicit Lane(int lane) {
    const int i = lane & 15, h = lane >> 5;
    rows = chunk_at<DP>(lane & 31, h);
    cols = chunk_at<DP>(4 * h + (i >> 2), 2 * ((lane >> 4) & 1) + ((i & 3) >> 1)) + 8 * (i & 1);
  }
};
// Left operand: rows 32 t + lane % 32, columns 16 kk + 8 (lane / 32) + 0..7.
template <int DP>
__device__ inline u32x4 rows_at(const char *lds, int rows, int t, int kk) {
  return *reinterpret_cast<const u32x4 *>(lds + (rows ^ (kk << 5)) + t * 32 * Lane<DP>::RB);
}
// Left operand of the transpose: its row 32 n + lane % 32 is a column of the
// tile, its k the tile's rows 16 j + 4 (lane / 32) + 0..3 and, behind them,
// those 8 further on.  A transposed read gives lane i of 16 lanes the i-th of
// 16 columns of four rows, of which lane i addresses row i / 4, columns 4 (i % 4) + 0..3.
template <int DP>
__device__ inline u32x4 cols_at(const char *lds, int cols, int n, int j) {
  typedef __attribute__((ext_vector_type(4))) short s16x4;
  typedef __attribute__((address_space(3))) s16x4 *lds_ptr;
  u32x4 a;
#pragma unroll
  for (int u = 0; u < 2; u++) {
    const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (lds_ptr)(lds + (cols ^ (n << 6) ^ (u << 5)) + (16 * j + 8 * u) * Lane<DP>::RB));
    const u32x2 y = __builtin_bit_cast(u32x2, x);
    a[2 * u] = y[0];
    a[2 * u + 1] = y[1];
  }
  return a;
}

// The 16-bit halves of x that are infinities or NaN, as all ones.
template <class T>
__device__ inline uint32_t not_numbers(uint32_t x) {
  const uint32_t e = __is_same(T, __bf16) ? 0x7f80u : 0x7c00u;
  return ((x & e) == e ? 0xffffu : 0u) | ((x >> 16 & e) == e ? 0xffff0000u : 0u);
}

// acc[n] += (columns of the staged tile)^T b[j], where entry x of the 16 J that b
// holds counts only for lo <= x <= hi of its column.  b's other entries are 0,
// which is enough unless the tile holds an infinity or NaN there, which 0
// times it would let in.  The products run on the tile's numbers, in the order
// and to the bits of a tile without others; each row x's infinities and NaN
// are a product of their own, added where the column sees x.
template <class T, int DP, int NB, int J>
__device__ __forceinline__ void careful_product(const char *lds, acc16 (&acc)[NB], const u32x4 (&b)[J], int cols,
                                                int lo, int hi, int lane, int a0) {
  lane = fresh(lane, a0), cols = fresh(cols, a0);
#pragma unroll
  for (int j = 0; j < J; j++)
#pragma unroll
    for (int n = 0; n < NB; n++) {
      u32x4 a = cols_at<DP>(lds, cols, n, j), off;
#pragma unroll
      for (int w = 0; w < 4; w++) {
        const uint32_t m = not_numbers<T>(a[w]);
        off[w] = a[w] & m;
        a[w] &= ~m;
      }
      acc[n] = Half<T>::mma(a, b[j], acc[n]);
      if (!__any((off[0] | off[1] | off[2] | off[3]) != 0)) continue;
#pragma unroll 1
      for (int k = 0; k < 16; k++) {
        const int e = (k & 3) | ((k >> 1) & 4), x = 16 * j + k;
        const uint32_t keep = (lane >> 5) == ((k >> 2) & 1) ? (e & 1 ? 0xffff0000u : 0xffffu) : 0u;
        u32x4 only;
#pragma unroll
        for (int w = 0; w < 4; w++) only[w] = w == (e >> 1) ? off[w] & keep : 0u;
        acc16 one = {};
        one = Half<T>::mma(only, b[j], one);
#pragma unroll
        for (int r = 0; r < 16; r++) acc[n][r] = x >= lo && x <= hi ? acc[n][r] + one[r] : acc[n][r];
      }
    }
}

// The sequence that holds token i of n: its tokens [a, b) of m, as ptr or, of the other
// side, `other` has them; empty if there is none.  Whatever they hold, the range lies within the buffer.
__device__ inline void sequence_of(const int32_t *ptr, int S, int n, const int32_t *other, int m, int i, int &a, int &b) {
  a = b = 0;
  if (i >= n) return;
  int lo = 0, hi = S;  // the last s with ptr[s] <= i, if any
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (ptr[mid] <= i) lo = mid;
    else hi = mid - 1;
  }
  if (lo >= S) return;
  int from = ptr[lo], to = ptr[lo + 1];
  if (from > i || to <= i) return;
  if (other != ptr) from = other[lo], to = other[lo + 1];
  a = from < 0 ? 0 : from;
  b = to > m ? m : to;
}

__device__ inline int wave_min(int x) {
  for (int o = 32; o; o >>= 1) x = min(x, __shfl_xor(x, o));
  return x;
}
__device__ inline int wave_max(int x) {
  for (int o = 32; o; o >>= 1) x = max(x, __shfl_xor(x, o));
  return x;
}

// Workgroups in an order that deals with the tiles of all heads (units) in turn,
// tile 0 first, so that a head's short tiles do not leave another's long ones to the
// end.  The 8 dies take workgroups in turn: a power of two of them share
// neighbouring heads, whose keys and values are then in those dies' L2 caches.
// Against one head after the other, 4 sequences of 1,024 tokens, 64 heads of 128: forward
// 131 -> 112 us, dk and dv 236 -> 217, dq 214 -> 203; 61 ragged ones, 32 heads of 128 over 8: 299
// -> 252; one of 16,384, 4 heads of 128: dk and dv 740 -> 592.  Slower where more
// heads at once mean more keys than L2 holds (8,192 tokens, 64 heads of 128: dk and dv 2.31 -> 2.39
// ms, but forward 1.10 -> 1.07) and where no tile is long (64 sequences of 256: 32.5 -> 34.3).
// Where a die's 32 compute units take all of its workgroups at once, two each, the second
// half comes backwards: the longest of a head's tiles then share their unit with
// the shortest (4,096 tokens in 4 sequences, 16 heads of 64: forward 29 -> 26 us, dq 39 -> 32).
struct Item {
  int unit, tile;
};
__device__ inline Item item_of(int block, int blocks, int units) {
  const int x = block & 7, all = (blocks >> 3) + (x < (blocks & 7));
  int s = block >> 3;
  if (all <= 64 && s >= 32) s = 32 + all - 1 - s;
  const int at = 8 * s + x, u = at % units, share = min(units & -units, 8);
  return {u % share * (units / share) + u / share, at / units};
}

// Right operand from global memory: column lane % 32 is a token, its k the
// dimensions 16 kk + 8 (lane / 32) + 0..7.
template <int KK>
__device__ inline void load_rows(u32x4 (&f)[KK], const Rows &x, int head, int i, int end, int d, int lane) {
  const char *p = x.p + 2 * ((int64_t)i * x.row + (int64_t)head * x.head);
#pragma unroll
  for (int kk = 0; kk < KK; kk++) {
    const int c = 16 * kk + 8 * (lane >> 5);
    f[kk] = i < end && c < d ? *reinterpret_cast<const u32x4 *>(p + 2 * c) : u32x4{0, 0, 0, 0};
  }
}
// A transposed result, acc[n][r] times `by`: dimension 32 (n0 + n) + 8 (r / 4) + 4 (lane / 32) + r % 4 of row i.
template <class T, int N>
__device__ inline void store_rows(const Rows &x, int head, int i, const acc16 (&acc)[N], int n0, float by, int d, int lane) {
  char *p = x.p + 2 * ((int64_t)i * x.row + (int64_t)head * x.head);
#pragma unroll
  for (int n = 0; n < N; n++)
#pragma unroll
    for (int g = 0; g < 4; g++) {
      const int c = 32 * (n0 + n) + 8 * g + 4 * (lane >> 5);
      if (c < d)
        *reinterpret_cast<u32x2 *>(p + 2 * c) = u32x2{pack2<T>(acc[n][4 * g] * by, acc[n][4 * g + 1] * by),
                                                      pack2<T>(acc[n][4 * g + 2] * by, acc[n][4 * g + 3] * by)};
    }
}
template <int N>
__device__ inline bool not_finite(const acc16 (&acc)[N], float by) {
  float t = 0.f;
#pragma unroll
  for (int n = 0; n < N; n++)
#pragma unroll
    for (int r = 0; r < 16; r++) t += acc[n][r] * by * 0.f;
  return !(t == 0.f);
}

// The tokens of the other side that a lane's token deals with, as an interval
// (empty: lo > hi), and what follows for its wave and workgroup: all that any of
// their tokens deals with, and what every token of the wave deals with.
struct Reach {
  int lo, hi;            // this lane's
  int any_lo, any_hi;    // this wave's union
  int all_lo, all_hi;    // this wave's intersection
  int from, to;          // the workgroup's union
  __device__ bool real() const { return lo <= hi; }
  // of the tile [a, a + kStep): whether the wave has no part in it, or only some of its tokens with some of it
  __device__ bool skips(int a) const { return a > any_hi || a + kStep <= any_lo; }
  __device__ bool masks(int a) const { return a < all_lo || a + kStep - 1 > all_hi; }
  __device__ int steps() const { return to < from ? 0 : (to - from) / kStep + 1; }
};
// forward: the keys that token i sees; else the rows that see it.
template <bool CROSS>
__device__ inline Reach reach_of(const AttnArgs &A, int i, bool forward, int (*s_reach)[kWaves], int wave) {
  int first, last;
  if constexpr (!CROSS) sequence_of(A.ptr, A.S, A.T, A.ptr, A.T, i, first, last);
  else if (forward) sequence_of(A.ptr, A.S, A.T, A.k_ptr, A.U, i, first, last);
  else sequence_of(A.k_ptr, A.S, A.U, A.ptr, A.T, i, first, last);
  Reach R;
  const bool real = last > first;
  R.lo = !real ? INT32_MAX : CROSS || forward ? first : i;
  R.hi = !real ? -1 : !CROSS && forward ? i : last - 1;
  R.any_lo = wave_min(R.lo), R.any_hi = wave_max(R.hi);
  R.all_lo = wave_max(real ? R.lo : -1), R.all_hi = wave_min(real ? R.hi : INT32_MAX);
  s_reach[0][wave] = R.any_lo;
  s_reach[1][wave] = R.any_hi;
  __syncthreads();
  R.from = INT32_MAX, R.to = -1;
#pragma unroll
  for (int w = 0; w < kWaves; w++) {
    R.from = min(R.from, s_reach[0][w]);
    R.to = max(R.to, s_reach[1][w]);
  }
  R.from = __builtin_amdgcn_readfirstlane(R.from), R.to = __builtin_amdgcn_readfirstlane(R.to);
  R.any_lo = __builtin_amdgcn_readfirstlane(R.any_lo), R.any_hi = __builtin_amdgcn_readfirstlane(R.any_hi);
  R.all_lo = __builtin_amdgcn_readfirstlane(R.all_lo), R.all_hi = __builtin_amdgcn_readfirstlane(R.all_hi);
  return R;
}

// n tiles through two buffers: load(t, buffer) starts the copy of tile t, which
// runs while step(t - 1, other buffer) computes.  The buffers are LDS variables
// of their own and the loop is written out for both, so that the compiler sees
// which reads a copy in flight concerns and waits for no other.
template <int I>
struct Buffer {
  static constexpr int at = I;
};
template <bool SLOWLY, class Load, class Step>  // one tile at a time: for the rare pass over infinities and NaN
__device__ __forceinline__ void through_tiles(int n, Load load, Step step) {
  if constexpr (SLOWLY) {
#pragma unroll 1
    for (int t = 0; t < n; t++) {
      next_tile();
      load(t, Buffer<0>{});
      next_tile();
      step(t, Buffer<0>{});
    }
    return;
  }
  if (n > 0) load(0, Buffer<0>{});
#pragma unroll 1
  for (int t = 0; t < n; t += 2) {
    next_tile();
    if (t + 1 < n) load(t + 1, Buffer<1>{});
    step(t, Buffer<0>{});
    if (t + 1 >= n) break;
    next_tile();
    if (t + 2 < n) load(t + 2, Buffer<0>{});
    step(t + 1, Buffer<1>{});
  }
}
// N matrix instructions, instruction x fed by read(x) from LDS kAhead instructions
// before: left to itself, or asked for this order as a preference, the compiler reads each
// operand right before its use where it runs short of registers, and waits.
template <int N, class Read, class Use>
__device__ __forceinline__ void feed(Read read, Use use) {
  u32x4 ring[kAhead + 1];
#pragma unroll
  for (int x = 0; x < kAhead && x < N; x++) ring[x] = read(x);
#pragma unroll
  for (int x = 0; x < N; x++) {
    if (x + kAhead < N) ring[(x + kAhead) % (kAhead + 1)] = read(x + kAhead);
    use(x, ring[x % (kAhead + 1)]);
    __builtin_amdgcn_sched_barrier(0x6);  // vector and scalar arithmetic may still move
  }
}
// acc += (columns of the staged tile)^T b, see careful_product.
template <class T, int DP, bool CAREFUL, int NB, int J>
__device__ __forceinline__ void product(const char *lds, acc16 (&acc)[NB], const u32x4 (&b)[J], int cols, bool masked,
                                        int lo, int hi, int lane, int a) {
  if (CAREFUL && masked) {
    careful_product<T, DP, NB, J>(lds, acc, b, cols, lo, hi, lane, a);
  } else {
    cols = fresh(cols, a);
    feed<J * NB>([&](int x) { return cols_at<DP>(lds, cols, x % NB, x / NB); },
                 [&](int x, u32x4 f) { acc[x % NB] = Half<T>::mma(f, b[x / NB], acc[x % NB]); });
  }
}
// x = rows 32 t .. of a staged tile times f, y = rows 32 u .. of another times g.
template <class T, int DP, int KK>
__device__ __forceinline__ void rows_products(acc16 &x, const char *lds, int t, const u32x4 (&f)[KK], acc16 &y,
                                              const char *lds2, int u, const u32x4 (&g)[KK], int rows, int a) {
  rows = fresh(rows, a);
  feed<2 * KK>([&](int n) { return rows_at<DP>(n & 1 ? lds2 : lds, rows, n & 1 ? u : t, n / 2); },
               [&](int n, u32x4 z) {
                 if (n & 1) y = Half<T>::mma(z, g[n / 2], n > 1 ? y : acc16{});
                 else x = Half<T>::mma(z, f[n / 2], n > 1 ? x : acc16{});
               });
}
// x's entries at 32 t .. of a tile outside lo .. hi, replaced.
__device__ __forceinline__ void mask(acc16 &x, int t, int lo, int hi, float by, int lane) {
#pragma unroll
  for (int r = 0; r < 16; r++) {
    const int at = 32 * t + 8 * (r / 4) + r % 4 + 4 * (lane >> 5);
    x[r] = at >= lo && at <= hi ? x[r] : by;
  }
}

// CROSS: this workgroup's share of a tile's keys, from R.from on; how many steps it is.
__device__ inline int share_of_keys(const AttnArgs &A, Reach &R) {
  const int all = R.steps();
  if (A.splits == 1) return all;
  const int first = (int)((int64_t)all * blockIdx.y / A.splits), end = (int)((int64_t)all * (blockIdx.y + 1) / A.splits);
  R.from += first * kStep;
  return end - first;
}
// Row i's place among the rows of all heads and shares.
__device__ inline int64_t split_row(const AttnArgs &A, int head, int i) { return ((int64_t)blockIdx.y * A.H + head) * A.T + i; }
// acc[n][r] times `by` to this workgroup's share of a row, laid out as in store_rows.
template <int N>
__device__ inline void store_split(const AttnArgs &A, int head, int i, const acc16 (&acc)[N], int n0, float by, int lane) {
  float *p = A.split + split_row(A, head, i) * A.d;
#pragma unroll
  for (int n = 0; n < N; n++)
#pragma unroll
    for (int g = 0; g < 4; g++) {
      const int c = 32 * (n0 + n) + 8 * g + 4 * (lane >> 5);
      if (c < A.d)
        *reinterpret_cast<acc4 *>(p + c) =
            acc4{acc[n][4 * g] * by, acc[n][4 * g + 1] * by, acc[n][4 * g + 2] * by, acc[n][4 * g + 3] * by};
    }
}

// One tile of 128 tokens of one query head: each wave 32 of them, over the
// keys from the first row's sequence on.  A softmax in one pass: the sums o and
// l stand relative to 2^mc and are rescaled when the maximum m has moved.
// Bound by the matrix cores and, next to them, by exponentials and maxima in the
// vector unit, which two waves on a SIMD overlap.  A tile of 128 rows reads each
// staged key and value four times from LDS, which then gives what the products
// take; more rows would not fit two waves' registers.  16,384 tokens in one sequence,
// 16 heads of 128 over 4: 1.01 ms, 1.09 PFLOP/s, where a large library product
// reaches 1.36 and this kernel without its softmax 1.25; 8,192 tokens, 32 heads
// over 8: 0.51 ms, 1.07 PFLOP/s, matrix cores 55 % busy, no bank conflicts.
// 4 sequences of 1,024, 16 heads of 64: 23 us, the 16 steps of a sequence's last
// tile (0.8 us each at 64 dimensions, 1.1 at 128) behind some 7 us of start and end.
template <class T, int DP, int DC, int G, bool CROSS, bool CAREFUL>
__device__ __forceinline__ bool attention_tile(const AttnArgs &A, char *s_k0, char *s_k1, char *s_v0, char *s_v1,
                                               int (*s_reach)[kWaves]) {
  constexpr int kTile = kStep * DP * 2;
  constexpr int NB = CAREFUL ? 1 : (DC + 31) / 32;  // sums a pass holds, see CEL_TILE_KERNEL
  const int tid = threadIdx.x % (kWaves * 64), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int group = G > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / (kWaves * 64)) : 0;
  const Item item = item_of(blockIdx.x, gridDim.x, A.H);
  const int head = item.unit, kvh = head / (A.H / A.K);
  const int tile = CROSS ? A.order ? A.order[item.tile] : item.tile : A.tiles - 1 - item.tile;
  const int i = tile * kBlock + wave * kRows + (lane & 31);  // this lane's row
  Reach R = reach_of<CROSS>(A, i, true, s_reach + 2 * group, wave);
  const int steps = CROSS ? share_of_keys(A, R) : R.steps();
  u32x4 q[DC / 16];
  load_rows(q, A.q, head, i, A.T, A.d, lane);
  const float c = A.scale * kLog2e, far = 8.f / c;
  const Lane<DP> L(lane);
  const Stager<DP> ks(A.k, A.d, tid), vs(A.v, A.d, tid);
  const int64_t k_head = 2 * kvh * A.k.head, v_head = 2 * kvh * A.v.head;
  // from block n0 of 32 dimensions on
  auto pass = [&](int n0) {
    const int cols = L.cols ^ (n0 << 6);
    acc16 o[NB];
    float m, mc, l;
    auto load = [&](int t, auto buf) {
      const int a = R.from + (t * G + group) * kStep;
      ks.load((buf.at ? s_k1 : s_k0) + group * kTile, k_head, a, R.to + 1, wave);
      vs.load((buf.at ? s_v1 : s_v0) + group * kTile, v_head, a, R.to + 1, wave);
    };
    auto step = [&](int t0, auto buf) {
      const int a = R.from + (t0 * G + group) * kStep;
      if (R.skips(a)) return;
      const char *s_k = (buf.at ? s_k1 : s_k0) + group * kTile, *s_v = (buf.at ? s_v1 : s_v0) + group * kTile;
      const bool masked = R.masks(a);
      const int lo = R.lo - a, hi = R.hi - a;  // of the 64 keys, those that this row sees
      acc16 s[2];
      // The products come first: matrix instructions take one issue slot in eight, so
      // the other wave's vector instructions still find theirs.
      __builtin_amdgcn_s_setprio(1);
      rows_products<T, DP>(s[0], s_k, 0, q, s[1], s_k, 1, q, L.rows, a);
      __builtin_amdgcn_s_setprio(0);
      if (masked) {
        mask(s[0], 0, lo, hi, -INFINITY, lane);
        mask(s[1], 1, lo, hi, -INFINITY, lane);
      }
      float top = s[0][0];
#pragma unroll
      for (int t = 0; t < 2; t++)
#pragma unroll
        for (int r = 0; r < 16; r++) top = fmaxf(top, s[t][r]);
      top = half_max(top);
      // The reference m of the exponents follows the maximum only once that is
      // 2^8 above it: p stays below 2^8, and the sums are seldom rescaled.  Each row's own
      // maximum decides, so that a row's bits do not hang on its neighbours'.
      const bool above = top > m + far;
      if (__any(above)) {
        const float by = above ? exp2_((m - top) * c) : 1.f;
        m = above ? top : m;
        mc = m == -INFINITY ? 0.f : m * c;
        l *= by;
#pragma unroll
        for (int n = 0; n < NB; n++) o[n] *= by;
      }
      u32x4 p[4];
#pragma unroll
      for (int t = 0; t < 2; t++) {
#pragma unroll
        for (int r = 0; r < 16; r++) {
          s[t][r] = exp2_(fmaf(s[t][r], c, -mc));
          l += s[t][r];
        }
        p[2 * t] = operand<T>(s[t], 0);
        p[2 * t + 1] = operand<T>(s[t], 1);
      }
      __builtin_amdgcn_s_setprio(1);
      product<T, DP, CAREFUL>(s_v, o, p, cols, masked, lo, hi, lane, a);
      __builtin_amdgcn_s_setprio(0);
    };
    auto clear = [&] {
#pragma unroll
      for (int n = 0; n < NB; n++) o[n] = acc16{};
      m = -INFINITY, mc = 0.f, l = 0.f;
    };
    clear();
    through_tiles<CAREFUL>((steps + G - 1) / G, load, step);
    // An infinity or NaN may come from a value that the row does not see.
    if (!CAREFUL && __syncthreads_or(R.real() && not_finite(o, 1.f))) return false;
    l = half_sum(l);
    if constexpr (G > 1) {  // the first group's sums and the second's, over the larger maximum
      float *theirs = reinterpret_cast<float *>((wave & 2 ? s_k1 : s_k0) + (wave & 1) * kTile) + lane;
      float *stats = reinterpret_cast<float *>(s_v0) + wave * 128 + lane;
      if (CAREFUL) __syncthreads();
      if (group) {
#pragma unroll
        for (int n = 0; n < NB; n++)
#pragma unroll
          for (int r = 0; r < 16; r++) theirs[(16 * n + r) * 64] = o[n][r];
        stats[0] = m, stats[64] = l;
      }
      __syncthreads();
      if (!group) {
        const float m1 = stats[0], to = fmaxf(m, m1);
        const float a0 = to == -INFINITY ? 1.f : exp2_((m - to) * c), a1 = to == -INFINITY ? 1.f : exp2_((m1 - to) * c);
        l = l * a0 + stats[64] * a1;
        mc = to == -INFINITY ? 0.f : to * c;
#pragma unroll
        for (int n = 0; n < NB; n++)
#pragma unroll
          for (int r = 0; r < 16; r++) o[n][r] = o[n][r] * a0 + theirs[(16 * n + r) * 64] * a1;
      }
    }
    if (CROSS && G == 1 && A.splits > 1) {
      if (i < A.T) {
        store_split(A, head, i, o, n0, 1.f, lane);
        float *stats = A.split + (int64_t)A.splits * A.H * A.T * A.d + 2 * split_row(A, head, i);
        if (lane < 32) *reinterpret_cast<f32x2 *>(stats) = R.real() ? f32x2{m, l} : f32x2{-INFINITY, -1.f};
      }
    } else if (i < A.T && group == 0) {
      if (!R.real()) {
#pragma unroll
        for (int n = 0; n < NB; n++) o[n] = acc16{};
      }
      store_rows<T>(A.out, head, i, o, n0, R.real() ? 1.f / l : 0.f, A.d, lane);
      if (lane < 32) A.lse[(int64_t)head * A.T + i] = R.real() ? (mc + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
    }
    return true;
  };
  if constexpr (!CAREFUL) return pass(0);
#pragma unroll 1
  for (int n0 = 0; n0 < (DC + 31) / 32; n0++) (void)pass(n0);
  return true;
}

// A workgroup runs its tile without regard to infinities and NaN, and where
// the result has any, all of it again with.  The second run takes 32 dimensions at a
// time, so that its own sums need few registers, but what both make from the lane's number
// stays in registers across the first: at 128 dimensions dq spills 36 registers (20 in float16), most of
// them outside its loop, and so does not have all of its rows' first loads on their way at once; the
// forward kernel spills 2.
// G = 2: two groups of waves share the rows and take their keys' tiles in turn,
// each with buffers of its own, and join their sums at the end.  A tile's chain of
// steps, each of which waits for the one before, is then half as long, with the
// same two waves on every SIMD; it is taken where each workgroup has a compute unit
// to itself, so that the longest chain is the time (see split_keys).
#define CEL_TILE_KERNEL(kernel, tile, a0, a1, b0, b1)                                                      \
  template <class T, int DP, int DC, int G, bool CROSS>                                                    \
  __global__ void __launch_bounds__(G *kWaves * 64, 2) kernel(AttnArgs A) {                                \
    constexpr int kTile = G * kStep * DP * 2;                                                              \
    __shared__ __align__(16) char a0[kTile], a1[kTile], b0[kTile], b1[kTile];                              \
    __shared__ int s_reach[2 * G][kWaves];                                                                 \
    if (!tile<T, DP, DC, G, CROSS, false>(A, a0, a1, b0, b1, s_reach))                                     \
      (void)tile<T, DP, DC, G, CROSS, true>(A, a0, a1, b0, b1, s_reach);                                   \
  }
CEL_TILE_KERNEL(k_attention, attention_tile, s_k0, s_k1, s_v0, s_v1)

// dq of a tile of 128 tokens of one query head; leaves lse_i and D_i in rows
// for k_attention_dkv.  D_i is <do_i, o_i> with the rounded o_i, except where a
// row's keys all lie in one tile: there, where o_i is large (few values
// averaged) and its rounding would weigh as much as that of ds, it is the sum of
// p_ij <do_i, v_j> in 32 bits, at the price of a wave's products twice on the tiles
// that hold such a row.  Those reach the wave's own rows, and only there is it looked for: looked for
// everywhere, 8,192 tokens took 4 % longer.
// Tiles and bounds are the forward pass's, with three products a step and 32 keys'
// scores in registers at a time: 8,192 tokens in one sequence, 32 heads of 128 over
// 8: 0.70 ms, 1.17 PFLOP/s, matrix cores 65 % busy.  dq has a kernel of its own since
// its sums run over the other axis than dk's and dv's: joined, one side would be
// added up in memory, by atomics in no fixed order.  The price is that scores and
// their gradients are made twice, 7 products where 5 would do.
template <class T, int DP, int DC, int G, bool CROSS, bool CAREFUL>
__device__ __forceinline__ bool dq_tile(const AttnArgs &A, char *s_k0, char *s_k1, char *s_v0, char *s_v1,
                                        int (*s_reach)[kWaves]) {
  constexpr int kTile = kStep * DP * 2;
  constexpr int NB = CAREFUL ? 1 : (DC + 31) / 32;  // sums a pass holds, see CEL_TILE_KERNEL
  const int tid = threadIdx.x % (kWaves * 64), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int group = G > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / (kWaves * 64)) : 0;
  const Item item = item_of(blockIdx.x, gridDim.x, A.H);
  const int head = item.unit, kvh = head / (A.H / A.K);
  const int tile = CROSS ? A.order ? A.order[item.tile] : item.tile : A.tiles - 1 - item.tile;
  const int first = tile * kBlock + wave * kRows, i = first + (lane & 31);
  Reach R = reach_of<CROSS>(A, i, true, s_reach + 2 * group, wave);
  const int from = R.from, steps = CROSS ? share_of_keys(A, R) : R.steps();
  u32x4 q[DC / 16], g[DC / 16];
  load_rows(q, A.q, head, i, A.T, A.d, lane);
  load_rows(g, A.dout, head, i, A.T, A.d, lane);
  float D = 0.f;
  {
    u32x4 o[DC / 16];
    load_rows(o, A.out, head, i, A.T, A.d, lane);
#pragma unroll
    for (int kk = 0; kk < DC / 16; kk++) {
      const typename Half<T>::v8 x = __builtin_bit_cast(typename Half<T>::v8, g[kk]);
      const typename Half<T>::v8 y = __builtin_bit_cast(typename Half<T>::v8, o[kk]);
#pragma unroll
      for (int e = 0; e < 8; e++) D = fmaf((float)x[e], (float)y[e], D);
    }
    D = half_sum(D);
  }
  const bool few = CROSS && __any(R.real() && R.hi - R.lo < kStep);
  const float lse2 = R.real() ? A.lse[(int64_t)head * A.T + i] * kLog2e : INFINITY;
  const float c = A.scale * kLog2e;
  const Lane<DP> L(lane);
  const Stager<DP> ks(A.k, A.d, tid), vs(A.v, A.d, tid);
  const int64_t k_head = 2 * kvh * A.k.head, v_head = 2 * kvh * A.v.head;
  // from block n0 of 32 dimensions on
  auto pass = [&](int n0) {
    const int cols = L.cols ^ (n0 << 6);
    acc16 dq[NB];
    int up = kUp<T>;
    auto load = [&](int t, auto buf) {
      const int a = R.from + (t * G + group) * kStep;
      ks.load((buf.at ? s_k1 : s_k0) + group * kTile, k_head, a, R.to + 1, wave);
      vs.load((buf.at ? s_v1 : s_v0) + group * kTile, v_head, a, R.to + 1, wave);
    };
    auto step = [&](int t0, auto buf) {
      const int a = R.from + (t0 * G + group) * kStep;
      if (R.skips(a)) return;
      const char *s_k = (buf.at ? s_k1 : s_k0) + group * kTile, *s_v = (buf.at ? s_v1 : s_v0) + group * kTile;
      const bool masked = R.masks(a);
      const int lo = R.lo - a, hi = R.hi - a;
      // All of a row's keys, of which it is itself the last: not in tiles before the wave's own rows.
      // Keys apart from the rows lie anywhere, and are looked for where a row of the wave has few enough.
      const bool looked = CROSS ? few : a + kStep > first;
      const bool inside = looked && R.real() && lo >= 0 && hi < kStep;
      if (looked && __any(inside)) {
        float sum = 0.f;
#pragma unroll
        for (int t = 0; t < 2; t++) {
          acc16 s, dp;
          rows_products<T, DP>(s, s_k, t, q, dp, s_v, t, g, L.rows, a);
#pragma unroll
          for (int r = 0; r < 16; r++) s[r] = exp2_(fmaf(s[r], c, -lse2)) * dp[r];
          mask(s, t, lo, hi, 0.f, lane);
#pragma unroll
          for (int r = 0; r < 16; r++) sum += s[r];
        }
        sum = half_sum(sum);
        D = inside ? sum : D;
      }
#pragma unroll
      for (int t = 0; t < 2; t++) {
        acc16 s, dp;
        rows_products<T, DP>(s, s_k, t, q, dp, s_v, t, g, L.rows, a);
        const float lift = up - lse2;
#pragma unroll
        for (int r = 0; r < 16; r++) s[r] = exp2_(fmaf(s[r], c, lift)) * (dp[r] - D);
        if (masked) mask(s, t, lo, hi, 0.f, lane);
        if constexpr (kScaled<T>) {
          float top = 0.f;
#pragma unroll
          for (int r = 0; r < 16; r++) top = fmaxf(top, fabsf(s[r]));
          if (__any(top > kTop)) {
            const int down = down_by(half_max(top));
            up += down;
            const float by = power(down);
            s *= by;
#pragma unroll
            for (int n = 0; n < NB; n++) dq[n] *= by;
          }
        }
        const u32x4 ds[2] = {operand<T>(s, 0), operand<T>(s, 1)};
        product<T, DP, CAREFUL>(s_k + t * 32 * Lane<DP>::RB, dq, ds, cols, masked, lo - 32 * t, hi - 32 * t, lane, a);
      }
    };
    auto clear = [&] {
#pragma unroll
      for (int n = 0; n < NB; n++) dq[n] = acc16{};
    };
    clear();
    through_tiles<CAREFUL>((steps + G - 1) / G, load, step);
    const float back = power(-up), by = A.scale * back;
    if (!CAREFUL && __syncthreads_or(R.real() && not_finite(dq, by))) return false;
    if constexpr (G > 1) {
      float *theirs = reinterpret_cast<float *>((wave & 2 ? s_k1 : s_k0) + (wave & 1) * kTile) + lane;
      float *their_D = reinterpret_cast<float *>(s_v0) + wave * 64 + lane;
      if (CAREFUL) __syncthreads();
      if (group) {
#pragma unroll
        for (int n = 0; n < NB; n++)
#pragma unroll
          for (int r = 0; r < 16; r++) theirs[(16 * n + r) * 64] = dq[n][r] * back;
        *their_D = D;
      }
      __syncthreads();
      if (!group) {
#pragma unroll
        for (int n = 0; n < NB; n++)
#pragma unroll
          for (int r = 0; r < 16; r++) dq[n][r] = dq[n][r] * back + theirs[(16 * n + r) * 64];
        const int t = (R.lo - from) / kStep;  // the tile with all of the row's keys, if there is one
        if (R.real() && (R.hi - from) / kStep == t && t & 1) D = *their_D;
      }
    }
    if (i < A.T && group == 0) {
      if (!R.real()) clear();
      bool states = true;  // whether this workgroup's D is the row's: of a row with its keys in one tile, that one's
      if (CROSS && G == 1 && A.splits > 1) {
        store_split(A, head, i, dq, n0, by, lane);
        const int t = (R.lo - from) / kStep, here = (R.from - from) / kStep;
        states = R.real() && (R.hi - from) / kStep == t ? t >= here && t < here + steps : blockIdx.y == 0;
      } else {
        store_rows<T>(A.dq, head, i, dq, n0, G > 1 ? A.scale : by, A.d, lane);
      }
      if (lane < 32 && states) {
        A.rows[(int64_t)head * A.T + i] = lse2 - kPUp<T>;
        A.rows[((int64_t)A.H + head) * A.T + i] = D;
      }
    }
    return true;
  };
  if constexpr (!CAREFUL) return pass(0);
#pragma unroll 1
  for (int n0 = 0; n0 < (DC + 31) / 32; n0++) (void)pass(n0);
  return true;
}
CEL_TILE_KERNEL(k_attention_dq, dq_tile, s_k0, s_k1, s_v0, s_v1)

// lse (which = 0) or D (1) of rows [a, a + kStep) to LDS, one behind the other; 0 at or past `end`.
__device__ __forceinline__ void load_row_values(float *lds, const AttnArgs &A, int which, int head, int a, int end,
                                                int lane) {
  const float *from = A.rows + ((int64_t)which * A.H + head) * A.T + a;
  const int rows = min(end - a, kStep);
  const __amdgpu_buffer_rsrc_t buf =
      __builtin_amdgcn_make_buffer_rsrc(const_cast<float *>(from), 0, rows > 0 ? 4 * rows : 0, 0x00020000);
  __builtin_amdgcn_raw_ptr_buffer_load_lds(buf, (__attribute__((address_space(3))) void *)(lds + which * kStep), 4, 4 * lane,
                                           0, 0, 0);
}
// The same as load_rows for 16 columns: dimensions 32 kk + 8 (lane / 16) + 0..7.
template <int KK>
__device__ inline void load_rows16(u32x4 (&f)[KK], const Rows &x, int head, int i, int end, int d, int lane) {
  const char *p = x.p + 2 * ((int64_t)i * x.row + (int64_t)head * x.head);
#pragma unroll
  for (int kk = 0; kk < KK; kk++) {
    const int c = 32 * kk + 8 * (lane >> 4);
    f[kk] = i < end && c < d ? *reinterpret_cast<const u32x4 *>(p + 2 * c) : u32x4{0, 0, 0, 0};
  }
}
// Sums of a key's gradients, dimensions 32 n0 + 16 n + 4 (lane / 16) + r: in the
// rows' type, or in 32 bits in A.part where several workgroups share a
// key/value head's query heads.
template <class T, int N>
__device__ __forceinline__ void store_sums(const AttnArgs &A, const Rows &x, int which, int kvh, int part, int j,
                                           const acc4 (&acc)[N], int n0, float by, int lane) {
  char *p = x.p + 2 * ((int64_t)j * x.row + (int64_t)kvh * x.head);
  float *q = A.part + ((((int64_t)part * 2 + which) * A.U + j) * A.K + kvh) * A.d;
#pragma unroll
  for (int n = 0; n < N; n++) {
    const int c = 32 * n0 + 16 * n + 4 * (lane >> 4);
    const acc4 y = acc[n] * by;
    if (c >= A.d) continue;
    if (A.parts == 1) *reinterpret_cast<u32x2 *>(p + 2 * c) = u32x2{pack2<T>(y[0], y[1]), pack2<T>(y[2], y[3])};
    else *reinterpret_cast<acc4 *>(q + c) = y;
  }
}
// Where a workgroup's walk over its query heads and their rows stands.
struct Walk {
  int head, a;
  __device__ void next(const Reach &R) {
    a += kStep;
    if (a > R.to) a = R.from, head++;
  }
};
// CROSS: a part's share of all of a key/value head's query heads and their rows: equal shares of the walk,
// wherever they begin.
__device__ inline Walk share_of_rows(const AttnArgs &A, const Reach &R, int kvh, int part, int &count) {
  const int group = A.H / A.K, steps = R.steps();
  const int64_t all = (int64_t)steps * group, first = all * part / A.parts;
  count = (int)(all * (part + 1) / A.parts - first);
  return Walk{kvh * group + (steps ? (int)(first / steps) : 0), R.from + (steps ? (int)(first % steps) * kStep : 0)};
}
// The query heads of a workgroup: part `part` of those that share head kvh.
__device__ inline void heads_of(const AttnArgs &A, int kvh, int part, int &first, int &count) {
  const int group = A.H / A.K, per = (group + A.parts - 1) / A.parts;
  first = kvh * group + part * per;
  count = min(per, group - part * per);
}

// dk and dv: a wave owns 16 keys, on 16x16x32 matrix instructions.  Their sums
// and operands take half the registers that 32 keys would, so that two waves
// share a SIMD and every product is made once; the reads of LDS a product are
// twice as many, 256 bytes a cycle at the matrix cores' full rate, which is what
// LDS gives.  8,192 tokens in one sequence, 32 heads of 128 over 8: 1.07 ms for four
// products, 1.02 PFLOP/s, matrix cores 49 % busy (32 keys a wave and a launch each for
// dk and dv, five products: 1.55 ms; pairs of waves that hand p over in LDS: 1.62 ms).
//   A result tile D[m][n] puts column n = lane % 16 and rows 4 (lane / 16) + r in
//   register r; two of them are a right operand of 32 rows, in the order
//   16 u + 4 (lane / 16) + r for its value 4 u + r.
constexpr int kKeys = 16, kKeyBlock = kWaves * kKeys;
template <class T>
__device__ inline acc4 mma16(u32x4 a, u32x4 b, acc4 c) {
  typedef typename Half<T>::v8 v8;
  if constexpr (__is_same(T, __bf16))
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
}
// The chunks' order here.  A transposed read takes two chunks each of eight
// rows at once (0..7, 8..15), which have to differ in their upper bits.  A plain
// read takes one chunk of rows 0..3 and 12..15 with the next chunk of rows 4..11
// (that is how a wave's 16-byte reads are grouped), or the other way round:
// each of these halves fills whole pairs of chunks.
template <int DP>
struct Swz16 {
  static __device__ int of(int r) {
    return DP == 128 ? (((r & 7) ^ ((r >> 1) & 4)) << 1) | ((r >> 3) & 1)
                     : ((((r >> 1) & 3) ^ ((r >> 2) & 2)) << 1) | ((r >> 3) & 1);
  }
};
template <int DP>
struct Lane16 {
  static constexpr int RB = 2 * DP;
  int rows, cols;
  __device__ explicit Lane16(int lane) {
    const int i = lane & 15, g = lane >> 4, r = 4 * g + (i >> 2);
    rows = i * RB + ((g ^ Swz16<DP>::of(i)) << 4);
    cols = r * RB + ((((i & 3) >> 1) ^ Swz16<DP>::of(r)) << 4) + 8 * (i & 1);
  }
};
// Rows 16 t + lane % 16, columns 32 kk + 8 (lane / 16) + 0..7.
template <int DP>
__device__ inline u32x4 rows16_at(const char *lds, int rows, int t, int kk) {
  return *reinterpret_cast<const u32x4 *>(lds + (rows ^ (kk << 6)) + t * 16 * Lane16<DP>::RB);
}
// The transpose: column 16 n + lane % 16 as a row, its k the rows 32 j + 16 u + 4 (lane / 16) + 0..3.
template <int DP>
__device__ inline u32x4 cols16_at(const char *lds, int cols, int n, int j) {
  typedef __attribute__((ext_vector_type(4))) short s16x4;
  typedef __attribute__((address_space(3))) s16x4 *lds_ptr;
  u32x4 a;
#pragma unroll
  for (int u = 0; u < 2; u++) {
    const s16x4 x =
        __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(lds + (cols ^ (n << 5)) + (32 * j + 16 * u) * Lane16<DP>::RB));
    const u32x2 y = __builtin_bit_cast(u32x2, x);
    a[2 * u] = y[0];
    a[2 * u + 1] = y[1];
  }
  return a;
}
// x[t] = rows 16 t .. of a staged tile times f, y[t] of another times g.
template <class T, int DP, int KK>
__device__ __forceinline__ void rows16_products(acc4 (&x)[4], const char *lds, const u32x4 (&f)[KK], acc4 (&y)[4],
                                                const char *lds2, const u32x4 (&g)[KK], int rows, int a) {
  rows = fresh(rows, a);
  feed<8 * KK>([&](int n) { return rows16_at<DP>(n < 4 * KK ? lds : lds2, rows, n % 4, n / 4 % KK); },
               [&](int n, u32x4 z) {
                 const int t = n % 4, kk = n / 4 % KK;
                 if (n < 4 * KK) x[t] = mma16<T>(z, f[kk], kk ? x[t] : acc4{});
                 else y[t] = mma16<T>(z, g[kk], kk ? y[t] : acc4{});
               });
}
// acc[n] += (columns of the staged tile)^T b, and its careful form: see product and careful_product.
template <class T, int DP, bool CAREFUL, int NB>
__device__ __forceinline__ void product16(const char *lds, acc4 (&acc)[NB], const u32x4 (&b)[2], int cols, bool masked,
                                          int lo, int hi, int lane, int a0) {
  cols = fresh(cols, a0);
  if (!CAREFUL || !masked) {
    feed<2 * NB>([&](int x) { return cols16_at<DP>(lds, cols, x % NB, x / NB); },
                 [&](int x, u32x4 f) { acc[x % NB] = mma16<T>(f, b[x / NB], acc[x % NB]); });
    return;
  }
#pragma unroll
  for (int j = 0; j < 2; j++)
#pragma unroll
    for (int n = 0; n < NB; n++) {
      u32x4 a = cols16_at<DP>(lds, cols, n, j), off;
#pragma unroll
      for (int w = 0; w < 4; w++) {
        const uint32_t m = not_numbers<T>(a[w]);
        off[w] = a[w] & m;
        a[w] &= ~m;
      }
      acc[n] = mma16<T>(a, b[j], acc[n]);
      if (!__any((off[0] | off[1] | off[2] | off[3]) != 0)) continue;
#pragma unroll 1
      for (int k = 0; k < 32; k++) {
        const int e = (k >> 4) * 4 + (k & 3), x = 32 * j + k;
        const uint32_t keep = (lane >> 4) == ((k >> 2) & 3) ? (e & 1 ? 0xffff0000u : 0xffffu) : 0u;
        u32x4 only;
#pragma unroll
        for (int w = 0; w < 4; w++) only[w] = w == (e >> 1) ? off[w] & keep : 0u;
        const acc4 one = mma16<T>(only, b[j], acc4{});
#pragma unroll
        for (int r = 0; r < 4; r++) acc[n][r] = x >= lo && x <= hi ? acc[n][r] + one[r] : acc[n][r];
      }
    }
}

// dk and dv of a tile of 64 tokens of one key/value head: each wave 16 of them,
// over the query heads and the rows up to the end of the last token's sequence,
// in that order whatever the launch.
template <class T, int DP, int DC, bool CROSS, bool CAREFUL>
__device__ __forceinline__ bool dkv_tile(const AttnArgs &A, char *s_q0, char *s_q1, char *s_g0, char *s_g1, float *s_r0,
                                         float *s_r1, int (*s_reach)[kWaves]) {
  constexpr int NB = CAREFUL ? 2 : DC / 16, KK = (DC + 31) / 32;  // sums a pass holds, see CEL_TILE_KERNEL
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g4 = 4 * (lane >> 4);
  const Item item = item_of(blockIdx.x, gridDim.x, A.K * A.parts);
  const int kvh = item.unit / A.parts, part = item.unit % A.parts;
  const int tile = CROSS && A.k_order ? A.k_order[item.tile] : item.tile;
  const int j = tile * kKeyBlock + wave * kKeys + (lane & 15);  // this lane's key
  int head0, heads;
  heads_of(A, kvh, part, head0, heads);
  const Reach R = reach_of<CROSS>(A, j, false, s_reach, wave);
  u32x4 k[KK], v[KK];
  load_rows16(k, A.k, kvh, j, A.U, A.d, lane);
  load_rows16(v, A.v, kvh, j, A.U, A.d, lane);
  const float c = A.scale * kLog2e;
  const Lane16<DP> L(lane);
  const Stager<DP, Swz16<DP>> qs(A.q, A.d, tid), gs(A.dout, A.d, tid);
  int all = R.steps() * heads;
  Walk start{head0, R.from};
  if constexpr (CROSS) start = share_of_rows(A, R, kvh, part, all);
  Walk copies, steps;
  auto load = [&](int, auto buf) {
    qs.load(buf.at ? s_q1 : s_q0, 2 * copies.head * A.q.head, copies.a, R.to + 1, wave);
    gs.load(buf.at ? s_g1 : s_g0, 2 * copies.head * A.dout.head, copies.a, R.to + 1, wave);
    if (wave < 2) load_row_values(buf.at ? s_r1 : s_r0, A, wave, copies.head, copies.a, R.to + 1, lane);
    copies.next(R);
  };
  auto pass = [&](int n0) {
    const int cols = L.cols ^ (n0 << 6);
    acc4 dk[NB], dv[NB];
    int up = kUp<T> - kPUp<T>;  // beside p's
    auto step = [&](int, auto buf) {
      const int a = steps.a;
      steps.next(R);
      if (R.skips(a)) return;
      const char *s_q = buf.at ? s_q1 : s_q0, *s_g = buf.at ? s_g1 : s_g0;
      const float *s_lse = buf.at ? s_r1 : s_r0, *s_D = s_lse + kStep;
      const bool masked = R.masks(a);
      const int lo = R.lo - a, hi = R.hi - a;  // of the 64 rows, those that see this key
      acc4 s[4], dp[4];
      rows16_products<T, DP>(s, s_q, k, dp, s_g, v, L.rows, a);
#pragma unroll
      for (int t = 0; t < 4; t++)
#pragma unroll
        for (int r = 0; r < 4; r++) {
          s[t][r] = exp2_(fmaf(s[t][r], c, -s_lse[16 * t + g4 + r]));
          dp[t][r] = s[t][r] * (dp[t][r] - s_D[16 * t + g4 + r]);
        }
      if (masked) {
        int from = lo - g4, to = hi - g4;
        // hides where the bounds come from: they are compared with constants, not
        // with 16 numbers of each lane's that would stay in registers across the loop
        asm volatile("" : "+v"(from), "+v"(to));
#pragma unroll
        for (int t = 0; t < 4; t++)
#pragma unroll
          for (int r = 0; r < 4; r++) {
            const int x = 16 * t + r;
            const bool seen = x >= from && x <= to;
            s[t][r] = seen ? s[t][r] : 0.f;
            dp[t][r] = seen ? dp[t][r] : 0.f;
          }
      }
      if constexpr (kScaled<T>) {
        const float lift = power(up);
        float top = 0.f;
#pragma unroll
        for (int t = 0; t < 4; t++)
#pragma unroll
          for (int r = 0; r < 4; r++) {
            dp[t][r] *= lift;
            top = fmaxf(top, fabsf(dp[t][r]));
          }
        if (__any(top > kTop)) {
          top = fmaxf(top, __shfl_xor(top, 16));
          const int down = down_by(half_max(top));
          up += down;
          const float by = power(down);
#pragma unroll
          for (int t = 0; t < 4; t++) dp[t] *= by;
#pragma unroll
          for (int n = 0; n < NB; n++) dk[n] *= by;
        }
      }
      u32x4 p[2], ds[2];
#pragma unroll
      for (int t = 0; t < 4; t++)
#pragma unroll
        for (int w = 0; w < 2; w++) {
          p[t / 2][2 * (t % 2) + w] = pack2<T>(s[t][2 * w], s[t][2 * w + 1]);
          ds[t / 2][2 * (t % 2) + w] = pack2<T>(dp[t][2 * w], dp[t][2 * w + 1]);
        }
      product16<T, DP, CAREFUL>(s_g, dv, p, cols, masked, lo, hi, lane, a);
      product16<T, DP, CAREFUL>(s_q, dk, ds, cols, masked, lo, hi, lane, a);
    };
    auto clear = [&] {
#pragma unroll
      for (int n = 0; n < NB; n++) dk[n] = dv[n] = acc4{};
    };
    clear();
    copies = steps = start;
    through_tiles<CAREFUL>(all, load, step);
    const float by = A.scale * power(-up - kPUp<T>);
    bool odd = false;
#pragma unroll
    for (int n = 0; n < NB; n++)
#pragma unroll
      for (int r = 0; r < 4; r++) odd |= !(fabsf(dk[n][r] * by) < INFINITY) || !(fabsf(dv[n][r]) < INFINITY);
    if (!CAREFUL && __syncthreads_or(R.real() && odd)) return false;
    if (j < A.U) {
      if (!R.real()) clear();
      store_sums<T>(A, A.dk, 0, kvh, part, j, dk, n0, by, lane);
      store_sums<T>(A, A.dv, 1, kvh, part, j, dv, n0, power(-kPUp<T>), lane);
    }
    return true;
  };
  if constexpr (!CAREFUL) return pass(0);
#pragma unroll 1
  for (int n0 = 0; n0 < (DC + 31) / 32; n0++) (void)pass(n0);
  return true;
}
template <class T, int DP, int DC, bool CROSS>
// Beyond 64 dimensions the bound leaves the compiler more registers than two waves
// have: it takes 237 of their 256 and keeps the reads of LDS ahead of their use,
// which it gives up under the tighter bound (8,192 tokens, 32 heads of 128 over 8:
// 1.06 against 1.27 ms).
__global__ void __launch_bounds__(kWaves * 64, DC > 64 ? 1 : 2) k_attention_dkv(AttnArgs A) {
  constexpr int kTile = kStep * DP * 2;
  __shared__ __align__(16) char s_q0[kTile], s_q1[kTile], s_g0[kTile], s_g1[kTile];
  __shared__ __align__(16) float s_r0[2 * kStep], s_r1[2 * kStep];  // lse and D of the rows
  __shared__ int s_reach[2][kWaves];
  if (!dkv_tile<T, DP, DC, CROSS, false>(A, s_q0, s_q1, s_g0, s_g1, s_r0, s_r1, s_reach))
    (void)dkv_tile<T, DP, DC, CROSS, true>(A, s_q0, s_q1, s_g0, s_g1, s_r0, s_r1, s_reach);
}

// dk and dv as the sums of their parts, in the order of the query heads.  Bound by
// memory: 2 parts of 8,192 tokens of 8 heads of 128, 101 MB, in 26 us (3.9 TB/s).
template <class T>
__global__ void __launch_bounds__(256) k_attention_join(AttnArgs A) {
  const int64_t n = (int64_t)A.U * A.K * A.d, at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (at >= n) return;
  const int c = (int)(at % A.d), kvh = (int)(at / A.d % A.K);
  const int64_t t = at / A.d / A.K;
#pragma unroll
  for (int which = 0; which < 2; which++) {
    acc4 sum = {0, 0, 0, 0};
    for (int p = 0; p < A.parts; p++) sum += *reinterpret_cast<const acc4 *>(A.part + (p * 2 + which) * n + at);
    const Rows &x = which ? A.dv : A.dk;
    *reinterpret_cast<u32x2 *>(x.p + 2 * (t * x.row + kvh * x.head + c)) = u32x2{pack2<T>(sum[0], sum[1]), pack2<T>(sum[2], sum[3])};
  }
}

// The tiles of rows (blockIdx.x = 0) and of keys (1) in the order of how many steps
// they walk, the longest first: with lengths apart from each other on the two sides, how long a tile
// takes does not follow from where it is, and a long one that starts at a launch's end is
// waited for alone.  37 sequences of 16 to 1,957 tokens and 0 to 1,288 states, 24 heads of 80 over 4, between events:
// forward 98 -> 79 us, dq 122 -> 101, dk and dv 186 -> 126, together 411 -> 328, for 5 us here, twice.  Lengths lie on
// the device, so that a batch of equal ones pays too: two of 4,096, 32 heads of 128 over 8, 2,270 -> 2,277.
constexpr int kOrderB = 1024, kOrderMost = 4096;  // threads; tiles that are ordered, at most
__global__ void __launch_bounds__(kOrderB) k_attention_order(AttnArgs A) {
  __shared__ int s_at[kOrderB], s_sum[kOrderB / 64];
  const bool keys = blockIdx.x != 0;
  const int32_t *own = keys ? A.k_ptr : A.ptr, *other = keys ? A.ptr : A.k_ptr;
  int32_t *order = keys ? A.k_order : A.order;
  const int n = keys ? A.U : A.T, m = keys ? A.T : A.U, size = keys ? kKeyBlock : kBlock, tiles = (n + size - 1) / size;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (!order) return;
  s_at[tid] = 0;
  __syncthreads();
  int bin[kOrderMost / kOrderB];
#pragma unroll
  for (int k = 0; k < kOrderMost / kOrderB; k++) {
    const int tile = k * kOrderB + tid;
    bin[k] = 0;
    if (tile >= tiles) continue;
    const int first = tile * size, last = min(n, first + size) - 1;
    int lo[2] = {0, 0}, hi[2] = {A.S, A.S};  // the last sequences that begin at or before the two
    while (lo[0] < hi[0] || lo[1] < hi[1]) {
#pragma unroll
      for (int x = 0; x < 2; x++) {
        if (lo[x] >= hi[x]) continue;
        const int mid = (lo[x] + hi[x] + 1) >> 1;
        if (own[mid] <= (x ? last : first)) lo[x] = mid;
        else hi[x] = mid - 1;
      }
    }
    const int64_t from = max(other[lo[0]], 0), to = min(other[min(lo[1] + 1, A.S)], m);
    bin[k] = kOrderB - 1 - (int)min(max((to - from + kStep - 1) / kStep, (int64_t)0), (int64_t)kOrderB - 1);
    atomicAdd(&s_at[bin[k]], 1);
  }
  __syncthreads();
  const int count = s_at[tid];
  int up = count;
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(up, o);
    if (lane >= o) up += y;
  }
  if (lane == 63) s_sum[wave] = up;
  __syncthreads();
  for (int w = 0; w < wave; w++) up += s_sum[w];
  s_at[tid] = up - count;
  __syncthreads();
  // tiles of as many steps stand in any order, which no result depends on
#pragma unroll
  for (int k = 0; k < kOrderMost / kOrderB; k++) {
    const int tile = k * kOrderB + tid;
    if (tile < tiles) order[atomicAdd(&s_at[bin[k]], 1)] = tile;
  }
}

// Rows of the forward pass (DQ: of dq) as the sums of the shares of their keys, in the keys' order,
// the forward pass's over the largest of their maxima.  Bound by latency: 32 shares of 16 rows of 128, 0.3 MB, in
// 20 us forward, two loops of dependent loads.
template <class T, bool DQ>
__global__ void __launch_bounds__(256) k_attention_unite(AttnArgs A) {
  const int64_t rows = (int64_t)A.H * A.T, at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (at >= rows * A.d) return;
  const int c = (int)(at % A.d);
  const int64_t row = at / A.d;
  const int head = (int)(row / A.T), i = (int)(row % A.T);
  acc4 sum = {0, 0, 0, 0};
  float by = 1.f;
  if constexpr (DQ) {
    for (int p = 0; p < A.splits; p++) sum += *reinterpret_cast<const acc4 *>(A.split + (p * rows + row) * A.d + c);
  } else {
    const f32x2 *stats = reinterpret_cast<const f32x2 *>(A.split + A.splits * rows * A.d) + row;
    const float scale = A.scale * kLog2e;
    float m = -INFINITY, l = 0.f;
    for (int p = 0; p < A.splits; p++) m = fmaxf(m, stats[p * rows][0]);
    for (int p = 0; p < A.splits; p++) {
      const f32x2 x = stats[p * rows];
      // A share without a maximum has no key that the row sees, and sums of 0; or only scores of minus infinity or
      // that are no numbers, and the sums tell: 0 times what is no number stays that.
      const float w = x[0] == -INFINITY ? 0.f : exp2_((x[0] - m) * scale);
      l += x[1] * w;
      sum += *reinterpret_cast<const acc4 *>(A.split + (p * rows + row) * A.d + c) * w;
    }
    const bool real = !(stats[0][1] < 0.f);
    by = real ? 1.f / l : 0.f;
    if (!real) sum = acc4{0, 0, 0, 0};
    if (c == 0) A.lse[row] = real ? ((m == -INFINITY ? 0.f : m * scale) + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
  }
  const Rows &x = DQ ? A.dq : A.out;
  *reinterpret_cast<u32x2 *>(x.p + 2 * ((int64_t)i * x.row + (int64_t)head * x.head + c)) =
      u32x2{pack2<T>(sum[0] * by, sum[1] * by), pack2<T>(sum[2] * by, sum[3] * by)};
}
template <class T, bool DQ>
void unite(const AttnArgs &A, hipStream_t s) {
  if (A.splits == 1) return;
  KTimer kt(s, "k_attention_unite");
  k_attention_unite<T, DQ><<<(unsigned)(((int64_t)A.H * A.T * A.d / 4 + 255) / 256), 256, 0, s>>>(A);
}

// ------------------------------------------------------------- entry points
// A view's address and strides: 16-byte loads and stores of whole chunks.
int check_rows(const cel_rows *x, const cel_attn *a, const char *fn, const char *what) {
  if (!x || !x->p) return set_error(CEL_E_ARG, "%s: %s is NULL", fn, what);
  if ((reinterpret_cast<uintptr_t>(x->p) & 15) || x->row % 8 || x->head % 8)
    return set_error(CEL_E_ARG, "%s: %s is not aligned to 16 bytes in its address and strides", fn, what);
  if (x->row < a->dim || x->head < 0 || x->row > (1 << 23) || x->head > (int64_t(1) << 40))
    return set_error(CEL_E_ARG, "%s: %s has a stride out of range", fn, what);
  return CEL_OK;
}
// A launch has fewer than 2^32 threads: that many workgroups at most, for tiles of `rows` tokens.
int check_grid(const cel_attn *a, int32_t tokens, int rows, const char *fn) {
  if (((int64_t)tokens + rows - 1) / rows * a->heads * (kWaves * 64) > UINT32_MAX)
    return set_error(CEL_E_ARG, "%s: %d tokens of %d heads", fn, tokens, a->heads);
  return CEL_OK;
}
int check_attn(const cel_attn *a, const char *fn) {
  if (!a) return set_error(CEL_E_ARG, "%s: NULL descriptor", fn);
  if (a->type != CEL_BF16 && a->type != CEL_F16) return set_error(CEL_E_ARG, "%s: type %d", fn, a->type);
  if (a->tokens < 0 || a->n_seq < 0 || a->tokens > INT32_MAX - 4096 || a->n_seq > INT32_MAX - 4096)
    return set_error(CEL_E_ARG, "%s: tokens %d, n_seq %d", fn, a->tokens, a->n_seq);
  if (a->heads < 1 || a->kv_heads < 1 || a->heads > 65535 || a->heads % a->kv_heads)
    return set_error(CEL_E_ARG, "%s: %d heads over %d key/value heads", fn, a->heads, a->kv_heads);
  if (a->dim < 8 || a->dim > 128 || a->dim % 8)
    return set_error(CEL_E_ARG, "%s: dim %d is not a multiple of 8 in 8..128", fn, a->dim);
  const float c = a->scale * kLog2e;  // of the exponents, to the base of 2
  if (!(c > 0.f) || !std::isfinite(c) || !std::isfinite(8.f / c))
    return set_error(CEL_E_ARG, "%s: scale %g is not positive and finite, in units of log 2 too", fn, (double)a->scale);
  return check_grid(a, a->tokens, kBlock, fn);  // the forward pass's and dq's launch
}
// Into how many workgroups a tile of keys deals out the query heads that share
// them: as many as bring six workgroups to each of the 256 compute units (the
// tiles at a long sequence's beginning take many times the average), each with the
// same number of heads but the last.  (Against four: 37 ragged sequences, 24 heads of 80
// over 4: 184 us with the join against 208; 8,192 tokens, 32 heads of 128 over 8: 1.15 ms against
// 1.20; but 4 sequences of 1,024, 32 heads over 8: 145 against 131 us.)
int parts_of(const cel_attn *a, int32_t keys) {
  const int64_t group = a->heads / a->kv_heads, tiles = ((int64_t)keys + kKeyBlock - 1) / kKeyBlock;
  const int64_t per = std::max<int64_t>(1, group * tiles * a->kv_heads / 1536);
  return per >= group ? 1 : (int)((group + per - 1) / per);
}
// Where the parts begin in the backward pass's scratch, in floats: behind lse and D of every row, on
// the 16 bytes of the vectors that they are written and read as.
int64_t part_at(const cel_attn *a) { return (2 * (int64_t)a->heads * a->tokens + 3) / 4 * 4; }
Rows rows_of(const cel_rows *x) { return Rows{static_cast<char *>(x->p), x->row, x->head}; }
AttnArgs args_of(const cel_attn *a) {
  AttnArgs A{};
  A.q = rows_of(&a->q), A.k = rows_of(&a->k), A.v = rows_of(&a->v);
  A.ptr = a->seq_ptr;
  A.S = a->n_seq, A.T = A.U = a->tokens, A.H = a->heads, A.K = a->kv_heads, A.d = a->dim;
  A.tiles = (a->tokens + kBlock - 1) / kBlock;
  A.scale = a->scale;
  A.splits = 1;
  return A;
}

// Whether a kernel's workgroups share their keys between two groups of waves: where
// there are no more of them than the GPU's 256 compute units, each then with as many
// waves as two workgroups would give it, and tokens enough for the join, about 1 us,
// to be won back.  One head of 64 over a sequence of 2,048 tokens: forward
// 33.0 -> 26.7 us, dq 41.9 -> 35.2; of 128: forward 45.3 -> 36.1; 8 heads of 64 over 4,096:
// 57.5 -> 45.2 and 73.1 -> 59.4; but at 512 workgroups (4 sequences of 1,024, 16 heads of
// 64) 23.9 -> 32.3 and 31.6 -> 43.6, and at 64 tokens 7.4 -> 8.6.  The tokens are the batch's: how
// long its sequences are only the device knows.  Where all are short the second group
// has nothing to do and costs up to 1.4 us (8 heads of 64, 16 sequences of 128: forward 10.2 -> 10.6,
// dq 13.0 -> 14.2; 600 of 1: 10.6 -> 10.7 and 14.4 -> 15.0; 4 of 512: 14.7 -> 13.7 and 18.0 -> 18.1).
bool split_keys(const AttnArgs &A) { return A.splits == 1 && (int64_t)A.tiles * A.H <= 256 && A.U >= 512; }

// kernel<T, DP, DC, ...> for the call's type and dimension: rows are staged DP
// wide (a power of two, for the chunks' order), products run over DC dimensions, in
// the steps of 16 or 32 that each has.  Heads of 65 to 80 (against 96 for them; the same
// bits): 37 ragged sequences, 24 heads of 80 over 4, all three kernels: 397 -> 387 us, their
// cross attention 332 -> 325; one of 4,096 to 4,096, 16 heads over 4: 535 -> 518.  Heads of 33 to 48 and of 97 to 112
// run as 64 and 128, though steps of 16 would win there too (that cross attention with heads of 48 262 -> 254 us, of 112
// 411 -> 400; two sequences of 4,096, 32 heads over 8: 1,273 -> 1,176 and 2,301 -> 2,225): they are
// some twenty kernels more for each of the two.
template <class F>
void by_dim(int d, F f) {
  typedef std::integral_constant<int, 32> c32;
  typedef std::integral_constant<int, 64> c64;
  typedef std::integral_constant<int, 80> c80;
  typedef std::integral_constant<int, 96> c96;
  typedef std::integral_constant<int, 128> c128;
  if (d <= 32) f(c64{}, c32{});
  else if (d <= 64) f(c64{}, c64{});
  else if (d <= 80) f(c128{}, c80{});
  else if (d <= 96) f(c128{}, c96{});
  else f(c128{}, c128{});
}
template <class T, bool CROSS>
void launch_attention(const AttnArgs &A, hipStream_t s) {
  {
    KTimer kt(s, "k_attention");
    by_dim(A.d, [&](auto dp, auto dc) {
      constexpr int DP = decltype(dp)::value, DC = decltype(dc)::value;
      const dim3 grid(A.tiles * A.H, A.splits);
      if (split_keys(A)) k_attention<T, DP, DC, 2, CROSS><<<grid, 2 * kWaves * 64, 0, s>>>(A);
      else k_attention<T, DP, DC, 1, CROSS><<<grid, kWaves * 64, 0, s>>>(A);
    });
  }
  if constexpr (CROSS) unite<T, false>(A, s);
}
template <class T, bool CROSS>
void launch_dq(const AttnArgs &A, hipStream_t s) {
  {
    KTimer kt(s, "k_attention_dq");
    by_dim(A.d, [&](auto dp, auto dc) {
      constexpr int DP = decltype(dp)::value, DC = decltype(dc)::value;
      const dim3 grid(A.tiles * A.H, A.splits);
      if constexpr (DC <= 64) {  // beyond, two groups' dq does not fit in the registers (60 -> 126 us at 2,048 tokens)
        if (split_keys(A)) return k_attention_dq<T, DP, DC, 2, CROSS><<<grid, 2 * kWaves * 64, 0, s>>>(A);
      }
      k_attention_dq<T, DP, DC, 1, CROSS><<<grid, kWaves * 64, 0, s>>>(A);
    });
  }
  if constexpr (CROSS) unite<T, true>(A, s);
}
template <class T, bool CROSS>
void launch_dkv(const AttnArgs &A, hipStream_t s) {
  {
    KTimer kt(s, "k_attention_dkv");
    by_dim(A.d, [&](auto dp, auto dc) {
      k_attention_dkv<T, decltype(dp)::value, decltype(dc)::value, CROSS>
          <<<(A.U + kKeyBlock - 1) / kKeyBlock * A.K * A.parts, kWaves * 64, 0, s>>>(A);
    });
  }
  if (A.parts > 1) {
    KTimer kt(s, "k_attention_join");
    k_attention_join<T><<<(unsigned)(((int64_t)A.U * A.K * A.d / 4 + 255) / 256), 256, 0, s>>>(A);
  }
}

// What the two kinds of attention share of their checks and launches; k_ptr and
// keys are the batch's own where it is causal.
struct Keys {
  bool cross;
  const int32_t *ptr;
  int32_t n;
};
int check_keys(const cel_attn *a, const Keys &k, const char *fn) {
  if (k.n < 0 || k.n > INT32_MAX - 4096) return set_error(CEL_E_ARG, "%s: %d keys", fn, k.n);
  return CEL_OK;
}
int64_t row_tiles(const cel_attn *a) { return ((int64_t)a->tokens + kBlock - 1) / kBlock; }
int64_t key_tiles(const Keys &k) { return ((int64_t)k.n + kKeyBlock - 1) / kKeyBlock; }
// The steps that a tile of `tile` of n tokens walks on the other side of m, if all sequences are as long.
int64_t steps_of(const cel_attn *a, int tile, int64_t n, int64_t m) {
  const double share = std::min(1.0, (double)tile / n + 1.0 / std::max(a->n_seq, 1));
  return (int64_t)(share * m / kStep);
}
// Into how many workgroups the keys of a tile of rows are dealt out where there are few rows: as many as give
// every compute unit two, of eight steps at least, which win back the 4 us of uniting their sums.
// One token of 16 heads of 128 over 4, 16,384 states: 205 -> 33 us; 16 sequences of one token and
// 1,500 states each: 389 -> 45; with the gradient 300 tokens of 4 heads of 128 over 2, 8,000 states: 317 -> 88,
// and 8,000 tokens of 2 heads of 64 over 1, 300 states (whose rows are dealt out): 122 -> 52.
int splits_of(const cel_attn *a, const Keys &k) {
  const int64_t units = row_tiles(a) * a->heads;
  if (!k.cross || units == 0) return 1;
  return (int)std::max<int64_t>(1, std::min(512 / units, steps_of(a, kBlock, a->tokens, k.n) / 8));
}
// The same of the rows of a tile of keys, of all query heads that share them.  Two workgroups a compute unit are
// one round, which is enough for one sequence, whose tiles are as long; of several the longest tile should be no
// longer than a round: one workgroup's share of a sequence of three times the mean, two of two.  Against six
// workgroups a compute unit for every batch: one sequence of 4,096 tokens to 4,096, 16 heads of 80 over 4: 517 -> 512 us;
// 2 of 4,096, 32 of 128 over 8: 2,398 -> 2,372; 4 of 1,024: 395 -> 384; 9 ragged ones, 7,000 to 5,000, 32 of 128
// over 4: 461 -> 443.  One round for all would be 352 in the third, but 487 rather than 326 for 37
// sequences of 16 to 1,957 tokens.
int parts_of(const cel_attn *a, const Keys &k) {
  const int64_t units = key_tiles(k) * a->kv_heads, group = a->heads / a->kv_heads;
  if (!k.cross || units == 0) return parts_of(a, k.n);
  const int64_t parts = std::min(group, (512 * std::min(std::max(a->n_seq, 1), 3) + units - 1) / units);
  return (int)std::max(parts, std::min(512 / units, steps_of(a, kKeyBlock, k.n, a->tokens) * group / 8));
}
// Whether `tiles` tiles of `units` heads are put in order: where more workgroups than the GPU holds at once leave
// an order to choose, and more sequences than one a reason to.
bool ordered(const cel_attn *a, const Keys &k, int64_t tiles, int64_t units) {
  return k.cross && a->n_seq > 1 && tiles * units > 512 && tiles <= kOrderMost;
}
// Where the orders begin in the backward pass's scratch, in 32-bit words.
int64_t order_at(const cel_attn *a, const Keys &k) {
  const int parts = parts_of(a, k);
  return part_at(a) + (parts > 1 ? 2 * (int64_t)parts * k.n * a->kv_heads * a->dim : 0);
}
bool rows_ordered(const cel_attn *a, const Keys &k) { return ordered(a, k, row_tiles(a), a->heads); }
bool keys_ordered(const cel_attn *a, const Keys &k) { return ordered(a, k, key_tiles(k), (int64_t)a->kv_heads * parts_of(a, k)); }
// Bytes of the shares' sums, with each row's maximum and sum (forward) or without.
int64_t split_bytes(const cel_attn *a, const Keys &k, int more) {
  const int64_t splits = splits_of(a, k);
  return splits > 1 ? 4 * splits * a->heads * a->tokens * (a->dim + more) : 0;
}
// Where they begin in the backward pass's scratch, in 32-bit words, on 16 bytes.
int64_t split_at(const cel_attn *a, const Keys &k) {
  return (order_at(a, k) + (rows_ordered(a, k) ? row_tiles(a) : 0) + (keys_ordered(a, k) ? key_tiles(k) : 0) + 3) / 4 * 4;
}
int64_t scratch_of(const cel_attn *a, const Keys &k, const char *fn) {
  CEL_TRY(check_attn(a, fn));
  CEL_TRY(check_keys(a, k, fn));
  return rows_ordered(a, k) ? 4 * row_tiles(a) : split_bytes(a, k, 2);  // few rows are split, many are ordered
}
int64_t grad_scratch(const cel_attn *a, const Keys &k, const char *fn) {
  CEL_TRY(check_attn(a, fn));
  CEL_TRY(check_keys(a, k, fn));
  CEL_TRY(check_grid(a, k.n, kKeyBlock, fn));
  const int64_t split = split_bytes(a, k, 0);
  if (split) return 4 * split_at(a, k) + split;
  return 4 * (order_at(a, k) + (rows_ordered(a, k) ? row_tiles(a) : 0) + (keys_ordered(a, k) ? key_tiles(k) : 0));
}
int put_in_order(const AttnArgs &A, hipStream_t s) {
  if (!A.order && !A.k_order) return CEL_OK;
  KTimer kt(s, "k_attention_order");
  k_attention_order<<<A.k_order ? 2 : 1, kOrderB, 0, s>>>(A);
  CEL_HIP(hipGetLastError());
  return CEL_OK;
}
template <class F>
int by_kind(const cel_attn *a, const Keys &k, F launch) {
  if (a->type == CEL_BF16) k.cross ? launch(__bf16{}, std::true_type{}) : launch(__bf16{}, std::false_type{});
  else k.cross ? launch(_Float16{}, std::true_type{}) : launch(_Float16{}, std::false_type{});
  CEL_HIP(hipGetLastError());
  return CEL_OK;
}
int attention(const cel_attn *a, const Keys &k, const cel_rows *out, float *lse, void *scratch, const char *fn, hipStream_t s) {
  int rc = check_attn(a, fn);
  if (rc || (rc = check_keys(a, k, fn))) return rc;
  if (!a->seq_ptr || !k.ptr) return set_error(CEL_E_ARG, "%s: seq_ptr is NULL", fn);
  if (a->tokens == 0) return CEL_OK;
  if ((rc = check_rows(&a->q, a, fn, "q")) || (k.n && ((rc = check_rows(&a->k, a, fn, "k")) || (rc = check_rows(&a->v, a, fn, "v")))) ||
      (rc = check_rows(out, a, fn, "out")))
    return rc;
  if (!lse) return set_error(CEL_E_ARG, "%s: lse is NULL", fn);
  AttnArgs A = args_of(a);
  A.k_ptr = k.ptr, A.U = k.n;
  A.out = rows_of(out);
  A.lse = lse;
  A.splits = splits_of(a, k);
  if (!scratch && (A.splits > 1 || rows_ordered(a, k))) return set_error(CEL_E_ARG, "%s: scratch is NULL", fn);
  if (rows_ordered(a, k)) {
    A.order = static_cast<int32_t *>(scratch);
    CEL_TRY(put_in_order(A, s));
  }
  A.split = static_cast<float *>(scratch);
  return by_kind(a, k, [&](auto t, auto cross) { launch_attention<decltype(t), decltype(cross)::value>(A, s); });
}
int attention_grad(const cel_attn *a, const Keys &k, const cel_rows *out, const float *lse, const cel_rows *dout, void *scratch_,
                   const cel_rows *dq, const cel_rows *dk, const cel_rows *dv, const char *fn, hipStream_t s) {
  int rc = check_attn(a, fn);
  if (rc || (rc = check_keys(a, k, fn)) || (rc = check_grid(a, k.n, kKeyBlock, fn))) return rc;
  if (!a->seq_ptr || !k.ptr) return set_error(CEL_E_ARG, "%s: seq_ptr is NULL", fn);
  if (a->tokens == 0 && k.n == 0) return CEL_OK;
  if ((a->tokens && ((rc = check_rows(&a->q, a, fn, "q")) || (rc = check_rows(out, a, fn, "out")) ||
                     (rc = check_rows(dout, a, fn, "dout")) || (rc = check_rows(dq, a, fn, "dq")))) ||
      (k.n && ((rc = check_rows(&a->k, a, fn, "k")) || (rc = check_rows(&a->v, a, fn, "v")) ||
               (rc = check_rows(dk, a, fn, "dk")) || (rc = check_rows(dv, a, fn, "dv")))))
    return rc;
  float *scratch = static_cast<float *>(scratch_);
  if ((a->tokens && !lse) || (!scratch && grad_scratch(a, k, fn))) return set_error(CEL_E_ARG, "%s: lse or scratch is NULL", fn);
  AttnArgs A = args_of(a);
  A.k_ptr = k.ptr, A.U = k.n;
  if (a->tokens) A.out = rows_of(out), A.dout = rows_of(dout), A.dq = rows_of(dq);
  if (k.n) A.dk = rows_of(dk), A.dv = rows_of(dv);
  A.lse = const_cast<float *>(lse);
  A.rows = scratch;
  A.parts = parts_of(a, k);
  A.part = scratch + part_at(a);
  A.splits = splits_of(a, k);
  A.split = scratch + split_at(a, k);
  int32_t *orders = reinterpret_cast<int32_t *>(scratch) + order_at(a, k);
  if (rows_ordered(a, k)) A.order = orders, orders += row_tiles(a);
  if (keys_ordered(a, k)) A.k_order = orders;
  CEL_TRY(put_in_order(A, s));
  return by_kind(a, k, [&](auto t, auto cross) {
    if (A.T) launch_dq<decltype(t), decltype(cross)::value>(A, s);
    if (A.U) launch_dkv<decltype(t), decltype(cross)::value>(A, s);
  });
}
// A cross attention's descriptor in the form of the other's.
cel_attn rows_part(const cel_cross_attn *a) {
  return cel_attn{a->type, a->tokens, a->n_seq, a->heads, a->kv_heads, a->dim, a->scale, a->seq_ptr, a->q, a->k, a->v};
}
Keys own_keys(const cel_attn *a) { return Keys{false, a ? a->seq_ptr : nullptr, a ? a->tokens : 0}; }

}  // namespace
}  // namespace cel

using namespace cel;

extern "C" int64_t cel_attention_grad_scratch(const cel_attn *a) {
  return grad_scratch(a, own_keys(a), "cel_attention_grad_scratch");
}
extern "C" int cel_attention(const cel_attn *a, const cel_rows *out, float *lse, hipStream_t s) {
  return attention(a, own_keys(a), out, lse, nullptr, "cel_attention", s);
}
extern "C" int cel_attention_grad(const cel_attn *a, const cel_rows *out, const float *lse, const cel_rows *dout,
                                  void *scratch, const cel_rows *dq, const cel_rows *dk, const cel_rows *dv,
                                  hipStream_t s) {
  return attention_grad(a, own_keys(a), out, lse, dout, scratch, dq, dk, dv, "cel_attention_grad", s);
}

extern "C" int64_t cel_cross_attention_grad_scratch(const cel_cross_attn *a) {
  const char *fn = "cel_cross_attention_grad_scratch";
  if (!a) return set_error(CEL_E_ARG, "%s: NULL descriptor", fn);
  const cel_attn b = rows_part(a);
  return grad_scratch(&b, Keys{true, a->key_ptr, a->keys}, fn);
}
extern "C" int64_t cel_cross_attention_scratch(const cel_cross_attn *a) {
  const char *fn = "cel_cross_attention_scratch";
  if (!a) return set_error(CEL_E_ARG, "%s: NULL descriptor", fn);
  const cel_attn b = rows_part(a);
  return scratch_of(&b, Keys{true, a->key_ptr, a->keys}, fn);
}
extern "C" int cel_cross_attention(const cel_cross_attn *a, const cel_rows *out, float *lse, void *scratch, hipStream_t s) {
  const char *fn = "cel_cross_attention";
  if (!a) return set_error(CEL_E_ARG, "%s: NULL descriptor", fn);
  const cel_attn b = rows_part(a);
  return attention(&b, Keys{true, a->key_ptr, a->keys}, out, lse, scratch, fn, s);
}
extern "C" int cel_cross_attention_grad(const cel_cross_attn *a, const cel_rows *out, const float *lse, const cel_rows *dout,
                                        void *scratch, const cel_rows *dq, const cel_rows *dk, const cel_rows *dv,
                                        hipStream_t s) {
  const char *fn = "cel_cross_attention_grad";
  if (!a) return set_error(CEL_E_ARG, "%s: NULL descriptor", fn);
  const cel_attn b = rows_part(a);
  return attention_grad(&b, Keys{true, a->key_ptr, a->keys}, out, lse, dout, scratch, dq, dk, dv, fn, s);
}
