// Causal attention over a packed batch with grouped heads, and its gradient.
//
// Token i of a sequence sees the tokens j <= i of the same sequence:
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
// adds the unrounded values.
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
  const int32_t *ptr;
  int32_t S, T, H, K, d, tiles;
  float *lse;
  float *rows;  // the backward pass's scratch: lse in units of log 2, D, each [heads][tokens]
  float scale;
};

// A staged tile: kStep rows of DP 16-bit values, in 16-byte chunks.  Chunk c
// of row r lies at position c ^ swz(r) of its row: the 16 rows that a wave's
// plain 16-byte reads touch at once, and the four rows of a transposed read,
// then lie in different banks.
template <int DP>
__device__ inline int swz(int r) {
  return DP == 128 ? ((r & 3) << 2) | ((r >> 2) & 3) : (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
}
template <int DP>
__device__ inline int chunk_at(int r, int c) {  // byte offset
  return r * (DP * 2) + ((c ^ swz<DP>(r)) << 4);
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
template <int DP>
struct Stager {
  static constexpr int C = DP / 8, kLoads = kStep * C / (kWaves * 64), kRowsApart = kWaves * 64 / C;
  const char *base;
  uint32_t at, row;  // this lane's offset in a tile; bytes between rows
  __device__ Stager(const Rows &x, int d, int tid) : base(x.p), row((uint32_t)(2 * x.row)) {
    const int r = tid / C, c = (tid % C) ^ swz<DP>(r);  // the rows of a lane's loads share swz: 16 divides kRowsApart
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
static_assert(Stager<64>::kRowsApart % 16 == 0 && Stager<128>::kRowsApart % 16 == 0, "swz repeats after 16 rows");
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

// acc[n] += (columns of the staged tile)^T b[j], where entry x of the 64 that b
// holds counts only for lo <= x <= hi of its column.  b's other entries are 0,
// which is enough unless the tile holds an infinity or NaN there, which 0
// times it would let in.  The products run on the tile's numbers, in the order
// and to the bits of a tile without others; each row x's infinities and NaN
// are a product of their own, added where the column sees x.
template <class T, int DP, int NB>
__device__ __forceinline__ void careful_product(const char *lds, acc16 (&acc)[NB], const u32x4 (&b)[4], int cols,
                                                int lo, int hi, int lane, int a0) {
  lane = fresh(lane, a0), cols = fresh(cols, a0);
#pragma unroll
  for (int j = 0; j < 4; j++)
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

// The sequence that holds a token: its tokens [a, b), empty if there is none.
// Whatever ptr holds, the range lies within the buffer.
__device__ inline void sequence_of(const AttnArgs &A, int i, int &a, int &b) {
  a = b = 0;
  if (i >= A.T) return;
  int lo = 0, hi = A.S;  // the last s with ptr[s] <= i, if any
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (A.ptr[mid] <= i) lo = mid;
    else hi = mid - 1;
  }
  if (lo >= A.S) return;
  const int from = A.ptr[lo], to = A.ptr[lo + 1];
  if (from > i || to <= i) return;
  a = from < 0 ? 0 : from;
  b = to > A.T ? A.T : to;
}

__device__ inline int wave_min(int x) {
  for (int o = 32; o; o >>= 1) x = min(x, __shfl_xor(x, o));
  return x;
}
__device__ inline int wave_max(int x) {
  for (int o = 32; o; o >>= 1) x = max(x, __shfl_xor(x, o));
  return x;
}

// Work items in an order that gives each of the 8 dies, which take
// workgroups in turn, a stretch of neighbouring items: tiles of one head
// share its keys and values in that die's L2.
__device__ inline int item_of(int block, int blocks) {
  const int x = block & 7, per = blocks >> 3, more = blocks & 7;
  return x * per + min(x, more) + (block >> 3);
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
  __device__ bool skips(int a) const { return a > any_hi || a + kStep <= any_lo; }
  __device__ bool masks(int a) const { return a < all_lo || a + kStep - 1 > all_hi; }
  __device__ int steps() const { return to < from ? 0 : (to - from) / kStep + 1; }
};
// forward: the keys that token i sees; else the rows that see it.
__device__ inline Reach reach_of(const AttnArgs &A, int i, bool forward, int (*s_reach)[kWaves], int wave) {
  int first, last;
  sequence_of(A, i, first, last);
  Reach R;
  const bool real = last > first;
  R.lo = !real ? INT32_MAX : forward ? first : i;
  R.hi = !real ? -1 : forward ? i : last - 1;
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
// Orders what the compiler schedules here: N matrix instructions, each fed by
// READS reads of LDS, with the reads AHEAD instructions before their use.
template <int N, int READS, int AHEAD>
__device__ __forceinline__ void feed() {
  __builtin_amdgcn_sched_group_barrier(0x100, AHEAD * READS, 0);
#pragma unroll
  for (int i = 0; i < N - AHEAD; i++) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
  }
  __builtin_amdgcn_sched_group_barrier(0x008, AHEAD, 0);
}
// acc += (columns of the staged tile)^T b, see careful_product.
template <class T, int DP, bool CAREFUL, int NB>
__device__ __forceinline__ void product(const char *lds, acc16 (&acc)[NB], const u32x4 (&b)[4], int cols, bool masked,
                                        int lo, int hi, int lane, int a) {
  if (CAREFUL && masked) {
    careful_product<T, DP, NB>(lds, acc, b, cols, lo, hi, lane, a);
  } else {
    cols = fresh(cols, a);
#pragma unroll
    for (int j = 0; j < 4; j++)
#pragma unroll
      for (int n = 0; n < NB; n++) acc[n] = Half<T>::mma(cols_at<DP>(lds, cols, n, j), b[j], acc[n]);
    feed<4 * NB, 2, kAhead>();
  }
}
// x = rows 32 t .. of a staged tile times f, y = rows 32 u .. of another times g.
template <class T, int DP, int KK>
__device__ __forceinline__ void rows_products(acc16 &x, const char *lds, int t, const u32x4 (&f)[KK], acc16 &y,
                                              const char *lds2, int u, const u32x4 (&g)[KK], int rows, int a) {
  rows = fresh(rows, a);
  x = y = acc16{};
#pragma unroll
  for (int kk = 0; kk < KK; kk++) {
    x = Half<T>::mma(rows_at<DP>(lds, rows, t, kk), f[kk], x);
    y = Half<T>::mma(rows_at<DP>(lds2, rows, u, kk), g[kk], y);
  }
  feed<2 * KK, 1, kAhead>();
}
// x's entries at 32 t .. of a tile outside lo .. hi, replaced.
__device__ __forceinline__ void mask(acc16 &x, int t, int lo, int hi, float by, int lane) {
#pragma unroll
  for (int r = 0; r < 16; r++) {
    const int at = 32 * t + 8 * (r / 4) + r % 4 + 4 * (lane >> 5);
    x[r] = at >= lo && at <= hi ? x[r] : by;
  }
}

// One tile of 128 tokens of one query head: each wave 32 of them, over the
// keys from the first row's sequence on.
template <class T, int DP, int DC, bool CAREFUL>
__device__ __forceinline__ bool attention_tile(const AttnArgs &A, char *s_k0, char *s_k1, char *s_v0, char *s_v1,
                                               int (*s_reach)[kWaves]) {
  constexpr int NB = CAREFUL ? 1 : DC / 32;  // sums a pass holds, see CEL_TILE_KERNEL
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int item = item_of(blockIdx.x, gridDim.x);
  const int head = item / A.tiles, tile = A.tiles - 1 - item % A.tiles, kvh = head / (A.H / A.K);
  const int i = tile * kBlock + wave * kRows + (lane & 31);  // this lane's row
  const Reach R = reach_of(A, i, true, s_reach, wave);
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
      const int a = R.from + t * kStep;
      ks.load(buf.at ? s_k1 : s_k0, k_head, a, R.to + 1, wave);
      vs.load(buf.at ? s_v1 : s_v0, v_head, a, R.to + 1, wave);
    };
    auto step = [&](int t0, auto buf) {
      const int a = R.from + t0 * kStep;
      if (R.skips(a)) return;
      const char *s_k = buf.at ? s_k1 : s_k0, *s_v = buf.at ? s_v1 : s_v0;
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
      // 2^8 above it: p stays below 2^8, and the sums are seldom rescaled.
      if (__any(top > m + far)) {
        const float to = fmaxf(m, top);
        const float by = to == -INFINITY ? 1.f : exp2_((m - to) * c);
        m = to;
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
    through_tiles<CAREFUL>(R.steps(), load, step);
    // An infinity or NaN may come from a value that the row does not see.
    if (!CAREFUL && __syncthreads_or(R.real() && not_finite(o, 1.f))) return false;
    l = half_sum(l);
    if (i < A.T) {
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
  for (int n0 = 0; n0 < DC / 32; n0++) (void)pass(n0);
  return true;
}

// A workgroup runs its tile without regard to infinities and NaN, and where
// the result has any, all of it again with: nothing of the first run is kept in
// registers for the second, which takes 32 dimensions at a time, so that it
// needs fewer than the first.
#define CEL_TILE_KERNEL(kernel, tile, a0, a1, b0, b1)                            \
  template <class T, int DP, int DC>                                             \
  __global__ void __launch_bounds__(kWaves * 64, 2) kernel(AttnArgs A) {         \
    constexpr int kTile = kStep * DP * 2;                                        \
    __shared__ __align__(16) char a0[kTile], a1[kTile], b0[kTile], b1[kTile];    \
    __shared__ int s_reach[2][kWaves];                                           \
    if (!tile<T, DP, DC, false>(A, a0, a1, b0, b1, s_reach))                     \
      (void)tile<T, DP, DC, true>(A, a0, a1, b0, b1, s_reach);                   \
  }
CEL_TILE_KERNEL(k_attention, attention_tile, s_k0, s_k1, s_v0, s_v1)

// dq of a tile of 128 tokens of one query head; leaves lse_i and D_i in rows
// for k_attention_dkv.  D_i is <do_i, o_i> with the rounded o_i, except where a
// wave's keys all lie in one tile: there, where o_i is large (few values
// averaged) and its rounding would weigh as much as that of ds, it is the sum of
// p_ij <do_i, v_j> in 32 bits, at the price of that tile's products twice.
template <class T, int DP, int DC, bool CAREFUL>
__device__ __forceinline__ bool dq_tile(const AttnArgs &A, char *s_k0, char *s_k1, char *s_v0, char *s_v1,
                                        int (*s_reach)[kWaves]) {
  constexpr int NB = CAREFUL ? 1 : DC / 32;  // sums a pass holds, see CEL_TILE_KERNEL
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int item = item_of(blockIdx.x, gridDim.x);
  const int head = item / A.tiles, tile = A.tiles - 1 - item % A.tiles, kvh = head / (A.H / A.K);
  const int i = tile * kBlock + wave * kRows + (lane & 31);
  const Reach R = reach_of(A, i, true, s_reach, wave);
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
  const float lse2 = R.real() ? A.lse[(int64_t)head * A.T + i] * kLog2e : INFINITY;
  const float c = A.scale * kLog2e;
  const Lane<DP> L(lane);
  const Stager<DP> ks(A.k, A.d, tid), vs(A.v, A.d, tid);
  const int64_t k_head = 2 * kvh * A.k.head, v_head = 2 * kvh * A.v.head;
  // from block n0 of 32 dimensions on
  auto pass = [&](int n0) {
    const int cols = L.cols ^ (n0 << 6);
    acc16 dq[NB];
    auto load = [&](int t, auto buf) {
      const int a = R.from + t * kStep;
      ks.load(buf.at ? s_k1 : s_k0, k_head, a, R.to + 1, wave);
      vs.load(buf.at ? s_v1 : s_v0, v_head, a, R.to + 1, wave);
    };
    auto step = [&](int t0, auto buf) {
      const int a = R.from + t0 * kStep;
      if (R.skips(a)) return;
      const char *s_k = buf.at ? s_k1 : s_k0, *s_v = buf.at ? s_v1 : s_v0;
      const bool masked = R.masks(a);
      const int lo = R.lo - a, hi = R.hi - a;
      if (R.any_lo >= a && R.any_hi < a + kStep) {
        D = 0.f;
#pragma unroll
        for (int t = 0; t < 2; t++) {
          acc16 s, dp;
          rows_products<T, DP>(s, s_k, t, q, dp, s_v, t, g, L.rows, a);
#pragma unroll
          for (int r = 0; r < 16; r++) s[r] = exp2_(fmaf(s[r], c, -lse2)) * dp[r];
          mask(s, t, lo, hi, 0.f, lane);
#pragma unroll
          for (int r = 0; r < 16; r++) D += s[r];
        }
        D = half_sum(D);
      }
      u32x4 ds[4];
#pragma unroll
      for (int t = 0; t < 2; t++) {
        acc16 s, dp;
        rows_products<T, DP>(s, s_k, t, q, dp, s_v, t, g, L.rows, a);
#pragma unroll
        for (int r = 0; r < 16; r++) s[r] = exp2_(fmaf(s[r], c, -lse2)) * (dp[r] - D);
        if (masked) mask(s, t, lo, hi, 0.f, lane);
        ds[2 * t] = operand<T>(s, 0);
        ds[2 * t + 1] = operand<T>(s, 1);
      }
      product<T, DP, CAREFUL>(s_k, dq, ds, cols, masked, lo, hi, lane, a);
    };
    auto clear = [&] {
#pragma unroll
      for (int n = 0; n < NB; n++) dq[n] = acc16{};
    };
    clear();
    through_tiles<CAREFUL>(R.steps(), load, step);
    if (!CAREFUL && __syncthreads_or(R.real() && not_finite(dq, A.scale))) return false;
    if (i < A.T) {
      if (!R.real()) clear();
      store_rows<T>(A.dq, head, i, dq, n0, A.scale, A.d, lane);
      if (lane < 32) {
        A.rows[(int64_t)head * A.T + i] = lse2;
        A.rows[((int64_t)A.H + head) * A.T + i] = D;
      }
    }
    return true;
  };
  if constexpr (!CAREFUL) return pass(0);
#pragma unroll 1
  for (int n0 = 0; n0 < DC / 32; n0++) (void)pass(n0);
  return true;
}
CEL_TILE_KERNEL(k_attention_dq, dq_tile, s_k0, s_k1, s_v0, s_v1)

// dk, dv or both of a tile of 128 tokens of one key/value head: each wave 32
// of them, over the query heads that share it and the rows up to the end of the
// last token's sequence, in that order whatever the launch.
template <class T, int DP, int DC, bool DK, bool DV, bool CAREFUL>
__device__ __forceinline__ bool dkv_tile(const AttnArgs &A, int kvh, int tile, char *s_q0, char *s_q1, char *s_g0,
                                         char *s_g1, float *s_r0, float *s_r1, int (*s_reach)[kWaves]) {
  constexpr int NB = CAREFUL ? 1 : DC / 32;  // sums a pass holds, see CEL_TILE_KERNEL
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h4 = 4 * (lane >> 5);
  const int group = A.H / A.K;
  const int j = tile * kBlock + wave * kRows + (lane & 31);  // this lane's key
  const Reach R = reach_of(A, j, false, s_reach, wave);
  u32x4 k[DC / 16], v[DC / 16];
  load_rows(k, A.k, kvh, j, A.T, A.d, lane);
  if (DK) load_rows(v, A.v, kvh, j, A.T, A.d, lane);
  const float c = A.scale * kLog2e;
  const Lane<DP> L(lane);
  const Stager<DP> qs(A.q, A.d, tid), gs(A.dout, A.d, tid);
  const int steps = R.steps(), all = steps * group;
  int l_head, l_a, s_a;  // where the copies and the steps stand
  auto load = [&](int, auto buf) {
    qs.load(buf.at ? s_q1 : s_q0, 2 * l_head * A.q.head, l_a, R.to + 1, wave);
    gs.load(buf.at ? s_g1 : s_g0, 2 * l_head * A.dout.head, l_a, R.to + 1, wave);
    if (wave < 2) {  // 64 rows' lse by wave 0, their D by wave 1
      const float *from = A.rows + ((int64_t)wave * A.H + l_head) * A.T + l_a;
      const int rows = min(R.to + 1 - l_a, kStep);
      const __amdgpu_buffer_rsrc_t buffer =
          __builtin_amdgcn_make_buffer_rsrc(const_cast<float *>(from), 0, 4 * rows, 0x00020000);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          buffer, (__attribute__((address_space(3))) void *)((buf.at ? s_r1 : s_r0) + wave * kStep), 4, 4 * lane, 0, 0, 0);
    }
    l_a += kStep;
    if (l_a > R.to) l_a = R.from, l_head++;
  };
  // from block n0 of 32 dimensions on
  auto pass = [&](int n0) {
    const int cols = L.cols ^ (n0 << 6);
    acc16 dk[NB], dv[NB];
    auto step = [&](int, auto buf) {
      const int a = s_a;
      s_a = a + kStep > R.to ? R.from : a + kStep;
      if (R.skips(a)) return;
      const char *s_q = buf.at ? s_q1 : s_q0, *s_g = buf.at ? s_g1 : s_g0;
      const float *s_lse = buf.at ? s_r1 : s_r0, *s_D = s_lse + kStep;
      const bool masked = R.masks(a);
      const int lo = R.lo - a, hi = R.hi - a;  // of the 64 rows, those that see this key
      u32x4 p[4], ds[4];
      acc16 s[2], dp[2];
      if (!DK) rows_products<T, DP>(s[0], s_q, 0, k, s[1], s_q, 1, k, L.rows, a);
#pragma unroll
      for (int t = 0; t < 2; t++) {
        if (DK) rows_products<T, DP>(s[t], s_q, t, k, dp[t], s_g, t, v, L.rows, a);
#pragma unroll
        for (int r = 0; r < 16; r++) s[t][r] = exp2_(fmaf(s[t][r], c, -s_lse[32 * t + 8 * (r / 4) + r % 4 + h4]));
        if (masked) mask(s[t], t, lo, hi, 0.f, lane);
        if (DV) {
          p[2 * t] = operand<T>(s[t], 0);
          p[2 * t + 1] = operand<T>(s[t], 1);
        }
        if (DK) {
#pragma unroll
          for (int r = 0; r < 16; r++) dp[t][r] = s[t][r] * (dp[t][r] - s_D[32 * t + 8 * (r / 4) + r % 4 + h4]);
          if (masked) mask(dp[t], t, lo, hi, 0.f, lane);
          ds[2 * t] = operand<T>(dp[t], 0);
          ds[2 * t + 1] = operand<T>(dp[t], 1);
        }
      }
      if (DV) product<T, DP, CAREFUL>(s_g, dv, p, cols, masked, lo, hi, lane, a);
      if (DK) product<T, DP, CAREFUL>(s_q, dk, ds, cols, masked, lo, hi, lane, a);
    };
    auto clear = [&] {
#pragma unroll
      for (int n = 0; n < NB; n++) dk[n] = dv[n] = acc16{};
      l_head = kvh * group, l_a = s_a = R.from;
    };
    clear();
    through_tiles<CAREFUL>(all, load, step);
    if (!CAREFUL && __syncthreads_or(R.real() && ((DK && not_finite(dk, A.scale)) || (DV && not_finite(dv, 1.f))))) return false;
    if (j < A.T) {
      if (!R.real()) clear();
      if (DK) store_rows<T>(A.dk, kvh, j, dk, n0, A.scale, A.d, lane);
      if (DV) store_rows<T>(A.dv, kvh, j, dv, n0, 1.f, A.d, lane);
    }
    return true;
  };
  if constexpr (!CAREFUL) return pass(0);
#pragma unroll 1
  for (int n0 = 0; n0 < DC / 32; n0++) (void)pass(n0);
  return true;
}

// Up to 64 dimensions a wave holds both sums (4 products a tile).  Beyond,
// both would take more than the 256 registers that let two waves share a SIMD:
// a workgroup takes dv (2 products) or dk (3), which computes the scores twice.
template <class T, int DP, int DC>
__global__ void __launch_bounds__(kWaves * 64, 2) k_attention_dkv(AttnArgs A) {
  constexpr int kTile = kStep * DP * 2;
  __shared__ __align__(16) char s_q0[kTile], s_q1[kTile], s_g0[kTile], s_g1[kTile];
  __shared__ __align__(16) float s_r0[2 * kStep], s_r1[2 * kStep];  // lse and D of the rows
  __shared__ int s_reach[2][kWaves];
  auto run = [&](auto dk, auto dv, int item) {
    constexpr bool DK = decltype(dk)::value, DV = decltype(dv)::value;
    const int kvh = item / A.tiles, tile = item % A.tiles;
    if (!dkv_tile<T, DP, DC, DK, DV, false>(A, kvh, tile, s_q0, s_q1, s_g0, s_g1, s_r0, s_r1, s_reach))
      (void)dkv_tile<T, DP, DC, DK, DV, true>(A, kvh, tile, s_q0, s_q1, s_g0, s_g1, s_r0, s_r1, s_reach);
  };
  const int item = item_of(blockIdx.x, gridDim.x);
  if constexpr (DC <= 64) run(std::true_type{}, std::true_type{}, item);
  else if (item & 1) run(std::true_type{}, std::false_type{}, item >> 1);
  else run(std::false_type{}, std::true_type{}, item >> 1);
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
int check_attn(const cel_attn *a, const char *fn) {
  if (!a) return set_error(CEL_E_ARG, "%s: NULL descriptor", fn);
  if (a->type != CEL_BF16 && a->type != CEL_F16) return set_error(CEL_E_ARG, "%s: type %d", fn, a->type);
  if (a->tokens < 0 || a->n_seq < 0 || a->tokens > INT32_MAX - 4096 || a->n_seq > INT32_MAX - 4096)
    return set_error(CEL_E_ARG, "%s: tokens %d, n_seq %d", fn, a->tokens, a->n_seq);
  if (a->heads < 1 || a->kv_heads < 1 || a->heads > 65535 || a->heads % a->kv_heads)
    return set_error(CEL_E_ARG, "%s: %d heads over %d key/value heads", fn, a->heads, a->kv_heads);
  if (a->dim < 8 || a->dim > 128 || a->dim % 8)
    return set_error(CEL_E_ARG, "%s: dim %d is not a multiple of 8 in 8..128", fn, a->dim);
  if (!(a->scale > 0.f) || !std::isfinite(a->scale) || !std::isfinite(8.f / (a->scale * kLog2e)))
    return set_error(CEL_E_ARG, "%s: scale %g is not positive and finite", fn, (double)a->scale);
  if (((int64_t)a->tokens + kBlock - 1) / kBlock * a->heads > INT32_MAX)
    return set_error(CEL_E_ARG, "%s: %d tokens of %d heads", fn, a->tokens, a->heads);
  if (!a->seq_ptr) return set_error(CEL_E_ARG, "%s: seq_ptr is NULL", fn);
  return CEL_OK;
}
Rows rows_of(const cel_rows *x) { return Rows{static_cast<char *>(x->p), x->row, x->head}; }
AttnArgs args_of(const cel_attn *a) {
  AttnArgs A{};
  A.q = rows_of(&a->q), A.k = rows_of(&a->k), A.v = rows_of(&a->v);
  A.ptr = a->seq_ptr;
  A.S = a->n_seq, A.T = a->tokens, A.H = a->heads, A.K = a->kv_heads, A.d = a->dim;
  A.tiles = (a->tokens + kBlock - 1) / kBlock;
  A.scale = a->scale;
  return A;
}

// f<T, DP, DC> for the call's type and dimension: rows are staged DP wide (a
// power of two, for the chunks' order), products run over DC dimensions.
#define CEL_BY_DIM(T, kernel, grid)                                                     \
  do {                                                                                  \
    if (A.d <= 32) kernel<T, 64, 32><<<grid, kWaves * 64, 0, s>>>(A);                   \
    else if (A.d <= 64) kernel<T, 64, 64><<<grid, kWaves * 64, 0, s>>>(A);              \
    else if (A.d <= 96) kernel<T, 128, 96><<<grid, kWaves * 64, 0, s>>>(A);             \
    else kernel<T, 128, 128><<<grid, kWaves * 64, 0, s>>>(A);                           \
  } while (0)
#define CEL_BY_TYPE(kernel, grid)                                                       \
  do {                                                                                  \
    KTimer kt(s, #kernel);                                                              \
    if (a->type == CEL_BF16) CEL_BY_DIM(__bf16, kernel, grid);                          \
    else CEL_BY_DIM(_Float16, kernel, grid);                                            \
    CEL_HIP(hipGetLastError());                                                         \
  } while (0)

}  // namespace
}  // namespace cel

using namespace cel;

extern "C" int cel_attention(const cel_attn *a, const cel_rows *out, float *lse, hipStream_t s) {
  const char *fn = "cel_attention";
  int rc = check_attn(a, fn);
  if (rc) return rc;
  if (a->tokens == 0) return CEL_OK;
  if ((rc = check_rows(&a->q, a, fn, "q")) || (rc = check_rows(&a->k, a, fn, "k")) ||
      (rc = check_rows(&a->v, a, fn, "v")) || (rc = check_rows(out, a, fn, "out")))
    return rc;
  if (!lse) return set_error(CEL_E_ARG, "%s: lse is NULL", fn);
  AttnArgs A = args_of(a);
  A.out = rows_of(out);
  A.lse = lse;
  CEL_BY_TYPE(k_attention, A.tiles * A.H);
  return CEL_OK;
}

extern "C" int cel_attention_grad(const cel_attn *a, const cel_rows *out, const float *lse, const cel_rows *dout,
                                  float *scratch, const cel_rows *dq, const cel_rows *dk, const cel_rows *dv,
                                  hipStream_t s) {
  const char *fn = "cel_attention_grad";
  int rc = check_attn(a, fn);
  if (rc) return rc;
  if (a->tokens == 0) return CEL_OK;
  if ((rc = check_rows(&a->q, a, fn, "q")) || (rc = check_rows(&a->k, a, fn, "k")) ||
      (rc = check_rows(&a->v, a, fn, "v")) || (rc = check_rows(out, a, fn, "out")) ||
      (rc = check_rows(dout, a, fn, "dout")) || (rc = check_rows(dq, a, fn, "dq")) ||
      (rc = check_rows(dk, a, fn, "dk")) || (rc = check_rows(dv, a, fn, "dv")))
    return rc;
  if (!lse || !scratch) return set_error(CEL_E_ARG, "%s: lse or scratch is NULL", fn);
  AttnArgs A = args_of(a);
  A.out = rows_of(out), A.dout = rows_of(dout), A.dq = rows_of(dq), A.dk = rows_of(dk), A.dv = rows_of(dv);
  A.lse = const_cast<float *>(lse);
  A.rows = scratch;
  CEL_BY_TYPE(k_attention_dq, A.tiles * A.H);
  CEL_BY_TYPE(k_attention_dkv, A.tiles * A.K * (A.d <= 64 ? 1 : 2));
  return CEL_OK;
}
