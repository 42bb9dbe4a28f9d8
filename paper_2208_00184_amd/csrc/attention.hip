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

#include "cel_internal.h"

namespace cel {
namespace {

constexpr int kWaves = 4;            // waves of a workgroup
constexpr int kRows = 32;            // tile rows a wave owns
constexpr int kBlock = kWaves * kRows;
constexpr int kStep = 64;            // rows of the other side staged at once
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

// Left operand: rows 32 t + lane % 32, columns 16 kk + 8 (lane / 32) + 0..7.
template <int DP>
__device__ inline u32x4 rows_at(const char *lds, int t, int kk, int lane) {
  return *reinterpret_cast<const u32x4 *>(lds + chunk_at<DP>(32 * t + (lane & 31), 2 * kk + (lane >> 5)));
}
// Left operand of the transpose: its row 32 n + lane % 32 is a column of the
// tile, its k the tile's rows 16 j + 4 (lane / 32) + 0..3 and, behind them,
// those 8 further on.  A transposed read gives lane i of 16 lanes the i-th of
// 16 columns of four rows, of which lane i addresses row i / 4, columns 4 (i % 4) + 0..3.
template <int DP>
__device__ inline u32x4 cols_at(const char *lds, int n, int j, int lane) {
  typedef __attribute__((ext_vector_type(4))) short s16x4;
  typedef __attribute__((address_space(3))) s16x4 *lds_ptr;
  const int i = lane & 15, c = 4 * n + 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
  u32x4 a;
#pragma unroll
  for (int u = 0; u < 2; u++) {
    const int r = 16 * j + 8 * u + 4 * (lane >> 5) + (i >> 2);
    const s16x4 x =
        __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(lds + chunk_at<DP>(r, c) + 8 * (i & 1)));
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
template <class T, int DP, int DC>
__device__ __forceinline__ void careful_product(const char *lds, acc16 (&acc)[DC / 32], const u32x4 (&b)[4],
                                                int lo, int hi, int lane) {
#pragma unroll
  for (int j = 0; j < 4; j++)
#pragma unroll
    for (int n = 0; n < DC / 32; n++) {
      u32x4 a = cols_at<DP>(lds, n, j, lane), off;
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
// A transposed result, acc[n][r] times `by`: dimension 32 n + 8 (r / 4) + 4 (lane / 32) + r % 4 of row i.
template <class T, int N>
__device__ inline void store_rows(const Rows &x, int head, int i, const acc16 (&acc)[N], float by, int d, int lane) {
  char *p = x.p + 2 * ((int64_t)i * x.row + (int64_t)head * x.head);
#pragma unroll
  for (int n = 0; n < N; n++)
#pragma unroll
    for (int g = 0; g < 4; g++) {
      const int c = 32 * n + 8 * g + 4 * (lane >> 5);
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

// One tile of 128 tokens of one query head: each wave 32 of them, over the
// keys from the first row's sequence on.
template <class T, int DP, int DC>
__global__ void __launch_bounds__(kWaves * 64, 2) k_attention(AttnArgs A) {
  constexpr int kTile = kStep * DP * 2;
  __shared__ __align__(16) char s_kv[2][2][kTile];  // two tiles of keys and values: one in use, one on its way
  __shared__ int s_range[2][kWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h4 = 4 * (lane >> 5);
  const int item = item_of(blockIdx.x, gridDim.x);
  const int head = item / A.tiles, tile = A.tiles - 1 - item % A.tiles, kvh = head / (A.H / A.K);
  const int i = tile * kBlock + wave * kRows + (lane & 31);  // this lane's row
  int first, last;                                           // its sequence
  sequence_of(A, i, first, last);
  const bool real = last > first;
  const int w_first = wave_min(real ? first : INT32_MAX), w_last = wave_max(real ? i : -1);
  const int w_upto = wave_min(real ? i : INT32_MAX), w_from = wave_max(real ? first : -1);
  if (lane == 0) {
    s_range[0][wave] = w_first;
    s_range[1][wave] = w_last;
  }
  __syncthreads();
  int k0 = INT32_MAX, k1 = -1;
#pragma unroll
  for (int w = 0; w < kWaves; w++) {
    k0 = min(k0, s_range[0][w]);
    k1 = max(k1, s_range[1][w]);
  }
  u32x4 q[DC / 16];
  load_rows(q, A.q, head, i, A.T, A.d, lane);
  const float c = A.scale * kLog2e, far = 8.f / c;
  const Stager<DP> ks(A.k, A.d, tid), vs(A.v, A.d, tid);
  const int64_t k_head = 2 * kvh * A.k.head, v_head = 2 * kvh * A.v.head;
  acc16 o[DC / 32];
  float m, mc, l;
  for (int careful = 0;; careful = 1) {
#pragma unroll
    for (int n = 0; n < DC / 32; n++) o[n] = acc16{};
    m = -INFINITY, mc = 0.f, l = 0.f;
    int now = 0;
    if (k0 <= k1) {
      ks.load(s_kv[0][0], k_head, k0, k1 + 1, wave);
      vs.load(s_kv[0][1], v_head, k0, k1 + 1, wave);
    }
    for (int a = k0; a <= k1; a += kStep, now ^= 1) {
      next_tile();
      if (a + kStep <= k1) {
        ks.load(s_kv[now ^ 1][0], k_head, a + kStep, k1 + 1, wave);
        vs.load(s_kv[now ^ 1][1], v_head, a + kStep, k1 + 1, wave);
      }
      if (a > w_last || a + kStep <= w_first) continue;
      const char *s_k = s_kv[now][0], *s_v = s_kv[now][1];
      acc16 s[2] = {};
#pragma unroll
      for (int t = 0; t < 2; t++)
#pragma unroll
        for (int kk = 0; kk < DC / 16; kk++) s[t] = Half<T>::mma(rows_at<DP>(s_k, t, kk, lane), q[kk], s[t]);
      const int lo = first - a, hi = i - a;  // of the 64 keys, those that this row sees
      const bool masked = a < w_from || a + kStep - 1 > w_upto;
      if (masked) {
#pragma unroll
        for (int t = 0; t < 2; t++)
#pragma unroll
          for (int r = 0; r < 16; r++) {
            const int x = 32 * t + 8 * (r / 4) + r % 4 + h4;
            s[t][r] = x >= lo && x <= hi ? s[t][r] : -INFINITY;
          }
      }
      float top = s[0][0];
#pragma unroll
      for (int t = 0; t < 2; t++)
#pragma unroll
        for (int r = 0; r < 16; r++) top = fmaxf(top, s[t][r]);
      top = half_max(top);
      // The reference m of the exponents follows the maximum only once that
      // is 2^8 above it: p stays below 2^8, and the sums are seldom rescaled.
      if (__any(top > m + far)) {
        const float to = fmaxf(m, top);
        const float by = to == -INFINITY ? 1.f : exp2_((m - to) * c);
        m = to;
        mc = m == -INFINITY ? 0.f : m * c;
        l *= by;
#pragma unroll
        for (int n = 0; n < DC / 32; n++) o[n] *= by;
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
      if (masked && careful) {
        careful_product<T, DP, DC>(s_v, o, p, lo, hi, lane);
      } else {
#pragma unroll
        for (int j = 0; j < 4; j++)
#pragma unroll
          for (int n = 0; n < DC / 32; n++) o[n] = Half<T>::mma(cols_at<DP>(s_v, n, j, lane), p[j], o[n]);
      }
    }
    // An infinity or NaN may come from a value that the row does not see.
    if (careful || !__syncthreads_or(real && not_finite(o, 1.f))) break;
  }
  l = half_sum(l);
  if (i < A.T) {
    if (!real) {
#pragma unroll
      for (int n = 0; n < DC / 32; n++) o[n] = acc16{};
    }
    store_rows<T>(A.out, head, i, o, real ? 1.f / l : 0.f, A.d, lane);
    if (lane < 32) A.lse[(int64_t)head * A.T + i] = real ? (mc + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
  }
}

// dq of a tile of 128 tokens of one query head; leaves lse_i and D_i in rows for k_attention_dkv.
template <class T, int DP, int DC>
__global__ void __launch_bounds__(kWaves * 64, 2) k_attention_dq(AttnArgs A) {
  constexpr int kTile = kStep * DP * 2;
  __shared__ __align__(16) char s_kv[2][2][kTile];
  __shared__ int s_range[2][kWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h4 = 4 * (lane >> 5);
  const int item = item_of(blockIdx.x, gridDim.x);
  const int head = item / A.tiles, tile = A.tiles - 1 - item % A.tiles, kvh = head / (A.H / A.K);
  const int i = tile * kBlock + wave * kRows + (lane & 31);
  int first, last;
  sequence_of(A, i, first, last);
  const bool real = last > first;
  const int w_first = wave_min(real ? first : INT32_MAX), w_last = wave_max(real ? i : -1);
  const int w_upto = wave_min(real ? i : INT32_MAX), w_from = wave_max(real ? first : -1);
  if (lane == 0) {
    s_range[0][wave] = w_first;
    s_range[1][wave] = w_last;
  }
  __syncthreads();
  int k0 = INT32_MAX, k1 = -1;
#pragma unroll
  for (int w = 0; w < kWaves; w++) {
    k0 = min(k0, s_range[0][w]);
    k1 = max(k1, s_range[1][w]);
  }
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
  const float lse2 = real ? A.lse[(int64_t)head * A.T + i] * kLog2e : INFINITY;
  if (i < A.T && lane < 32) {
    A.rows[(int64_t)head * A.T + i] = lse2;
    A.rows[((int64_t)A.H + head) * A.T + i] = D;
  }
  const float c = A.scale * kLog2e;
  const Stager<DP> ks(A.k, A.d, tid), vs(A.v, A.d, tid);
  const int64_t k_head = 2 * kvh * A.k.head, v_head = 2 * kvh * A.v.head;
  acc16 dq[DC / 32];
  for (int careful = 0;; careful = 1) {
#pragma unroll
    for (int n = 0; n < DC / 32; n++) dq[n] = acc16{};
    int now = 0;
    if (k0 <= k1) {
      ks.load(s_kv[0][0], k_head, k0, k1 + 1, wave);
      vs.load(s_kv[0][1], v_head, k0, k1 + 1, wave);
    }
    for (int a = k0; a <= k1; a += kStep, now ^= 1) {
      next_tile();
      if (a + kStep <= k1) {
        ks.load(s_kv[now ^ 1][0], k_head, a + kStep, k1 + 1, wave);
        vs.load(s_kv[now ^ 1][1], v_head, a + kStep, k1 + 1, wave);
      }
      if (a > w_last || a + kStep <= w_first) continue;
      const char *s_k = s_kv[now][0], *s_v = s_kv[now][1];
      const int lo = first - a, hi = i - a;
      const bool masked = a < w_from || a + kStep - 1 > w_upto;
      u32x4 ds[4];
#pragma unroll
      for (int t = 0; t < 2; t++) {
        acc16 s = {}, dp = {};
#pragma unroll
        for (int kk = 0; kk < DC / 16; kk++) {
          s = Half<T>::mma(rows_at<DP>(s_k, t, kk, lane), q[kk], s);
          dp = Half<T>::mma(rows_at<DP>(s_v, t, kk, lane), g[kk], dp);
        }
#pragma unroll
        for (int r = 0; r < 16; r++) s[r] = exp2_(fmaf(s[r], c, -lse2)) * (dp[r] - D);
        if (masked) {
#pragma unroll
          for (int r = 0; r < 16; r++) {
            const int x = 32 * t + 8 * (r / 4) + r % 4 + h4;
            s[r] = x >= lo && x <= hi ? s[r] : 0.f;
          }
        }
        ds[2 * t] = operand<T>(s, 0);
        ds[2 * t + 1] = operand<T>(s, 1);
      }
      if (masked && careful) {
        careful_product<T, DP, DC>(s_k, dq, ds, lo, hi, lane);
      } else {
#pragma unroll
        for (int j = 0; j < 4; j++)
#pragma unroll
          for (int n = 0; n < DC / 32; n++) dq[n] = Half<T>::mma(cols_at<DP>(s_k, n, j, lane), ds[j], dq[n]);
      }
    }
    if (careful || !__syncthreads_or(real && not_finite(dq, A.scale))) break;
  }
  if (i < A.T) {
    if (!real) {
#pragma unroll
      for (int n = 0; n < DC / 32; n++) dq[n] = acc16{};
    }
    store_rows<T>(A.dq, head, i, dq, A.scale, A.d, lane);
  }
}

// dk and dv of a tile of 128 tokens of one key/value head: each wave 32 of
// them, over the query heads that share it and the rows up to the end of the
// last token's sequence, in that order whatever the launch.
template <class T, int DP, int DC>
__global__ void __launch_bounds__(kWaves * 64, DP == 64 ? 2 : 1) k_attention_dkv(AttnArgs A) {
  constexpr int kTile = kStep * DP * 2;
  __shared__ __align__(16) char s_qg[2][2][kTile];
  __shared__ __align__(16) float s_row[2][2][kStep];  // of A.rows
  __shared__ int s_range[2][kWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h4 = 4 * (lane >> 5);
  const int item = item_of(blockIdx.x, gridDim.x);
  const int kvh = item / A.tiles, tile = item % A.tiles, group = A.H / A.K;
  const int j = tile * kBlock + wave * kRows + (lane & 31);  // this lane's key
  int first, last;
  sequence_of(A, j, first, last);
  const bool real = last > first;
  // rows that see a key of this wave, of this workgroup; rows that see all of the wave's
  const int w_first = wave_min(real ? j : INT32_MAX), w_last = wave_max(real ? last - 1 : -1);
  const int w_upto = wave_min(real ? last - 1 : INT32_MAX), w_from = wave_max(real ? j : -1);
  if (lane == 0) {
    s_range[0][wave] = w_first;
    s_range[1][wave] = w_last;
  }
  __syncthreads();
  int i0 = INT32_MAX, i1 = -1;
#pragma unroll
  for (int w = 0; w < kWaves; w++) {
    i0 = min(i0, s_range[0][w]);
    i1 = max(i1, s_range[1][w]);
  }
  u32x4 k[DC / 16], v[DC / 16];
  load_rows(k, A.k, kvh, j, A.T, A.d, lane);
  load_rows(v, A.v, kvh, j, A.T, A.d, lane);
  const float c = A.scale * kLog2e;
  const Stager<DP> qs(A.q, A.d, tid), gs(A.dout, A.d, tid);
  const int steps = i1 < i0 ? 0 : (i1 - i0) / kStep + 1, all = steps * group;
  // tile n of all: rows i0 + kStep (n % steps) on of the group's head n / steps
  auto load = [&](int n, int to) {
    const int head = kvh * group + n / steps, a = i0 + kStep * (n % steps);
    qs.load(s_qg[to][0], 2 * head * A.q.head, a, i1 + 1, wave);
    gs.load(s_qg[to][1], 2 * head * A.dout.head, a, i1 + 1, wave);
    if (wave < 2) {  // 64 rows' lse by wave 0, their D by wave 1
      const float *from = A.rows + ((int64_t)wave * A.H + head) * A.T + a;
      const int rows = min(i1 + 1 - a, kStep);
      const __amdgpu_buffer_rsrc_t buf =
          __builtin_amdgcn_make_buffer_rsrc(const_cast<float *>(from), 0, 4 * rows, 0x00020000);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(buf, (__attribute__((address_space(3))) void *)s_row[to][wave], 4,
                                               4 * lane, 0, 0, 0);
    }
  };
  acc16 dk[DC / 32], dv[DC / 32];
  for (int careful = 0;; careful = 1) {
#pragma unroll
    for (int n = 0; n < DC / 32; n++) dk[n] = dv[n] = acc16{};
    if (all) load(0, 0);
    for (int n = 0; n < all; n++) {
      const int a = i0 + kStep * (n % steps), now = n & 1;
      next_tile();
      if (n + 1 < all) load(n + 1, now ^ 1);
      if (a > w_last || a + kStep <= w_first) continue;
      const char *s_q = s_qg[now][0], *s_g = s_qg[now][1];
      const float *s_lse = s_row[now][0], *s_delta = s_row[now][1];
      const int lo = j - a, hi = last - 1 - a;  // of the 64 rows, those that see this key
      const bool masked = a < w_from || a + kStep - 1 > w_upto;
      u32x4 p[4], ds[4];
#pragma unroll
      for (int t = 0; t < 2; t++) {
        acc16 s = {}, dp = {};
#pragma unroll
        for (int kk = 0; kk < DC / 16; kk++) {
          s = Half<T>::mma(rows_at<DP>(s_q, t, kk, lane), k[kk], s);
          dp = Half<T>::mma(rows_at<DP>(s_g, t, kk, lane), v[kk], dp);
        }
#pragma unroll
        for (int r = 0; r < 16; r++) {
          const int x = 32 * t + 8 * (r / 4) + r % 4 + h4;
          s[r] = exp2_(fmaf(s[r], c, -s_lse[x]));
          dp[r] = s[r] * (dp[r] - s_delta[x]);
          if (masked) {
            const bool seen = x >= lo && x <= hi;
            s[r] = seen ? s[r] : 0.f;
            dp[r] = seen ? dp[r] : 0.f;
          }
        }
        p[2 * t] = operand<T>(s, 0);
        p[2 * t + 1] = operand<T>(s, 1);
        ds[2 * t] = operand<T>(dp, 0);
        ds[2 * t + 1] = operand<T>(dp, 1);
      }
      if (masked && careful) {
        careful_product<T, DP, DC>(s_g, dv, p, lo, hi, lane);
        careful_product<T, DP, DC>(s_q, dk, ds, lo, hi, lane);
      } else {
#pragma unroll
        for (int jj = 0; jj < 4; jj++)
#pragma unroll
          for (int n = 0; n < DC / 32; n++) {
            dv[n] = Half<T>::mma(cols_at<DP>(s_g, n, jj, lane), p[jj], dv[n]);
            dk[n] = Half<T>::mma(cols_at<DP>(s_q, n, jj, lane), ds[jj], dk[n]);
          }
      }
    }
    if (careful || !__syncthreads_or(real && (not_finite(dk, A.scale) || not_finite(dv, 1.f)))) break;
  }
  if (j < A.T) {
    if (!real) {
#pragma unroll
      for (int n = 0; n < DC / 32; n++) dk[n] = dv[n] = acc16{};
    }
    store_rows<T>(A.dk, kvh, j, dk, A.scale, A.d, lane);
    store_rows<T>(A.dv, kvh, j, dv, 1.f, A.d, lane);
  }
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
  CEL_BY_TYPE(k_attention_dkv, A.tiles * A.K);
  return CEL_OK;
}
