// The end of a block and the beginning of the next, and their gradient:
//   n = norm(f) post + post_bias, or f;  y = scale x + gate drop(n)
//   z = norm(y) pre + pre_bias;  norm(v) = v / sqrt(mean v^2 + eps), of v less its mean if centered
// Backwards from dy, dz, f and y, with Y = norm(y), N = norm(f) and r their factors:
//   g = pre dz;  t = dy + r_y (g - [mean g] - Y mean(g Y));  dx = scale t
//   e = drop'(gate t), the mask's factors applied once more;  dgate = sum t drop(n)
//   df = r_f (post e - [mean post e] - N mean(post e N)), or e
//   dpre = sum dz Y;  dpre_bias = sum dz;  dpost = sum e N;  dpost_bias = sum e
// A row is read once and its statistics are made where it lies, in registers, so
// that nothing but y and z is kept for the backward pass and nothing is read twice.
//
// A team of W waves takes a row, eight columns a lane (beyond 8,192 columns kMost
// times as many); the teams of a workgroup take the rows of its range in turn.  Gradients
// of vectors are sums over rows: a lane adds its columns' over its team's rows, the teams
// join theirs in LDS, and k_norm_sums adds the workgroups', all in a fixed order.
// Where every sequence has a gate of its own, a workgroup walks its range in
// segments of one sequence, and leaves a sum for each.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <type_traits>

#include "elements.h"

namespace cel {
namespace {

constexpr int kMost = 2;        // eights of a row a lane holds
constexpr int kWidest = 16;     // waves of a row, and of a workgroup
constexpr int kForward = 4, kBackward = 16;  // waves of a workgroup, unless a row takes more
constexpr int kGroups = 256;    // workgroups that leave sums, at most; four times that forward

// Which vectors there are, as far as registers are held for them.
constexpr int kBias = 1, kBranch = 2;  // biases; a norm of f or a gate

__host__ __device__ constexpr int vectors_of(int kind) { return kind & kBranch ? kind & kBias ? 4 : 3 : 1; }

struct NormArgs {
  const char *f, *x, *dy, *dz;  // x: the stream read (x, or y backwards)
  char *y, *z;                  // written: y and z, or dx and df
  int64_t f_row, x_row, dy_row, dz_row, y_row, z_row;  // strides in elements
  const void *pre, *pre_bias, *post, *post_bias, *gate;
  bool wide;                    // parameters of 32 bits
  bool center;
  bool has_dy;
  const int32_t *ptr;           // NULL: one gate for all rows
  int32_t S;
  int64_t T, per;               // rows; rows of a workgroup
  int32_t h, W, teams;
  Divisor waves;                // of a row
  float eps, scale;
  Mask mask;
  float *part;                  // sums that workgroups leave: [vector][slot][h]
  int64_t slots;
};

// The kernel's arguments as they lie in memory, read anew: a loop that holds all of them has no scalar
// registers left, and spills some into vector registers' lanes.
__device__ inline NormArgs again() {
  typedef const __attribute__((address_space(4))) uint32_t *args_ptr;
  static_assert(sizeof(NormArgs) % 4 == 0, "whole words");
  args_ptr p = (args_ptr)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  uint32_t w[sizeof(NormArgs) / 4];
#pragma unroll
  for (int i = 0; i < (int)(sizeof(NormArgs) / 4); i++) w[i] = p[i];
  NormArgs A;
  __builtin_memcpy(&A, w, sizeof A);
  return A;
}

// Where a lane stands in its row: its first column and how many of the eight lack at the row's end (8 and more: all).
struct Column {
  int at, lack;
  bool tail;  // of any lane of the wave
  // lack, for comparisons that are made where they are used: the few waves with a tail make them anew for
  // every row, and the others' scalar registers are not full of their results.
  __device__ int lack_here() const {
    int x = lack;
    asm volatile("" : "+v"(x));
    return x;
  }
};
template <class T, bool NARROW>  // rows of less than eight columns
__device__ inline Eight<T> load_piece(const T *row, Column c, int h) {
  if constexpr (NARROW) return load_eight(row, h - c.at);
  else return load_back(row, c.at, h);
}
template <class T, bool NARROW>
__device__ inline void piece_values(float (&f)[8], const Eight<T> &r, Column c, int h) {
  values<T>(f, r);
  if (!NARROW && c.tail) shift_down(f, c.lack_here());
}

// The sequence that holds row t and the first row behind t that need not be in it; -1: none.
// Whatever ptr holds, end > t.
__device__ inline int sequence_at(const NormArgs &A, int64_t t, int hint, int64_t &end) {
  const int32_t *ptr = A.ptr;
  int lo = 0;
  if (hint >= 0 && hint < A.S && ptr[hint] <= t && ptr[hint + 1] > t) {
    lo = hint;
  } else {
    int hi = A.S;  // the last s with ptr[s] <= t, if any
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (ptr[mid] <= t) lo = mid;
      else hi = mid - 1;
    }
  }
  int s = -1;
  if (ptr[lo] > t) end = ptr[lo];
  else if (lo >= A.S) end = A.T;
  else end = ptr[lo + 1], s = end > t ? lo : -1;
  end = min(max(end, t + 1), A.T);
  return s;
}

// Sums over a row's columns, in all of its lanes: over the lanes, and through
// LDS over the team's waves.  Two buffers in turn make one barrier enough.
constexpr int kSums = 8;
struct RowSum {
  float (*red)[kSums][kWidest];
  int wave, team, W, turn;
  template <int N>
  __device__ void operator()(float (&x)[N]) {
    LaneSums<N> s(x);
    if (W > 1) {
      float (*to)[kWidest] = red[turn];
      turn ^= 1;
      const int lane = threadIdx.x & 63, row = lane >> 4, i = lane & 15;
      if (i == 0) {
#pragma unroll
        for (int j = 0; j < LaneSums<N>::kRegisters; j++) to[4 * j + row][wave] = s.r[j];
      }
      lds_barrier();
#pragma unroll
      for (int j = 0; j < LaneSums<N>::kRegisters; j++) {
        const float y = to[4 * j + row][team * W + min(i, W - 1)];
        s.r[j] = sixteen_sum(i < W ? y : 0.f);
      }
    }
    s.get(x);
  }
};

// A row as it comes from memory, and as numbers.
template <class T, int C, bool NARROW>
struct Raw {
  Eight<T> e[C];
  __device__ void load(const char *p, int64_t at, const Column (&c)[C], int h) {
#pragma unroll
    for (int u = 0; u < C; u++) e[u] = load_piece<T, NARROW>(reinterpret_cast<const T *>(p) + at, c[u], h);
  }
};
template <int C>
struct Row {
  float v[C][8];
  template <class T, bool NARROW>
  __device__ void from(const Raw<T, C, NARROW> &r, const Column (&c)[C], int h) {
#pragma unroll
    for (int u = 0; u < C; u++) piece_values<T, NARROW>(v[u], r.e[u], c[u], h);
  }
  __device__ void fill(float x) {
#pragma unroll
    for (int u = 0; u < C; u++)
#pragma unroll
      for (int e = 0; e < 8; e++) v[u][e] = x;
  }
  __device__ void cut(const Column (&c)[C]) {  // 0 past the row's end
#pragma unroll
    for (int u = 0; u < C; u++)
      if (c[u].tail) {
        const int left = 8 - c[u].lack_here();
#pragma unroll
        for (int e = 0; e < 8; e++) v[u][e] = e < left ? v[u][e] : 0.f;
      }
  }
  template <class T>
  __device__ void store(char *p, int64_t at, const Column (&c)[C]) const {
#pragma unroll
    for (int u = 0; u < C; u++) {
      T *to = reinterpret_cast<T *>(p) + at + c[u].at;
      if (!c[u].tail) {
        store_eight(to, v[u], 8);
      } else {
        const int left = 8 - c[u].lack_here();
        if (left > 0) store_eight(to, v[u], left);
      }
    }
  }
};
// N vectors of parameters, all loads before the first use; `none` where there is no such vector.
template <class T, bool NARROW, int C, int N>
__device__ inline void parameters(Row<C> *const (&to)[N], const void *const (&from)[N], const float (&none)[N], const Column (&c)[C], int h) {
  Raw<T, C, NARROW> r[N];
#pragma unroll
  for (int n = 0; n < N; n++)
    if (from[n]) r[n].load(static_cast<const char *>(from[n]), 0, c, h);
#pragma unroll
  for (int n = 0; n < N; n++) {
    if (from[n]) to[n]->from(r[n], c, h);
    else to[n]->fill(none[n]);
  }
}
#define EACH(u, e) \
  _Pragma("unroll") for (int u = 0; u < C; u++) _Pragma("unroll") for (int e = 0; e < 8; e++)

// v less its mean if centered, and the factor that makes it a norm.  Columns past the row's end stay 0.
template <int C>
__device__ inline float normalise(Row<C> &v, const NormArgs &A, const Column (&c)[C], RowSum &sum) {
  if (A.center) {
    float m[1] = {0.f};
    EACH(u, e) m[0] += v.v[u][e];
    sum(m);
    m[0] /= A.h;
    EACH(u, e) v.v[u][e] -= m[0];
    v.cut(c);
  }
  float q[1] = {0.f};
  EACH(u, e) q[0] = fmaf(v.v[u][e], v.v[u][e], q[0]);
  sum(q);
  return rsqrtf(q[0] / A.h + A.eps);
}

template <int C>
__device__ inline void columns_of(Column (&c)[C], const NormArgs &A, int team) {
  const int lane = threadIdx.x - team * 64 * A.W;
#pragma unroll
  for (int u = 0; u < C; u++) {
    c[u].at = 8 * (u * 64 * A.W + lane);
    c[u].lack = max(0, c[u].at + 8 - A.h);
    c[u].tail = __any(c[u].lack);
  }
}
// The gates of sequence s.
template <class T, bool NARROW, int C>
__device__ inline void gates_of(Row<C> &gate, const NormArgs &A, int s, const Column (&c)[C]) {
  Row<C> *const to[1] = {&gate};
  const float none[1] = {1.f};
  const void *const from[1] = {static_cast<const char *>(A.gate) + (int64_t)s * A.h * (A.wide ? 4 : sizeof(T))};
  if (A.wide) parameters<float, NARROW>(to, from, none, c, A.h);
  else parameters<T, NARROW>(to, from, none, c, A.h);
}

// T: of f and z; R: of the stream x and y.  The next row is on its way while one is dealt with.
// Bound by memory: 4,096 rows of 8,192, f in 16 bits and a stream in 32, 403 MB in 85 us (4.7 TB/s); all in
// 16 bits without gate and second norm 268 MB in 45 us, part of them from the caches.  4,096 rows of 1,024 take 11 us, of which
// start, the vectors' loads and a row's two or three sums are half.  What counts is that no load stands in a branch:
// with each row's end as a branch of its own, 9,973 rows of 2,049 columns took 89 us instead of 39.
// 16 columns a lane: 8 % faster without gate and second norm, 3 to 6 % slower with them.
template <class T, class R, int C, int KIND, bool NARROW>
__global__ void __launch_bounds__(64 * kWidest) k_residual_norm(NormArgs A) {
  __shared__ float s_red[2][kSums][kWidest];
  constexpr bool bias = (KIND & kBias) != 0, branch = (KIND & kBranch) != 0;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), team = A.waves.quotient(wave);
  RowSum sum{s_red, wave, team, A.W, 0};
  Column c[C];
  columns_of(c, A, team);
  const int64_t first = blockIdx.x * A.per, last = min(A.T, first + A.per);
  const int teams = A.teams;
  Raw<T, C, NARROW> f_next;
  Raw<R, C, NARROW> x_next;
  auto load = [&](const NormArgs &A, int64_t t) {  // rows that are not there: the last in their place
    t = min(t, last - 1);
    if (A.f) f_next.load(A.f, t * A.f_row, c, A.h);
    x_next.load(A.x, t * A.x_row, c, A.h);
  };
  load(A, first + team);
  Mask mask = A.mask;
  mask.begin();
  Row<C> pre, pre_bias, post, post_bias, gate;
  {
    Row<C> *const to[5] = {&pre, &gate, &post, &pre_bias, &post_bias};
    const void *const from[5] = {A.pre, branch && !A.ptr ? A.gate : nullptr, branch ? A.post : nullptr, bias ? A.pre_bias : nullptr,
                                 bias && branch ? A.post_bias : nullptr};
    const float none[5] = {0.f, 1.f, 0.f, 0.f, 0.f};
    if (A.wide) parameters<float, NARROW>(to, from, none, c, A.h);
    else parameters<T, NARROW>(to, from, none, c, A.h);
  }
  int s = -1;
  int64_t s_end = branch && A.ptr ? first : A.T;
  for (int64_t base = first; base < last; base += teams) {
    const NormArgs A = again();
    mask.k0 = A.mask.k0, mask.k1 = A.mask.k1, mask.least = A.mask.least, mask.by = A.mask.by;
    const int64_t t = base + team;
    const bool real = t < last;
    Row<C> f, x;
    if (A.f) f.from(f_next, c, A.h);
    x.from(x_next, c, A.h);
    load(A, t + teams);
    if (branch && A.ptr && real && t >= s_end) {
      s = sequence_at(A, t, s + 1, s_end);
      if (s >= 0) gates_of<T, NARROW>(gate, A, s, c);
    }
    if (A.f) {
      if (branch && A.post) {
        const float r = normalise(f, A, c, sum);
        EACH(u, e) f.v[u][e] = f.v[u][e] * r * post.v[u][e] + (bias ? post_bias.v[u][e] : 0.f);
      }
      if (mask.least) {
#pragma unroll
        for (int u = 0; u < C; u++) mask.apply(f.v[u], c[u].at >> 3, (uint32_t)t);
      }
      if (branch) EACH(u, e) f.v[u][e] *= gate.v[u][e];
      if (branch && A.ptr && s < 0) f.fill(0.f);
      EACH(u, e) x.v[u][e] = fmaf(x.v[u][e], A.scale, f.v[u][e]);
      if (real) x.template store<R>(A.y, t * A.y_row, c);
    }
    if (A.pre) {
      const float r = normalise(x, A, c, sum);
      EACH(u, e) x.v[u][e] = x.v[u][e] * r * pre.v[u][e] + (bias ? pre_bias.v[u][e] : 0.f);
      if (real) x.template store<T>(A.z, t * A.z_row, c);
    }
  }
}

// The vectors that the gradient's rows need, where rows have need of the registers: in 32 bits in
// LDS, each padded with zeros to whole eights and eight more, which lanes past the row's end read; or of
// rows beyond 8,192 columns, whose vectors LDS does not hold, read anew.
enum { kPre, kPost, kGate, kPostBias };
__host__ __device__ inline int padded_of(int h) { return ((h + 7) & ~7) + 8; }
template <class T>
struct Vectors {
  float *lds;
  const void *at[4];
  bool wide;
  int h, padded;
  __device__ void stage(int which) const {
    const void *p = at[which];
    for (int k = threadIdx.x; k < padded; k += blockDim.x)
      lds[which * padded + k] = k >= h ? 0.f : !p ? 1.f : wide ? static_cast<const float *>(p)[k] : (float)static_cast<const T *>(p)[k];
  }
  template <int C>
  __device__ void get(Row<C> &to, int which, const Column (&c)[C]) const {
    if constexpr (C == 1) {
      typedef __attribute__((ext_vector_type(4))) float f32x4;
      const f32x4 *p = reinterpret_cast<const f32x4 *>(lds + which * padded + min(c[0].at, padded - 8));
      const f32x4 a = p[0], b = p[1];
#pragma unroll
      for (int e = 0; e < 4; e++) to.v[0][e] = a[e], to.v[0][4 + e] = b[e];
    } else {
      Row<C> *const rows[1] = {&to};
      const void *const from[1] = {at[which]};
      const float none[1] = {1.f};
      if (wide) parameters<float, false>(rows, from, none, c, h);
      else parameters<T, false>(rows, from, none, c, h);
    }
  }
};

// The teams' sums of up to two vectors' gradients (`to` NULL: none) to the workgroup's slots.
template <int C>
__device__ inline void leave_sums(Row<C> &one, float *to_one, Row<C> &two, float *to_two, const NormArgs &A, const Column (&c)[C], int team,
                                  float *s_join) {
  if (A.teams > 1) {
    float *s_two = s_join + A.teams * A.h;
    __syncthreads();
    if (to_one) one.template store<float>(reinterpret_cast<char *>(s_join), (int64_t)team * A.h, c);
    if (to_two) two.template store<float>(reinterpret_cast<char *>(s_two), (int64_t)team * A.h, c);
    __syncthreads();
    for (int k = threadIdx.x; k < A.h; k += blockDim.x) {
      float x = 0.f, y = 0.f;
      for (int w = 0; w < A.teams; w++) {
        if (to_one) x += s_join[w * A.h + k];
        if (to_two) y += s_two[w * A.h + k];
      }
      if (to_one) to_one[k] = x;
      if (to_two) to_two[k] = y;
    }
  } else {
    if (to_one) one.template store<float>(reinterpret_cast<char *>(to_one), 0, c);
    if (to_two) two.template store<float>(reinterpret_cast<char *>(to_two), 0, c);
  }
}

// The vectors' order in the sums that workgroups leave: pre, pre_bias, post, post_bias, gate.
// A row's sums over its waves are barriers, which all 16 waves of a compute unit wait in: they are taken together
// as far as they do not need each other, means first where they come out, then squares and products with
// g, then those with post e.  The next row's loads stand behind the last use of this one's, dy, dz and y before the second
// half, so that both halves have some under way.
// Bound by memory and these waits: 4,096 rows of 8,192 in 16 bits with both norms, gates and dropout 403 MB and 50 of sums in
// 106 us (4.3 TB/s), 2 of them since f is multiplied by r, 2 since dropped products are chosen; without gate and second norm
// 335 MB in 69 us.  Tried beside 101: dy, dz and y loaded at a row's beginning 112; all of a row's sums at once (those with
// post e from the three parts of t), one barrier of two, 35 registers spilled, 133; 16 columns a lane, 8 waves, 127; 512 workgroups
// 141, twice the sums to leave.  At 513 to 1,024 columns 16 a lane saved 1 to 3 % (8,192 rows of 1,000: 36.6 -> 35.6, forward
// 16.3 -> 14.7) for a further instance of each kernel.  Beyond 8,192 columns a lane's 16 spill some 200 registers: 2,048 rows of
// 16,384, 403 MB, in 336 us.
template <class T, class R, int C, int KIND, bool NARROW>
__global__ void __launch_bounds__(64 * kWidest) k_residual_norm_grad(NormArgs A) {
  extern __shared__ __align__(16) float s_dynamic[];
  __shared__ float s_red[2][kSums][kWidest];
  __shared__ int s_sequence;
  __shared__ int64_t s_end;
  constexpr bool bias = (KIND & kBias) != 0, branch = (KIND & kBranch) != 0;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), team = A.waves.quotient(wave);
  RowSum sum{s_red, wave, team, A.W, 0};
  Column c[C];
  columns_of(c, A, team);
  const int padded = padded_of(A.h);
  Vectors<T> vectors{s_dynamic, {A.pre, A.post, A.ptr ? nullptr : A.gate, A.post_bias}, A.wide, A.h, padded};
  float *const s_join = s_dynamic + (C == 1 ? vectors_of(KIND) * padded : 0);
  const int64_t first = blockIdx.x * A.per, last = min(A.T, first + A.per);
  Raw<T, C, NARROW> f_next, dz_next;
  Raw<R, C, NARROW> y_next, dy_next;
  const int teams = A.teams;
  // Every load of a row, whether the call has need of it or not (then it is another's place): a branch
  // between them would make a wave wait for the ones before it.  Rows that are not there: the last in their place.
  auto load = [&](int64_t t) {
    t = min(t, last - 1);
    dz_next.load(A.dz, t * A.dz_row, c, A.h);
    y_next.load(A.x, t * A.x_row, c, A.h);
    dy_next.load(A.dy, t * A.dy_row, c, A.h);
    if (branch) f_next.load(A.f, t * A.f_row, c, A.h);
  };
  load(first + team);
  Mask mask = A.mask;
  mask.begin();
  Row<C> d_pre = {}, d_pre_bias = {}, d_post = {}, d_post_bias = {}, d_gate = {};
  if (C == 1) {
    if (A.pre) vectors.stage(kPre);
    if (branch) {
      if (A.post) vectors.stage(kPost);
      if (!A.ptr) vectors.stage(kGate);
      if (bias && A.post_bias) vectors.stage(kPostBias);
    }
    lds_barrier();
  }
  const float over = 1.f / A.h;
  int s = -1;
  for (int64_t from = first; from < last;) {
    int64_t to = last;
    if (branch && A.ptr) {
      lds_barrier();  // the segment before has read its gates
      if (threadIdx.x == 0) {  // one thread looks, so that all waves walk the same segments whatever happens to ptr
        int64_t end;
        s_sequence = sequence_at(A, from, s + 1, end);
        s_end = min(last, end);
      }
      lds_barrier();
      s = __builtin_amdgcn_readfirstlane(s_sequence);
      to = first + __builtin_amdgcn_readfirstlane((int)(s_end - first));
      if (s >= 0) {
        vectors.at[kGate] = static_cast<const char *>(A.gate) + (int64_t)s * A.h * (A.wide ? 4 : sizeof(T));
        if (C == 1) {
          vectors.stage(kGate);
          lds_barrier();
        }
      }
      if (from > first) load(from + team);
    }
    const bool open = !(branch && A.ptr) || s >= 0;
    for (int64_t base = from; base < to; base += teams) {
      const int64_t t = base + team;
      const bool real = t < to;
      Row<C> dy, y, f, g, dz;
      dz.from(dz_next, c, A.h);
      y.from(y_next, c, A.h);
      dy.from(dy_next, c, A.h);
      if (branch) f.from(f_next, c, A.h);
      const int64_t tn = min(t + teams, last - 1);
      if (branch) f_next.load(A.f, tn * A.f_row, c, A.h);
      if (!A.has_dy) dy.fill(0.f);
      float m[3] = {0.f, 0.f, 0.f}, q[3] = {0.f, 0.f, 0.f};
      if (A.pre) {
        vectors.get(g, kPre, c);
        EACH(u, e) g.v[u][e] *= dz.v[u][e];
      }
      if (A.center) {
        if (A.pre) EACH(u, e) m[0] += y.v[u][e], m[1] += g.v[u][e];
        if (branch && A.post) EACH(u, e) m[2] += f.v[u][e];
        sum(m);
        m[0] *= over, m[1] *= over, m[2] *= over;
        if (A.pre) {
          EACH(u, e) y.v[u][e] -= m[0];
          y.cut(c);
        }
        if (branch && A.post) {
          EACH(u, e) f.v[u][e] -= m[2];
          f.cut(c);
        }
      }
      if (A.pre) EACH(u, e) q[0] = fmaf(y.v[u][e], y.v[u][e], q[0]), q[1] = fmaf(g.v[u][e], y.v[u][e], q[1]);
      if (branch && A.post) EACH(u, e) q[2] = fmaf(f.v[u][e], f.v[u][e], q[2]);
      if (A.pre || (branch && A.post)) sum(q);
      if (A.pre) {
        const float r = rsqrtf(q[0] * over + A.eps), k = q[1] * over * r, b = m[1] * r;
        EACH(u, e) y.v[u][e] *= r;
        if (real) {  // a row that is not there may have no norm
          EACH(u, e) {
            d_pre.v[u][e] = fmaf(dz.v[u][e], y.v[u][e], d_pre.v[u][e]);
            if (bias) d_pre_bias.v[u][e] += dz.v[u][e];
          }
        }
        EACH(u, e) dy.v[u][e] = fmaf(fmaf(y.v[u][e], -k, g.v[u][e]), r, dy.v[u][e]);
        if (A.center) EACH(u, e) dy.v[u][e] -= b;
        dy.cut(c);  // k may be no number, and a sum over the row follows
      }
      if (A.scale == 1.f) {
        if (real) dy.template store<R>(A.y, t * A.y_row, c);
      } else {
        EACH(u, e) g.v[u][e] = dy.v[u][e] * A.scale;
        if (real) g.template store<R>(A.y, t * A.y_row, c);
      }
      dz_next.load(A.dz, tn * A.dz_row, c, A.h);
      y_next.load(A.x, tn * A.x_row, c, A.h);
      dy_next.load(A.dy, tn * A.dy_row, c, A.h);
      if (!A.z) continue;  // no branch at all
      if (!open) {  // a row of no sequence
        dy.fill(0.f);
        if (real) dy.template store<T>(A.z, t * A.z_row, c);
        continue;
      }
      // f becomes N: with r in dy instead, the products that lack one of the two would have to be divided by it, or
      // pass 32 bits where r is 0 for a row whose squares did.
      const float r = branch && A.post ? rsqrtf(q[2] * over + A.eps) : 1.f;
      // What the mask keeps, a bit each, since n and t times the gate are 0 where it drops, whatever they are; as conditions
      // held so long they would fill the scalar registers.
      uint32_t kept[C];
      if (mask.least) {
#pragma unroll
        for (int u = 0; u < C; u++) {
          bool k[8];
          // the ten rounds' keys are made anew for every row, beside the vector unit: twenty scalar registers less
          asm volatile("" : "+s"(mask.k0), "+s"(mask.k1));
          mask.kept(k, c[u].at >> 3, (uint32_t)t);
          if (branch) kept[u] = Mask::bits(k);
#pragma unroll
          for (int e = 0; e < 8; e++) dy.v[u][e] = branch || k[e] ? dy.v[u][e] * mask.by : 0.f;
        }
      }
      if (branch && A.post) EACH(u, e) f.v[u][e] *= r;
      if (branch && A.gate) {
        if (A.post) {
          vectors.get(g, kPost, c);
          EACH(u, e) g.v[u][e] *= f.v[u][e];
          if (bias && A.post_bias) {
            Row<C> b;
            vectors.get(b, kPostBias, c);
            EACH(u, e) g.v[u][e] += b.v[u][e];
          }
        } else {
          g = f;
        }
        if (mask.least) EACH(u, e) g.v[u][e] = Mask::where(kept[u], e, g.v[u][e]);
        if (real) EACH(u, e) d_gate.v[u][e] = fmaf(dy.v[u][e], g.v[u][e], d_gate.v[u][e]);
        vectors.get(g, kGate, c);
        EACH(u, e) dy.v[u][e] *= g.v[u][e];
      }
      if (branch && mask.least) EACH(u, e) dy.v[u][e] = Mask::where(kept[u], e, dy.v[u][e]);
      if (branch && A.post) {
        if (real) {
          EACH(u, e) d_post.v[u][e] = fmaf(dy.v[u][e], f.v[u][e], d_post.v[u][e]);
          if (bias && A.post_bias) EACH(u, e) d_post_bias.v[u][e] += dy.v[u][e];
        }
        vectors.get(g, kPost, c);
        float p[1] = {0.f};
        EACH(u, e) {
          dy.v[u][e] *= g.v[u][e];
          p[0] = fmaf(dy.v[u][e], f.v[u][e], p[0]);
        }
        if (A.center) {
          float both[2] = {p[0], 0.f};
          EACH(u, e) both[1] += dy.v[u][e];
          sum(both);
          p[0] = both[0], both[1] *= over;
          EACH(u, e) dy.v[u][e] -= both[1];
        } else {
          sum(p);
        }
        p[0] *= over;
        EACH(u, e) dy.v[u][e] = fmaf(f.v[u][e], -p[0], dy.v[u][e]) * r;
      }
      if (real) dy.template store<T>(A.z, t * A.z_row, c);
    }
    if (branch && A.gate && open) {
      float *slot = A.part + (4 * A.slots + blockIdx.x + (A.ptr ? s : 0)) * A.h;
      if (to - from > 1) leave_sums(d_gate, slot, d_gate, nullptr, A, c, team, s_join);
      else if (team == 0) d_gate.template store<float>(reinterpret_cast<char *>(slot), 0, c);  // one row, of the first team
      d_gate.fill(0.f);
    }
    from = to;
  }
  float *part = A.part + (int64_t)blockIdx.x * A.h;
  const int64_t apart = A.slots * A.h;
  if (A.pre) leave_sums(d_pre, part, d_pre_bias, bias && A.pre_bias ? part + apart : nullptr, A, c, team, s_join);
  if (branch && A.post)
    leave_sums(d_post, part + 2 * apart, d_post_bias, bias && A.post_bias ? part + 3 * apart : nullptr, A, c, team, s_join);
}

struct SumArgs {
  const float *part;
  float *to[5];
  int64_t slots, T, per;
  const int32_t *ptr;
  int32_t h, S, groups;
};
// Bound by latency: 256 workgroups' sums of three vectors of 8,192, 25 MB, in 7.6 us, of two of 1,024 in 3.8.
// Vector blockIdx.y as the sum of the workgroups' slots, in their order; from
// blockIdx.y = 4 on sequence blockIdx.y - 4's gate.  64 columns a workgroup, its waves share the slots.
constexpr int kSumWaves = 16;
__global__ void __launch_bounds__(64 * kSumWaves) k_norm_sums(SumArgs A) {
  __shared__ float s_sum[kSumWaves][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, which = min((int)blockIdx.y, 4);
  float *to = A.to[which];
  if (!to) return;
  const int s = blockIdx.y - which;
  const int64_t column = blockIdx.x * 64 + lane;
  int64_t a = 0, b = A.groups;  // slots
  if (which == 4 && A.ptr) {
    const int64_t first = max(A.ptr[s], 0), end = min((int64_t)A.ptr[s + 1], A.T);
    a = first / A.per, b = end > first ? (end - 1) / A.per + 1 : a;
    a += s, b += s;
  }
  float x = 0.f;
  const int64_t each = (b - a + kSumWaves - 1) / kSumWaves;
  if (column < A.h) {
    const float *p = A.part + which * A.slots * A.h + column;
    int64_t k = a + wave * each;
    const int64_t end = min(b, k + each);
    for (; k + 8 <= end; k += 8) {  // eight on their way at once
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; i++) y[i] = p[(k + i) * A.h];
#pragma unroll
      for (int i = 0; i < 8; i++) x += y[i];
    }
    for (; k < end; k++) x += p[k * A.h];
  }
  s_sum[wave][lane] = x;
  __syncthreads();
  if (wave || column >= A.h) return;
  x = 0.f;
  for (int w = 0; w < kSumWaves; w++) x += s_sum[w][lane];
  to[(int64_t)s * A.h + column] = x;
}

// ------------------------------------------------------------- entry points
struct Shape {
  int C, W, teams;
  int64_t per, groups;
};
Shape shape_of(const cel_norm_args *a, int waves, int64_t most) {
  Shape s;
  const int eights = (int)((a->hidden + 7) / 8);
  s.C = eights > 64 * kWidest ? kMost : 1;
  s.W = (eights + 64 * s.C - 1) / (64 * s.C);
  s.teams = std::max(1, waves / s.W);
  // With sequences shorter than the teams are many, a workgroup's would stand idle while it walks them one by one.
  const int64_t each = a->seq_ptr ? std::min<int64_t>(s.teams, a->rows / std::max(a->n_seq, 1) + 1) : s.teams;
  const int64_t groups = std::max<int64_t>(1, std::min(most, (a->rows + each - 1) / each));
  s.per = std::max<int64_t>(1, (a->rows + groups - 1) / groups);
  s.groups = (a->rows + s.per - 1) / s.per;
  return s;
}
int check_norm(const cel_norm_args *a, const char *fn) {
  if (!a) return set_error(CEL_E_ARG, "%s: NULL descriptor", fn);
  if (a->type < CEL_BF16 || a->type > CEL_F32 || (a->stream_type != a->type && a->stream_type != CEL_F32) ||
      (a->param_type != a->type && a->param_type != CEL_F32))
    return set_error(CEL_E_ARG, "%s: types %d, %d and %d", fn, a->type, a->stream_type, a->param_type);
  if (a->rows < 0 || a->rows > INT32_MAX || a->hidden < 1 || a->hidden > 8 * 64 * kMost * kWidest)
    return set_error(CEL_E_ARG, "%s: %lld rows of %lld", fn, (long long)a->rows, (long long)a->hidden);
  if (!(a->eps >= 0.f) || !std::isfinite(a->eps)) return set_error(CEL_E_ARG, "%s: eps %g", fn, (double)a->eps);
  if (!std::isfinite(a->scale)) return set_error(CEL_E_ARG, "%s: scale %g", fn, (double)a->scale);
  if (a->seq_ptr && (a->n_seq < 0 || a->n_seq > 65535 - 5 || !a->gate))
    return set_error(CEL_E_ARG, "%s: %d sequences, and %s gate", fn, a->n_seq, a->gate ? "a" : "no");
  if ((a->pre_bias && !a->pre) || (a->post_bias && !a->post)) return set_error(CEL_E_ARG, "%s: a bias without its norm", fn);
  return check_mask(&a->mask, fn);
}
int check_matrix(const cel_matrix *x, const cel_norm_args *a, int type, const char *fn, const char *what) {
  if (!x || !x->p) return set_error(CEL_E_ARG, "%s: %s is NULL", fn, what);
  if (reinterpret_cast<uintptr_t>(x->p) % (type == CEL_F32 ? 4 : 2))
    return set_error(CEL_E_ARG, "%s: %s is not aligned to its elements", fn, what);
  if (x->stride < a->hidden || x->stride > (int64_t(1) << 40))
    return set_error(CEL_E_ARG, "%s: %s has rows of %lld values %lld apart", fn, what, (long long)a->hidden, (long long)x->stride);
  return CEL_OK;
}
NormArgs args_of(const cel_norm_args *a, const Shape &s) {
  NormArgs A;
  memset(static_cast<void *>(&A), 0, sizeof A);
  A.waves = Divisor(s.W);
  A.pre = a->pre, A.pre_bias = a->pre_bias, A.post = a->post, A.post_bias = a->post_bias, A.gate = a->gate;
  A.wide = a->param_type == CEL_F32;
  A.center = a->center != 0;
  A.ptr = a->seq_ptr, A.S = a->n_seq;
  A.T = a->rows, A.per = s.per, A.h = (int)a->hidden, A.W = s.W, A.teams = s.teams;
  A.eps = a->eps, A.scale = a->scale;
  A.mask = mask_of(&a->mask);
  return A;
}
int64_t slots_of(const cel_norm_args *a) { return kGroups + (a->seq_ptr ? a->n_seq : 0); }

// go(type, stream type, eights of a lane, kind, whether rows are narrower than eight)
template <class F>
void by_type(const cel_norm_args *a, const Shape &s, F go) {
  const int kind = (a->pre_bias || a->post_bias ? kBias : 0) | (a->post || a->gate ? kBranch : 0);
  auto with = [&](auto t, auto r) {
    auto more = [&](auto c, auto narrow) {
      if (kind == 0) go(t, r, c, std::integral_constant<int, 0>{}, narrow);
      else if (kind == 1) go(t, r, c, std::integral_constant<int, 1>{}, narrow);
      else if (kind == 2) go(t, r, c, std::integral_constant<int, 2>{}, narrow);
      else go(t, r, c, std::integral_constant<int, 3>{}, narrow);
    };
    constexpr std::integral_constant<int, 1> one{};
    if (a->hidden < 8) more(one, std::true_type{});
    else if (s.C == 1) more(one, std::false_type{});
    else more(std::integral_constant<int, kMost>{}, std::false_type{});
  };
  const bool wide = a->stream_type == CEL_F32;
  if (a->type == CEL_F32) with(float{}, float{});
  else if (a->type == CEL_BF16) wide ? with(__bf16{}, float{}) : with(__bf16{}, __bf16{});
  else wide ? with(_Float16{}, float{}) : with(_Float16{}, _Float16{});
}

}  // namespace
}  // namespace cel

using namespace cel;

extern "C" int cel_residual_norm(const cel_norm_args *a, const cel_matrix *f, const cel_matrix *x, const cel_matrix *y,
                                 const cel_matrix *z, hipStream_t st) {
  const char *fn = "cel_residual_norm";
  CEL_TRY(check_norm(a, fn));
  if (!f && (a->post || a->gate || a->mask.p != 0.0 || a->scale != 1.f || !a->pre))
    return set_error(CEL_E_ARG, "%s: without f there is a norm of x alone", fn);
  if (a->rows == 0) return CEL_OK;
  if (f) CEL_TRY(check_matrix(f, a, a->type, fn, "f"));
  CEL_TRY(check_matrix(x, a, a->stream_type, fn, "x"));
  if (f) CEL_TRY(check_matrix(y, a, a->stream_type, fn, "y"));
  if (a->pre) CEL_TRY(check_matrix(z, a, a->type, fn, "z"));
  const Shape s = shape_of(a, kForward, 4 * kGroups);
  NormArgs A = args_of(a, s);
  if (f) A.f = (const char *)f->p, A.f_row = f->stride, A.y = (char *)y->p, A.y_row = y->stride;
  A.x = (const char *)x->p, A.x_row = x->stride;
  if (a->pre) A.z = (char *)z->p, A.z_row = z->stride;
  KTimer kt(st, "k_residual_norm");
  by_type(a, s, [&](auto t, auto r, auto c, auto kind, auto narrow) {
    k_residual_norm<decltype(t), decltype(r), decltype(c)::value, decltype(kind)::value, decltype(narrow)::value>
        <<<(unsigned)s.groups, 64 * s.W * s.teams, 0, st>>>(A);
  });
  CEL_HIP(hipGetLastError());
  return CEL_OK;
}

extern "C" int64_t cel_residual_norm_grad_scratch(const cel_norm_args *a) {
  CEL_TRY(check_norm(a, "cel_residual_norm_grad_scratch"));
  return 5 * 4 * slots_of(a) * a->hidden;
}

extern "C" int cel_residual_norm_grad(const cel_norm_args *a, const cel_matrix *dy, const cel_matrix *dz, const cel_matrix *f,
                                      const cel_matrix *y, void *scratch, const cel_matrix *dx, const cel_matrix *df,
                                      const cel_norm_grads *g, hipStream_t st) {
  const char *fn = "cel_residual_norm_grad";
  CEL_TRY(check_norm(a, fn));
  if (!df && (a->post || a->gate || a->mask.p != 0.0 || a->scale != 1.f || !a->pre))
    return set_error(CEL_E_ARG, "%s: without df there is the gradient of a norm of x alone", fn);
  if (!g || (a->pre && !g->pre) || (a->pre_bias && !g->pre_bias) || (a->post && !g->post) || (a->post_bias && !g->post_bias) ||
      (a->gate && !g->gate))
    return set_error(CEL_E_ARG, "%s: a parameter without a place for its gradient", fn);
  if (!scratch) return set_error(CEL_E_ARG, "%s: scratch is NULL", fn);
  if (!dy && !a->pre) return set_error(CEL_E_ARG, "%s: neither dy nor a norm before the next block", fn);
  const Shape s = shape_of(a, kBackward, kGroups);
  NormArgs A = args_of(a, s);
  A.part = static_cast<float *>(scratch);
  A.slots = slots_of(a);
  if (a->rows) {
    if (dy) CEL_TRY(check_matrix(dy, a, a->stream_type, fn, "dy"));
    if (a->pre) {
      CEL_TRY(check_matrix(dz, a, a->type, fn, "dz"));
      CEL_TRY(check_matrix(y, a, a->stream_type, fn, "y"));
    }
    if (a->post || a->gate) CEL_TRY(check_matrix(f, a, a->type, fn, "f"));
    CEL_TRY(check_matrix(dx, a, a->stream_type, fn, "dx"));
    if (df) CEL_TRY(check_matrix(df, a, a->type, fn, "df"));
    // what a call lacks is read where another array lies, and not looked at
    A.has_dy = dy != nullptr;
    const cel_matrix *some = dy ? dy : y;
    A.dy = (const char *)some->p, A.dy_row = some->stride;
    A.x = A.dz = A.dy, A.x_row = A.dy_row, A.dz_row = A.dy_row * (a->stream_type == a->type ? 1 : 2);
    if (a->pre) A.dz = (const char *)dz->p, A.dz_row = dz->stride, A.x = (const char *)y->p, A.x_row = y->stride;
    if (a->post || a->gate) A.f = (const char *)f->p, A.f_row = f->stride;
    A.y = (char *)dx->p, A.y_row = dx->stride;
    if (df) A.z = (char *)df->p, A.z_row = df->stride;
    KTimer kt(st, "k_residual_norm_grad");
    int rc = CEL_OK;
    by_type(a, s, [&](auto t, auto r, auto c, auto kind, auto narrow) {
      const auto kernel = k_residual_norm_grad<decltype(t), decltype(r), decltype(c)::value, decltype(kind)::value, decltype(narrow)::value>;
      const int lds = 4 * ((s.C == 1 ? vectors_of(kind) * padded_of(A.h) : 0) + (s.teams > 1 ? (kind & kBias ? 2 : 1) * s.teams * A.h : 0));
      rc = [&]() -> int {
        if (lds > 65536) CEL_HIP(hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds));
        kernel<<<(unsigned)s.groups, 64 * s.W * s.teams, lds, st>>>(A);
        CEL_HIP(hipGetLastError());
        return CEL_OK;
      }();
    });
    CEL_TRY(rc);
  }
  if (!a->pre && !a->post && !a->gate) return CEL_OK;
  SumArgs S{A.part,
            {a->pre ? g->pre : nullptr, a->pre_bias ? g->pre_bias : nullptr, a->post ? g->post : nullptr,
             a->post_bias ? g->post_bias : nullptr, a->gate ? g->gate : nullptr},
            A.slots, a->rows, s.per, a->seq_ptr, A.h, a->n_seq, (int)s.groups};
  const int gates = !a->gate ? 0 : a->seq_ptr ? a->n_seq : 1;
  KTimer kt(st, "k_norm_sums");
  k_norm_sums<<<dim3((unsigned)((A.h + 63) / 64), 4 + gates), 64 * kSumWaves, 0, st>>>(S);
  CEL_HIP(hipGetLastError());
  return CEL_OK;
}
