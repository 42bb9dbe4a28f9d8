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
// A team of W waves takes a row, 8 columns of each lane at a time, up to kMost
// times; the teams of a workgroup take the rows of its range in turn.  Gradients
// of vectors are sums over rows: a lane adds its columns' over its team's rows, the teams
// join theirs in LDS, and k_norm_sums adds the workgroups', all in a fixed order.
// Where every sequence has a gate of its own, a workgroup walks its range in
// segments of one sequence, and leaves a sum for each.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "elements.h"

namespace cel {
namespace {

constexpr int kMost = 2;        // eights of a row a lane holds
constexpr int kWaves = 8;       // waves of a workgroup, unless a row takes more
constexpr int kWidest = 16;     // waves of a row
constexpr int kGroups = 256;    // workgroups that leave sums, at most

// Which vectors there are, as far as registers are held for them.
constexpr int kBias = 1, kBranch = 2;  // biases; a norm of f or a gate

struct NormArgs {
  const char *f, *x, *dy, *dz;  // x: the stream read (x, or y backwards)
  char *y, *z;                  // written: y and z, or dx and df
  int64_t f_row, x_row, dy_row, dz_row, y_row, z_row;  // strides in elements
  const void *pre, *pre_bias, *post, *post_bias, *gate;
  bool wide;                    // parameters of 32 bits
  bool center;
  const int32_t *ptr;           // NULL: one gate for all rows
  int32_t S;
  int64_t T, per;               // rows; rows of a workgroup
  int32_t h, W, teams;
  float eps, scale;
  Mask mask;
  float *part;                  // sums that workgroups leave: [vector][slot][h]
  int64_t slots;
};

struct Column {  // where a lane stands in its row
  int at, left;
};

// Eight values of a vector of parameters; `none` where there is no such vector.
template <class T>
__device__ inline void parameters(float (&f)[8], const void *p, bool wide, Column c, float none) {
  if (!p || c.left <= 0) {
#pragma unroll
    for (int e = 0; e < 8; e++) f[e] = none;
  } else if (wide) {
    values<float>(f, load_eight(static_cast<const float *>(p) + c.at, c.left));
  } else {
    values<T>(f, load_eight(static_cast<const T *>(p) + c.at, c.left));
  }
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
struct RowSum {
  float (*red)[kWidest][4];
  int wave, W, turn;
  template <int N>
  __device__ void operator()(float (&x)[N]) {
#pragma unroll
    for (int n = 0; n < N; n++) x[n] = wave_sum(x[n]);
    if (W == 1) return;
    float (*r)[4] = red[turn];
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int n = 0; n < N; n++) r[wave][n] = x[n];
    }
    lds_barrier();
    const int first = wave / W * W;
#pragma unroll
    for (int n = 0; n < N; n++) x[n] = 0.f;
    for (int w = 0; w < W; w++)
#pragma unroll
      for (int n = 0; n < N; n++) x[n] += r[first + w][n];
  }
};

template <int C>
struct Row {
  float v[C][8];
  template <class T>
  __device__ void load(const char *p, int64_t at, const Column (&c)[C], bool real) {
#pragma unroll
    for (int u = 0; u < C; u++) {
      if (real && c[u].left > 0) {
        values<T>(v[u], load_eight(reinterpret_cast<const T *>(p) + at + c[u].at, c[u].left));
      } else {
#pragma unroll
        for (int e = 0; e < 8; e++) v[u][e] = 0.f;
      }
    }
  }
  template <class T>
  __device__ void store(char *p, int64_t at, const Column (&c)[C]) const {
#pragma unroll
    for (int u = 0; u < C; u++)
      if (c[u].left > 0) store_eight(reinterpret_cast<T *>(p) + at + c[u].at, v[u], c[u].left);
  }
};
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
    EACH(u, e) v.v[u][e] = e < c[u].left ? v.v[u][e] - m[0] : 0.f;
  }
  float q[1] = {0.f};
  EACH(u, e) q[0] = fmaf(v.v[u][e], v.v[u][e], q[0]);
  sum(q);
  return 1.f / sqrtf(q[0] / A.h + A.eps);
}

template <int C>
__device__ inline void columns_of(Column (&c)[C], const NormArgs &A) {
  const int lane = threadIdx.x % (64 * A.W);
#pragma unroll
  for (int u = 0; u < C; u++) c[u].at = 8 * (u * 64 * A.W + lane), c[u].left = A.h - c[u].at;
}

// T: of f and z; R: of the stream x and y.
template <class T, class R, int C, int KIND, int THREADS>
__global__ void __launch_bounds__(THREADS) k_residual_norm(NormArgs A) {
  __shared__ float s_red[2][kWidest][4];
  constexpr bool bias = (KIND & kBias) != 0, branch = (KIND & kBranch) != 0;
  A.mask.begin();
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), team = wave / A.W;
  RowSum sum{s_red, wave, A.W, 0};
  Column c[C];
  columns_of(c, A);
  Row<C> pre, pre_bias, post, post_bias, gate;
#pragma unroll
  for (int u = 0; u < C; u++) {
    parameters<T>(pre.v[u], A.pre, A.wide, c[u], 0.f);
    if (bias) parameters<T>(pre_bias.v[u], A.pre_bias, A.wide, c[u], 0.f);
    if (branch) {
      parameters<T>(post.v[u], A.post, A.wide, c[u], 0.f);
      if (bias) parameters<T>(post_bias.v[u], A.post_bias, A.wide, c[u], 0.f);
      parameters<T>(gate.v[u], A.ptr ? nullptr : A.gate, A.wide, c[u], 1.f);
    }
  }
  const int64_t first = blockIdx.x * A.per, last = min(A.T, first + A.per);
  int s = -1;
  int64_t s_end = branch && A.ptr ? first : A.T;
  for (int64_t base = first; base < last; base += A.teams) {
    const int64_t t = base + team;
    const bool real = t < last;
    Row<C> f, x;
    if (A.f) f.template load<T>(A.f, t * A.f_row, c, real);
    x.template load<R>(A.x, t * A.x_row, c, real);
    if (branch && A.ptr && real && t >= s_end) {
      s = sequence_at(A, t, s + 1, s_end);
#pragma unroll
      for (int u = 0; u < C; u++)
        if (s >= 0)
          parameters<T>(gate.v[u], static_cast<const char *>(A.gate) + (int64_t)s * A.h * (A.wide ? 4 : sizeof(T)), A.wide, c[u], 0.f);
    }
    if (A.f) {
      if (branch && A.post) {
        const float r = normalise(f, A, c, sum);
        EACH(u, e) f.v[u][e] = f.v[u][e] * r * post.v[u][e] + (bias ? post_bias.v[u][e] : 0.f);
      }
      if (A.mask.least) {
#pragma unroll
        for (int u = 0; u < C; u++) A.mask.apply(f.v[u], c[u].at >> 3, (uint32_t)t);
      }
      const bool open = !(branch && A.ptr) || s >= 0;
      EACH(u, e) {
        const float n = branch ? f.v[u][e] * gate.v[u][e] : f.v[u][e];
        x.v[u][e] = fmaf(x.v[u][e], A.scale, open ? n : 0.f);
      }
      if (real) x.template store<R>(A.y, t * A.y_row, c);
    }
    if (A.pre) {
      const float r = normalise(x, A, c, sum);
      EACH(u, e) x.v[u][e] = x.v[u][e] * r * pre.v[u][e] + (bias ? pre_bias.v[u][e] : 0.f);
      if (real) x.template store<T>(A.z, t * A.z_row, c);
    }
  }
}

// The gradient of v = (a norm's value) at g, both as they stand in the row: v less
// its mean if centered, r its factor.  -> g; v becomes the norm's value.
template <int C>
__device__ inline void norm_gradient(Row<C> &g, Row<C> &v, float r, const NormArgs &A, const Column (&c)[C], RowSum &sum) {
  float m[2] = {0.f, 0.f};
  EACH(u, e) {
    v.v[u][e] *= r;
    m[0] = fmaf(g.v[u][e], v.v[u][e], m[0]);
    m[1] += g.v[u][e];
  }
  sum(m);
  const float a = m[0] / A.h, b = A.center ? m[1] / A.h : 0.f;
  EACH(u, e) g.v[u][e] = (g.v[u][e] - b - v.v[u][e] * a) * r;
}

// A team's sums of a vector's gradient to the workgroup's slot.
template <int C>
__device__ inline void leave_sums(Row<C> &acc, const NormArgs &A, float *to, const Column (&c)[C], int team, float *s_join) {
  if (A.teams > 1) {
    __syncthreads();
#pragma unroll
    for (int u = 0; u < C; u++)
      if (c[u].left > 0) {
#pragma unroll
        for (int e = 0; e < 8; e++)
          if (e < c[u].left) s_join[team * A.h + c[u].at + e] = acc.v[u][e];
      }
    __syncthreads();
    for (int k = threadIdx.x; k < A.h; k += blockDim.x) {
      float x = 0.f;
      for (int w = 0; w < A.teams; w++) x += s_join[w * A.h + k];
      to[k] = x;
    }
  } else {
    acc.template store<float>(reinterpret_cast<char *>(to), 0, c);
  }
  EACH(u, e) acc.v[u][e] = 0.f;
}

// The vectors' order in the sums that workgroups leave: pre, pre_bias, post, post_bias, gate.
template <class T, class R, int C, int KIND, int THREADS>
__global__ void __launch_bounds__(THREADS) k_residual_norm_grad(NormArgs A) {
  extern __shared__ float s_join[];
  __shared__ float s_red[2][kWidest][4];
  constexpr bool bias = (KIND & kBias) != 0, branch = (KIND & kBranch) != 0;
  A.mask.begin();
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), team = wave / A.W;
  RowSum sum{s_red, wave, A.W, 0};
  Column c[C];
  columns_of(c, A);
  Row<C> pre, post, post_bias, gate;
  Row<C> d_pre = {}, d_pre_bias = {}, d_post = {}, d_post_bias = {}, d_gate = {};
#pragma unroll
  for (int u = 0; u < C; u++) {
    parameters<T>(pre.v[u], A.pre, A.wide, c[u], 0.f);
    if (branch) {
      parameters<T>(post.v[u], A.post, A.wide, c[u], 0.f);
      if (bias) parameters<T>(post_bias.v[u], A.post_bias, A.wide, c[u], 0.f);
      parameters<T>(gate.v[u], A.ptr ? nullptr : A.gate, A.wide, c[u], 1.f);
    }
  }
  const bool reads_f = branch && (A.post || A.gate);
  const int64_t first = blockIdx.x * A.per, last = min(A.T, first + A.per);
  int s = -1;
  for (int64_t from = first; from < last;) {
    int64_t to = last;
    if (branch && A.ptr) {
      int64_t end;
      s = sequence_at(A, from, s + 1, end);
      to = min(last, end);
#pragma unroll
      for (int u = 0; u < C; u++)
        if (s >= 0)
          parameters<T>(gate.v[u], static_cast<const char *>(A.gate) + (int64_t)s * A.h * (A.wide ? 4 : sizeof(T)), A.wide, c[u], 0.f);
    }
    const bool open = !(branch && A.ptr) || s >= 0;
    for (int64_t base = from; base < to; base += A.teams) {
      const int64_t t = base + team;
      const bool real = t < to, live = real && open;
      Row<C> dy, dz, y, f;
      dy.template load<R>(A.dy, t * A.dy_row, c, real && A.dy);
      if (A.pre) {
        dz.template load<T>(A.dz, t * A.dz_row, c, real);
        y.template load<R>(A.x, t * A.x_row, c, real);
      }
      if (reads_f) f.template load<T>(A.f, t * A.f_row, c, real);
      if (A.pre) {
        const float r = normalise(y, A, c, sum);
        Row<C> g;
        EACH(u, e) g.v[u][e] = dz.v[u][e] * pre.v[u][e];
        norm_gradient(g, y, r, A, c, sum);
        if (real) {  // a row that is not there may have no norm
          EACH(u, e) {
            d_pre.v[u][e] = fmaf(dz.v[u][e], y.v[u][e], d_pre.v[u][e]);
            if (bias) d_pre_bias.v[u][e] += dz.v[u][e];
          }
        }
        EACH(u, e) dy.v[u][e] += g.v[u][e];
      }
      Row<C> dx;
      EACH(u, e) dx.v[u][e] = dy.v[u][e] * A.scale;
      if (real) dx.template store<R>(A.y, t * A.y_row, c);
      if (!A.z) continue;  // no branch at all
      float r = 0.f;
      if (branch && A.post) r = normalise(f, A, c, sum);
      if (branch && A.gate) {
        Row<C> n;
        EACH(u, e) n.v[u][e] = A.post ? f.v[u][e] * r * post.v[u][e] + (bias ? post_bias.v[u][e] : 0.f) : f.v[u][e];
        if (A.mask.least) {
#pragma unroll
          for (int u = 0; u < C; u++) A.mask.apply(n.v[u], c[u].at >> 3, (uint32_t)t);
        }
        if (live) {
          EACH(u, e) d_gate.v[u][e] = fmaf(dy.v[u][e], n.v[u][e], d_gate.v[u][e]);
        }
        EACH(u, e) dy.v[u][e] = open ? dy.v[u][e] * gate.v[u][e] : 0.f;
      }
      if (A.mask.least) {
#pragma unroll
        for (int u = 0; u < C; u++) A.mask.apply(dy.v[u], c[u].at >> 3, (uint32_t)t);
      }
      if (branch && A.post) {
        Row<C> g;
        EACH(u, e) g.v[u][e] = dy.v[u][e] * post.v[u][e];
        norm_gradient(g, f, r, A, c, sum);
        if (live) {
          EACH(u, e) {
            d_post.v[u][e] = fmaf(dy.v[u][e], f.v[u][e], d_post.v[u][e]);
            if (bias) d_post_bias.v[u][e] += dy.v[u][e];
          }
        }
        EACH(u, e) dy.v[u][e] = open ? g.v[u][e] : 0.f;
      }
      if (real) dy.template store<T>(A.z, t * A.z_row, c);
    }
    if (branch && A.gate && s + 1 + (A.ptr == nullptr) > 0)
      leave_sums(d_gate, A, A.part + (4 * A.slots + blockIdx.x + (A.ptr ? s : 0)) * A.h, c, team, s_join);
    from = to;
  }
  float *part = A.part + (int64_t)blockIdx.x * A.h;
  if (A.pre) leave_sums(d_pre, A, part, c, team, s_join);
  if (bias && A.pre_bias) leave_sums(d_pre_bias, A, part + A.slots * A.h, c, team, s_join);
  if (branch && A.post) leave_sums(d_post, A, part + 2 * A.slots * A.h, c, team, s_join);
  if (branch && bias && A.post_bias) leave_sums(d_post_bias, A, part + 3 * A.slots * A.h, c, team, s_join);
}

struct SumArgs {
  const float *part;
  float *to[5];
  int64_t slots, T, per;
  const int32_t *ptr;
  int32_t h, S, groups;
};
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
    for (int64_t k = a + wave * each; k < min(b, a + (wave + 1) * each); k++) x += p[k * A.h];
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
Shape shape_of(const cel_norm_args *a, int64_t most) {
  Shape s;
  const int eights = (int)((a->hidden + 7) / 8);
  s.C = eights > 64 ? kMost : 1;
  s.W = (eights + 64 * s.C - 1) / (64 * s.C);
  s.teams = std::max(1, kWaves / s.W);
  const int64_t groups = std::max<int64_t>(1, std::min(most, (a->rows + s.teams - 1) / s.teams));
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
  NormArgs A{};
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

// go(type, stream type, eights of a lane, kind, threads at most)
template <class F>
void by_type(const cel_norm_args *a, const Shape &s, F go) {
  const int kind = (a->pre_bias || a->post_bias ? kBias : 0) | (a->post || a->gate ? kBranch : 0);
  auto with = [&](auto t, auto r) {
    auto more = [&](auto c, auto threads) {
      if (kind == 0) go(t, r, c, std::integral_constant<int, 0>{}, threads);
      else if (kind == 1) go(t, r, c, std::integral_constant<int, 1>{}, threads);
      else if (kind == 2) go(t, r, c, std::integral_constant<int, 2>{}, threads);
      else go(t, r, c, std::integral_constant<int, 3>{}, threads);
    };
    constexpr std::integral_constant<int, kMost> most{};
    constexpr std::integral_constant<int, 64 * kWaves> usual{};
    if (s.C == 1) more(std::integral_constant<int, 1>{}, usual);
    else if (s.W <= kWaves) more(most, usual);
    else more(most, std::integral_constant<int, 64 * kWidest>{});
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
  const Shape s = shape_of(a, 4 * kGroups);
  NormArgs A = args_of(a, s);
  if (f) A.f = (const char *)f->p, A.f_row = f->stride, A.y = (char *)y->p, A.y_row = y->stride;
  A.x = (const char *)x->p, A.x_row = x->stride;
  if (a->pre) A.z = (char *)z->p, A.z_row = z->stride;
  KTimer kt(st, "k_residual_norm");
  by_type(a, s, [&](auto t, auto r, auto c, auto kind, auto threads) {
    k_residual_norm<decltype(t), decltype(r), decltype(c)::value, decltype(kind)::value, decltype(threads)::value>
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
  const Shape s = shape_of(a, kGroups);
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
    if (dy) A.dy = (const char *)dy->p, A.dy_row = dy->stride;
    if (a->pre) A.dz = (const char *)dz->p, A.dz_row = dz->stride, A.x = (const char *)y->p, A.x_row = y->stride;
    if (a->post || a->gate) A.f = (const char *)f->p, A.f_row = f->stride;
    A.y = (char *)dx->p, A.y_row = dx->stride;
    if (df) A.z = (char *)df->p, A.z_row = df->stride;
    KTimer kt(st, "k_residual_norm_grad");
    by_type(a, s, [&](auto t, auto r, auto c, auto kind, auto threads) {
      k_residual_norm_grad<decltype(t), decltype(r), decltype(c)::value, decltype(kind)::value, decltype(threads)::value>
          <<<(unsigned)s.groups, 64 * s.W * s.teams, s.teams > 1 ? 4 * s.teams * A.h : 0, st>>>(A);
    });
    CEL_HIP(hipGetLastError());
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
