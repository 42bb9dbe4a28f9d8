// Rotary positions with several axes, and their gradient.
//
// Pair p of a head's dimensions turns by a = position[axis_p][t] freq_p:
//   u' = u cos a - v sin a,  v' = v cos a + u sin a
// and the gradient turns back.  Pairs are dimensions (p, p + P) or (2 p, 2 p + 1).
//
// The angle is made in 64 bits: at position 2^20 a product in 32 bits is off by
// 0.03.  It is reduced to a part of one turn before sine and cosine, which then take 32 bits.
#include <algorithm>

#include "elements.h"

namespace cel {
namespace {

constexpr int kThreads = 256;

struct RotArgs {
  const char *x;
  char *out;
  int64_t row, head, out_row, out_head;  // strides in elements
  const void *positions, *freqs;
  const int32_t *axes;
  int64_t axis_stride;
  int32_t n_axes, wide_positions, wide_freqs;
  int32_t T, H, d, P;
  int32_t tokens;        // of a workgroup
  int32_t share;         // threads that share a token's heads: each takes every share-th
  Divisor chunks, shares, pairs;
  int32_t turning;       // of a head's chunks, those with pairs; the others are copied
  float sign;
};

// In a cosine's place: the pair has no axis and is copied, not turned by 0, which would make an
// infinity's partner no number.
constexpr float kStays = 2.f;

// Sine and cosine of pair p's angle at token t.  With the product's and the
// factor's rest the turns are exact to 2^-52 of one up to positions of 2^53.
__device__ inline void angle(const RotArgs &A, int p, int t, float &c, float &s) {
#pragma clang fp contract(off)  // n is the rounded product: low is what that lacks
  const int axis = A.axes ? A.axes[p] : 0;
  c = kStays, s = 0.f;
  if (axis < 0 || axis >= A.n_axes) return;
  const int64_t at = axis * A.axis_stride + t;
  const double pos = A.wide_positions ? (double)static_cast<const int64_t *>(A.positions)[at] : (double)static_cast<const int32_t *>(A.positions)[at];
  const double f = A.wide_freqs ? static_cast<const double *>(A.freqs)[p] : (double)static_cast<const float *>(A.freqs)[p];
  constexpr double kTurn = 0.15915494309189535, kTurnRest = -9.839338337591166e-18;  // 1 / (2 pi)
  const double a = pos * f, rest = fma(pos, f, -a);
  const double n = a * kTurn;
  const double low = fma(a, kTurn, -n) + fma(a, kTurnRest, rest * kTurn);
  const float turn = (float)((n - rint(n)) + low);
  sincospif(2.f * turn, &s, &c);
  s *= A.sign;
}

// A workgroup takes some tokens with all their heads: it makes their sines and
// cosines once, in LDS, while the first values are on their way, and a thread then holds those of eight
// pairs and turns them in one head after the other.  Bound by memory: 4,096 tokens of 72 heads of 128,
// 16 bits, in 28 us, 151 MB at 5.4 TB/s, part of them from the caches; 9,973 of 28 heads of 80 in 17 us.  With angles made
// anew for every eight heads 42 and 39 us; with two, four or eight heads' loads on their way at once,
// which takes registers from further waves, 29, 35 and 33 us, and 17, 21 and 24.  In 32 bits 57 us for 302 MB, with
// neighbours as pairs 76: a thread's sixteen are 64 bytes then, and each of its loads takes 16 of every 64.
template <class T, bool PAIRS>
__global__ void __launch_bounds__(kThreads) k_rotary(RotArgs A) {
  extern __shared__ float2 s_angle[];  // [tokens][P]
  const int64_t first_token = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * A.tokens;
  if (first_token >= A.T) return;
  const int t0 = (int)first_token, tokens = min(A.tokens, A.T - t0);
  const int pieces = tokens * A.share * A.chunks.d;
  for (int first = 0; first < pieces; first += kThreads) {
    uint32_t j = first + threadIdx.x;
    const bool in = (int)j < pieces;
    uint32_t h0 = A.chunks.split(j);
    const int t = in ? A.shares.split(h0) : 0;
    const T *x = reinterpret_cast<const T *>(A.x) + (t0 + t) * A.row;
    T *out = reinterpret_cast<T *>(A.out) + (t0 + t) * A.out_row;
    const bool turns = (int)j < A.turning;
    // this thread's two eights of a head, and what there is of each
    int a, b, left_a, left_b;
    if (!turns) {
      a = 2 * A.P + 16 * (j - A.turning), b = a + 8;
      left_a = A.d - a, left_b = A.d - b;
    } else if (PAIRS) {
      a = 16 * j, b = a + 8;
      left_a = 2 * A.P - a, left_b = 2 * A.P - b;
    } else {
      a = 8 * j, b = a + A.P;
      left_a = left_b = A.P - a;
    }
    Eight<T> ra, rb;
    auto load = [&](int h) {
      if (!in || h >= A.H) return;
      ra = load_eight(x + h * A.head + a, left_a);
      rb = load_eight(x + h * A.head + b, left_b);
    };
    load(h0);
    if (first == 0) {
      for (int k = threadIdx.x; k < tokens * A.P; k += kThreads) {
        uint32_t p = k;
        const int u = A.pairs.split(p);
        float2 y;
        angle(A, p, t0 + u, y.x, y.y);
        s_angle[k] = y;
      }
      lds_barrier();
    }
    if (!in) continue;
    float c[8], s[8];
    bool all = turns;  // whether every pair of the eight turns
#pragma unroll
    for (int e = 0; e < 8; e++) {
      c[e] = 1.f, s[e] = 0.f;
      if (turns && 8 * (int)j + e < A.P) {
        const float2 y = s_angle[t * A.P + 8 * j + e];
        c[e] = y.x, s[e] = y.y;
        all = all && y.x != kStays;
      }
    }
    // pair e: (u[e], v[e]), or the neighbours 2 e and 2 e + 1 of the sixteen
    auto turn = [&](float (&u)[8], float (&v)[8], int e) {
      float &p = PAIRS ? (e < 4 ? u[2 * e & 7] : v[2 * e & 7]) : u[e];
      float &q = PAIRS ? (e < 4 ? u[(2 * e + 1) & 7] : v[(2 * e + 1) & 7]) : v[e];
      const float p0 = p, q0 = q;
      p = p0 * c[e] - q0 * s[e];
      q = q0 * c[e] + p0 * s[e];
    };
    for (int h = h0; h < A.H; h += A.share) {
      if (h > (int)h0) load(h);
      float u[8], v[8];
      values<T>(u, ra);
      values<T>(v, rb);
      if (all) {
#pragma unroll
        for (int e = 0; e < 8; e++) turn(u, v, e);
      } else if (turns) {
#pragma unroll
        for (int e = 0; e < 8; e++)
          if (c[e] != kStays) turn(u, v, e);
      }
      store_eight(out + h * A.out_head + a, u, left_a);
      store_eight(out + h * A.out_head + b, v, left_b);
    }
  }
}

int check_view(const cel_rows *x, int size, const char *fn, const char *what) {
  if (!x || !x->p) return set_error(CEL_E_ARG, "%s: %s is NULL", fn, what);
  if (reinterpret_cast<uintptr_t>(x->p) % size) return set_error(CEL_E_ARG, "%s: %s is not aligned to its elements", fn, what);
  if (x->row < 0 || x->head < 0 || x->row > (int64_t(1) << 40) || x->head > (int64_t(1) << 40))
    return set_error(CEL_E_ARG, "%s: %s has a stride out of range", fn, what);
  return CEL_OK;
}

template <class T>
int launch(RotArgs A, bool pairs, hipStream_t s) {
  KTimer kt(s, "k_rotary");
  // a launch has fewer than 2^32 threads along x
  const unsigned groups = (unsigned)((A.T + (int64_t)A.tokens - 1) / A.tokens), x = std::min(groups, 1u << 23);
  const dim3 grid(x, (groups + x - 1) / x);
  const unsigned lds = (unsigned)(sizeof(float2) * A.tokens * A.P);
  if (pairs) k_rotary<T, true><<<grid, kThreads, lds, s>>>(A);
  else k_rotary<T, false><<<grid, kThreads, lds, s>>>(A);
  CEL_HIP(hipGetLastError());
  return CEL_OK;
}

int rotary(const cel_rotary_args *a, const cel_rows *x, const cel_rows *out, float sign, const char *fn, hipStream_t s) {
  if (!a) return set_error(CEL_E_ARG, "%s: NULL descriptor", fn);
  if (a->type < CEL_BF16 || a->type > CEL_F32) return set_error(CEL_E_ARG, "%s: type %d", fn, a->type);
  if (a->tokens < 0 || a->heads < 0 || a->heads > 65535 || a->dim < 1 || a->dim > 4096 || a->pairs < 0 || 2 * a->pairs > a->dim)
    return set_error(CEL_E_ARG, "%s: %d tokens, %d heads of %d, %d pairs", fn, a->tokens, a->heads, a->dim, a->pairs);
  if (a->n_axes < 1 || (a->n_axes > 1 && !a->axes && a->pairs)) return set_error(CEL_E_ARG, "%s: %d axes", fn, a->n_axes);
  if (a->axis_stride < 0 || a->axis_stride > (int64_t(1) << 40)) return set_error(CEL_E_ARG, "%s: axes %lld apart", fn, (long long)a->axis_stride);
  if ((a->position_bytes != 4 && a->position_bytes != 8) || (a->freq_bytes != 4 && a->freq_bytes != 8))
    return set_error(CEL_E_ARG, "%s: positions of %d bytes, frequencies of %d", fn, a->position_bytes, a->freq_bytes);
  if (a->tokens == 0 || a->heads == 0) return CEL_OK;
  const int size = a->type == CEL_F32 ? 4 : 2;
  CEL_TRY(check_view(x, size, fn, "x"));
  CEL_TRY(check_view(out, size, fn, "out"));
  if (a->pairs && (!a->positions || !a->freqs)) return set_error(CEL_E_ARG, "%s: positions or freqs is NULL", fn);
  const int turning = (a->pairs + 7) / 8, copied = (a->dim - 2 * a->pairs + 15) / 16, chunks = turning + copied;
  // As many tokens as give every thread an angle, unless that leaves compute units without a workgroup.
  int tokens = 1;
  while (2 * tokens * std::max(a->pairs, 1) <= kThreads && 2 * tokens * chunks <= kThreads && a->tokens / (2 * tokens) >= 1024) tokens *= 2;
  const int share = std::max(1, std::min(a->heads, kThreads / (tokens * chunks)));
  RotArgs A{(const char *)x->p, (char *)out->p, x->row, x->head, out->row, out->head, a->positions, a->freqs, a->axes, a->axis_stride,
            a->n_axes, a->position_bytes == 8, a->freq_bytes == 8, a->tokens, a->heads, a->dim, a->pairs, tokens, share,
            Divisor(chunks), Divisor(share), Divisor(std::max(a->pairs, 1)), turning, sign};
  const bool pairs = a->interleaved != 0;
  return a->type == CEL_BF16  ? launch<__bf16>(A, pairs, s)
         : a->type == CEL_F16 ? launch<_Float16>(A, pairs, s)
                              : launch<float>(A, pairs, s);
}

}  // namespace
}  // namespace cel

using namespace cel;

extern "C" int cel_rotary(const cel_rotary_args *a, const cel_rows *x, const cel_rows *out, hipStream_t s) {
  return rotary(a, x, out, 1.f, "cel_rotary", s);
}
extern "C" int cel_rotary_grad(const cel_rotary_args *a, const cel_rows *dout, const cel_rows *dx, hipStream_t s) {
  return rotary(a, dout, dx, -1.f, "cel_rotary_grad", s);
}
