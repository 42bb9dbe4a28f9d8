// Rows of numbers eight at a time, sums over a wave, and the generator of
// dropout's masks: what the element-wise operations of a training step share.
#pragma once
#include "cel_internal.h"

namespace cel {

// Eight numbers at any address of their type, as accesses of up to 16 bytes.
template <class T>
struct __attribute__((packed, aligned(2))) Eight {
  uint32_t w[2 * sizeof(T)];
};
// Numbers p[0] .. p[7], of which those at or past `left` do not exist (0 in their place).
template <class T>
__device__ inline Eight<T> load_eight(const T *p, int64_t left) {
  Eight<T> r;
  if (left >= 8) {
    r = *reinterpret_cast<const Eight<T> *>(p);
  } else {
    T x[8];
#pragma unroll
    for (int e = 0; e < 8; e++) x[e] = e < left ? p[e] : (T)0.f;
    __builtin_memcpy(&r, x, sizeof r);
  }
  return r;
}
template <class T>
__device__ inline void values(float (&f)[8], const Eight<T> &r) {
  T x[8];
  __builtin_memcpy(x, &r, sizeof r);
#pragma unroll
  for (int e = 0; e < 8; e++) f[e] = (float)x[e];
}
template <class T>
__device__ inline void store_eight(T *p, const float (&f)[8], int64_t left) {
  T x[8];
#pragma unroll
  for (int e = 0; e < 8; e++) x[e] = (T)f[e];
  if (left >= 8) {
    Eight<T> r;
    __builtin_memcpy(&r, x, sizeof r);
    *reinterpret_cast<Eight<T> *>(p) = r;
  } else {
#pragma unroll
    for (int e = 0; e < 8; e++)
      if (e < left) p[e] = x[e];
  }
}

// Counter-based generator of Salmon, Moraes, Dror and Shaw ("Parallel random
// numbers: as easy as 1, 2, 3", SC 2011): Philox4x32 with ten rounds.  Four words
// are a function of a 128-bit counter and a 64-bit key alone.
struct Words {
  uint32_t w[4];
};
__host__ __device__ inline Words philox(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int i = 0; i < 10; i++) {
    const uint64_t a = uint64_t(0xd2511f53u) * c0, b = uint64_t(0xcd9e8d57u) * c2;
    c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
    c1 = (uint32_t)b;
    c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
    c3 = (uint32_t)a;
    k0 += 0x9e3779b9u, k1 += 0xbb67ae85u;
  }
  return Words{{c0, c1, c2, c3}};
}
// Dropout of value (r, c): the counter is (c / 8, r, step), the key the seed, and
// value c has 16 of the 128 bits, c % 8 from below.  It stays where these are at least `least`.
struct Mask {
  uint32_t k0, k1, s0, s1;  // seed and step
  uint32_t least;           // 2^16 p, rounded; 0: nothing is dropped
  float by;                 // 1 / (1 - least / 2^16), of what stays
  const int64_t *step;      // NULL, or added to the step on the device
  // The step as the kernel finds it.
  __device__ void begin() {
    if (!step) return;
    const uint64_t s = ((uint64_t)s1 << 32 | s0) + (uint64_t)*step;
    s0 = (uint32_t)s, s1 = (uint32_t)(s >> 32);
  }
  // Values of row r, block c / 8: what is dropped becomes 0 whatever it was.
  __device__ void apply(float (&f)[8], uint32_t block, uint32_t row) const {
    const Words x = philox(block, row, s0, s1, k0, k1);
#pragma unroll
    for (int e = 0; e < 8; e++) f[e] = (e & 1 ? x.w[e / 2] >> 16 : x.w[e / 2] & 0xffffu) >= least ? f[e] * by : 0.f;
  }
};
inline int check_mask(const cel_mask *m, const char *fn) {
  if (!(m->p >= 0.0 && m->p <= 1.0)) return set_error(CEL_E_ARG, "%s: a probability of %g", fn, m->p);
  return CEL_OK;
}
inline Mask mask_of(const cel_mask *m) {
  const uint32_t least = (uint32_t)(m->p * 65536.0 + 0.5);
  return Mask{(uint32_t)m->seed, (uint32_t)(m->seed >> 32), (uint32_t)m->step, (uint32_t)((uint64_t)m->step >> 32), least,
              least >= 65536u ? 0.f : (float)(65536.0 / (65536.0 - least)), m->step_at};
}

// Sums over the 64 lanes, in all of them, in a fixed order.
template <int CTRL>
__device__ inline float dpp_add(float x) {
  return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
__device__ inline float wave_sum(float x) {
  typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
  x = dpp_add<0x128>(x);  // rotations inside 16 lanes by 8, 4, 2 and 1
  x = dpp_add<0x124>(x);
  x = dpp_add<0x122>(x);
  x = dpp_add<0x121>(x);
  u32x2 r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// n / d for a divisor that the host knows.
struct Divisor {
  uint32_t d, m;  // m = 2^32 / d rounded down, at most 2^32 - 1
  explicit Divisor(uint32_t d_) : d(d_), m(d_ > 1 ? (uint32_t)((uint64_t(1) << 32) / d_) : ~0u) {}
  // -> the quotient; n becomes the remainder.  n m / 2^32 is less than 1 below n / d.
  __device__ uint32_t split(uint32_t &n) const {
    uint32_t q = __umulhi(n, m);
    n -= q * d;
    if (n >= d) q++, n -= d;
    return q;
  }
};

}  // namespace cel
