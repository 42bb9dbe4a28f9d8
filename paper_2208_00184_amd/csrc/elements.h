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
// The same of a row of n >= 8 numbers from number `at` on, without a branch that a wave would wait in: where
// the row ends inside the eight they come from its last eight, and shift_down puts them in their place.
template <class T>
__device__ inline Eight<T> load_back(const T *row, int at, int n) {
  return *reinterpret_cast<const Eight<T> *>(row + min(at, n - 8));
}
// f[e] = f[e + by], 0 behind the last.
__device__ inline void shift_down(float (&f)[8], int by) {
#pragma unroll
  for (int step = 4; step; step /= 2) {
    const bool on = by & step;
#pragma unroll
    for (int e = 0; e < 8; e++) f[e] = on ? (e + step < 8 ? f[e + step] : 0.f) : f[e];
  }
#pragma unroll
  for (int e = 0; e < 8; e++) f[e] = by >= 8 ? 0.f : f[e];
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
    // As words that the compiler does not know from the single stores below: it would make one
    // of both branches' first store, and the wide store three narrow ones.
    uint32_t w[2 * sizeof(T)];
    __builtin_memcpy(w, x, sizeof w);
#pragma unroll
    for (uint32_t &y : w) asm("" : "+v"(y));
    Eight<T> r;
    __builtin_memcpy(&r, w, sizeof r);
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
  // Which values of row r, block c / 8 stay: a condition of each, which takes no vector registers.
  __device__ void kept(bool (&k)[8], uint32_t block, uint32_t row) const {
    const Words x = philox(block, row, s0, s1, k0, k1);
#pragma unroll
    for (int e = 0; e < 8; e++) k[e] = (e & 1 ? x.w[e / 2] >> 16 : x.w[e / 2] & 0xffffu) >= least;
  }
  // The conditions as bits, for later; x where condition e of them holds, else 0.
  __device__ static uint32_t bits(const bool (&k)[8]) {
    uint32_t b = 0;
#pragma unroll
    for (int e = 7; e >= 0; e--) b = b + b + k[e];
    return b;
  }
  __device__ static float where(uint32_t b, int e, float x) {
    return __uint_as_float(__float_as_uint(x) & (uint32_t)__builtin_amdgcn_sbfe((int)b, e, 1));
  }
  // What is dropped becomes 0 whatever it was.
  __device__ void apply(float (&f)[8], const bool (&k)[8]) const {
#pragma unroll
    for (int e = 0; e < 8; e++) f[e] = k[e] ? f[e] * by : 0.f;
  }
  __device__ void apply(float (&f)[8], uint32_t block, uint32_t row) const {
    bool k[8];
    kept(k, block, row);
    apply(f, k);
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

template <int CTRL>
__device__ inline float dpp_add(float x) {
  return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
// The sum over 16 lanes beside each other, in all of them, by rotations.
__device__ inline float sixteen_sum(float x) {
  x = dpp_add<0x128>(x);
  x = dpp_add<0x124>(x);
  x = dpp_add<0x122>(x);
  return dpp_add<0x121>(x);
}
// Sums of N numbers a lane over 64 lanes, in a fixed order.  A swap of halves (or of 16 lanes) puts two
// numbers' sums into one register, so that N of them take little more than one: value v's sum is
// in register v / 4, in the 16 lanes from at(v) on.
template <int N>
struct LaneSums {
  static constexpr int kRegisters = (N + 3) / 4;
  float r[kRegisters];
  static constexpr int at(int v) {
    constexpr int rows[4] = {0, 2, 1, 3};
    const bool alone = v / 4 * 4 + 2 >= N;  // a register with two numbers
    return 16 * (alone ? v % 4 * 2 : rows[v % 4]);
  }
  __device__ explicit LaneSums(const float (&x)[N]) {
    typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
#pragma unroll
    for (int j = 0; j < kRegisters; j++) {
      float a[2];
#pragma unroll
      for (int k = 0; k < 2; k++) {
        const int v = 4 * j + 2 * k;
        if (v >= N) continue;
        const u32x2 y = __builtin_amdgcn_permlane32_swap(__float_as_uint(x[v]), v + 1 < N ? __float_as_uint(x[v + 1 < N ? v + 1 : v]) : 0u,
                                                         false, false);
        a[k] = __uint_as_float(y[0]) + __uint_as_float(y[1]);
      }
      const float b = 4 * j + 2 < N ? a[1] : a[0];
      const u32x2 y = __builtin_amdgcn_permlane16_swap(__float_as_uint(a[0]), __float_as_uint(b), false, false);
      r[j] = sixteen_sum(__uint_as_float(y[0]) + __uint_as_float(y[1]));
    }
  }
  __device__ void get(float (&x)[N]) const {
#pragma unroll
    for (int v = 0; v < N; v++) x[v] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(r[v / 4]), at(v)));
  }
};

// n / d for a divisor that the host knows.
struct Divisor {
  uint32_t d, m;  // m = 2^32 / d rounded down, at most 2^32 - 1
  Divisor() = default;
  explicit Divisor(uint32_t d_) : d(d_), m(d_ > 1 ? (uint32_t)((uint64_t(1) << 32) / d_) : ~0u) {}
  // -> the quotient; n becomes the remainder.  n m / 2^32 is less than 1 below n / d.
  __device__ uint32_t split(uint32_t &n) const {
    uint32_t q = __umulhi(n, m);
    n -= q * d;
    if (n >= d) q++, n -= d;
    return q;
  }
  __device__ uint32_t quotient(uint32_t n) const { return split(n); }
};

}  // namespace cel
