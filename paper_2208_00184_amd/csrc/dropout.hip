// Dropout from a counter-based generator: no mask is stored, forward and
// backward passes make the same one anew.
//
//   y_rc = x_rc / (1 - p) where value (r, c) stays, else 0
//
// Every thread makes one block of the generator, 128 bits, for eight values of a row.
#include <algorithm>

#include "elements.h"

namespace cel {
namespace {

constexpr int kThreads = 256;
constexpr int kEach = 4;  // pieces of eight values a thread takes

struct DropArgs {
  const char *x;
  char *out;
  int64_t stride, out_stride;  // in elements
  int64_t columns;
  uint32_t pieces, row0;       // eights in this launch; its first row
  Divisor blocks;              // eights of a row
  Mask mask;
};

// The loads of all of a thread's pieces are on their way before the generator runs.
template <class T>
__global__ void __launch_bounds__(kThreads) k_dropout(DropArgs A) {
  A.mask.begin();
  const uint32_t first = blockIdx.x * (kThreads * kEach) + threadIdx.x;
  Eight<T> x[kEach];
  uint32_t row[kEach], block[kEach];
#pragma unroll
  for (int i = 0; i < kEach; i++) {
    block[i] = first + i * kThreads;
    const bool in = block[i] < A.pieces;
    row[i] = A.blocks.split(block[i]);
    if (in)
      x[i] = load_eight(reinterpret_cast<const T *>(A.x) + row[i] * A.stride + (int64_t)block[i] * 8, A.columns - (int64_t)block[i] * 8);
  }
#pragma unroll
  for (int i = 0; i < kEach; i++) {
    if (first + i * kThreads >= A.pieces) break;
    float f[8];
    values<T>(f, x[i]);
    A.mask.apply(f, block[i], A.row0 + row[i]);
    store_eight(reinterpret_cast<T *>(A.out) + row[i] * A.out_stride + (int64_t)block[i] * 8, f, A.columns - (int64_t)block[i] * 8);
  }
}

int check_matrix(const cel_matrix *x, const cel_dropout_args *a, int size, const char *what) {
  if (!x || !x->p) return set_error(CEL_E_ARG, "cel_dropout: %s is NULL", what);
  if (reinterpret_cast<uintptr_t>(x->p) % size) return set_error(CEL_E_ARG, "cel_dropout: %s is not aligned to its elements", what);
  if (x->stride < a->columns || x->stride > (int64_t(1) << 40))
    return set_error(CEL_E_ARG, "cel_dropout: %s has rows of %lld values %lld apart", what, (long long)a->columns, (long long)x->stride);
  return CEL_OK;
}

template <class T>
int dropout(const cel_dropout_args *a, const cel_matrix *x, const cel_matrix *out, hipStream_t s) {
  const int64_t blocks = (a->columns + 7) / 8;
  // a launch's pieces are counted in 32 bits, the surplus of its last workgroup among them
  const int64_t rows = std::max<int64_t>(1, (UINT32_MAX - kThreads * kEach) / blocks);
  KTimer kt(s, "k_dropout");
  for (int64_t r = 0; r < a->rows; r += rows) {
    const int64_t n = std::min(rows, a->rows - r);
    DropArgs A{(const char *)x->p + r * x->stride * (int64_t)sizeof(T),
               (char *)out->p + r * out->stride * (int64_t)sizeof(T),
               x->stride, out->stride, a->columns, (uint32_t)(n * blocks), (uint32_t)r, Divisor((uint32_t)blocks), mask_of(&a->mask)};
    k_dropout<T><<<(unsigned)((n * blocks + kThreads * kEach - 1) / (kThreads * kEach)), kThreads, 0, s>>>(A);
    CEL_HIP(hipGetLastError());
  }
  return CEL_OK;
}

}  // namespace
}  // namespace cel

using namespace cel;

extern "C" int cel_dropout(const cel_dropout_args *a, const cel_matrix *x, const cel_matrix *out, hipStream_t s) {
  const char *fn = "cel_dropout";
  if (!a) return set_error(CEL_E_ARG, "%s: NULL descriptor", fn);
  if (a->type < CEL_BF16 || a->type > CEL_F32) return set_error(CEL_E_ARG, "%s: type %d", fn, a->type);
  if (a->rows < 0 || a->rows > UINT32_MAX || a->columns < 0 || a->columns > INT32_MAX)
    return set_error(CEL_E_ARG, "%s: %lld rows of %lld values", fn, (long long)a->rows, (long long)a->columns);
  CEL_TRY(check_mask(&a->mask, fn));
  if (a->rows == 0 || a->columns == 0) return CEL_OK;
  const int size = a->type == CEL_F32 ? 4 : 2;
  CEL_TRY(check_matrix(x, a, size, "x"));
  CEL_TRY(check_matrix(out, a, size, "out"));
  return a->type == CEL_BF16  ? dropout<__bf16>(a, x, out, s)
         : a->type == CEL_F16 ? dropout<_Float16>(a, x, out, s)
                              : dropout<float>(a, x, out, s);
}
