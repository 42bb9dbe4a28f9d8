// Dropout from a counter-based generator: no mask is stored, forward and
// backward passes make the same one anew.
//
//   y_rc = x_rc / (1 - p) where value (r, c) stays, else 0
//
// Every thread makes one block of the generator, 128 bits, for eight values of a row, while
// these are on their way.  Bound by memory: 4,096 rows of 32,768 in 16 bits in 89 us, 537 MB
// at 6.0 TB/s, part of them from the caches; a thread with two, four or eight pieces one behind the other
// leaves fewer waves to wait for memory (93, 99 and 104 us).
#include <algorithm>

#include "elements.h"

namespace cel {
namespace {

constexpr int kThreads = 256;

struct DropArgs {
  const char *x;
  char *out;
  int64_t stride, out_stride;  // in elements
  int64_t columns;
  uint32_t pieces, row0;       // eights in this launch; its first row
  Divisor blocks;              // eights of a row
  Mask mask;
};

template <class T>
__global__ void __launch_bounds__(kThreads) k_dropout(DropArgs A) {
  uint32_t block = blockIdx.x * kThreads + threadIdx.x;
  if (block >= A.pieces) return;
  const uint32_t row = A.blocks.split(block);
  const int64_t c = (int64_t)block * 8;
  const Eight<T> x = load_eight(reinterpret_cast<const T *>(A.x) + row * A.stride + c, A.columns - c);
  A.mask.begin();
  float f[8];
  values<T>(f, x);
  A.mask.apply(f, block, A.row0 + row);
  store_eight(reinterpret_cast<T *>(A.out) + row * A.out_stride + c, f, A.columns - c);
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
  const int64_t rows = std::max<int64_t>(1, (UINT32_MAX - kThreads) / blocks);
  KTimer kt(s, "k_dropout");
  for (int64_t r = 0; r < a->rows; r += rows) {
    const int64_t n = std::min(rows, a->rows - r);
    DropArgs A{(const char *)x->p + r * x->stride * (int64_t)sizeof(T),
               (char *)out->p + r * out->stride * (int64_t)sizeof(T),
               x->stride, out->stride, a->columns, (uint32_t)(n * blocks), (uint32_t)r, Divisor((uint32_t)blocks), mask_of(&a->mask)};
    k_dropout<T><<<(unsigned)((n * blocks + kThreads - 1) / kThreads), kThreads, 0, s>>>(A);
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
