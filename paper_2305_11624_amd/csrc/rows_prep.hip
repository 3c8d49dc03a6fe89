// Copies of operands in front of a forward product (rows_prep.h).
#include "rows_prep.h"

namespace convbn {

namespace {

template <typename T> __global__ __launch_bounds__(256) void rows_copy_kernel(RowsCopy a, RowsCopy b, unsigned first) {
  if (blockIdx.x < first) rows_copy<T, 256>(a, blockIdx.x, first);
  else rows_copy<T, 256>(b, blockIdx.x - first, gridDim.x - first);
}

}  // namespace

hipError_t launch_rows_copies(int dtype, const RowsCopy& a, const RowsCopy& b, hipStream_t st) {
  const unsigned na = piece_blocks<256>(a.rows, a.width, a.out), nb = piece_blocks<256>(b.rows, b.width, b.out);
  if (!(na + nb)) return hipSuccess;
  if (dtype == CONVBN_BF16) rows_copy_kernel<bf16_t><<<na + nb, 256, 0, st>>>(a, b, na);
  else rows_copy_kernel<float><<<na + nb, 256, 0, st>>>(a, b, na);
  return hipGetLastError();
}

}  // namespace convbn
