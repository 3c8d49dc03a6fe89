// The two products of a backward pass: launcher of grads.hip.
#pragma once
#include "rows_prep.h"

namespace convbn {

// dx [M][K] = a . w + add, dW [N][K] = a^T . x (either null = not wanted) for a [M][N], w [N][K], x [M][K] as bf16 operands; pairs = 1: of one plane each, 3: a has
// three, 6: all have.  `sum` is joined on the way.
struct Grads {
  i64 M, N, ldx;
  int K, pairs, dtype;
  RowsOp a, w, x;
  void* dx; const void* add;
  void* dW;
  SumJob sum;
};
size_t grads_scratch(i64 M, i64 N, int K, int pairs);
hipError_t launch_grads(const Grads& g, float* part, hipStream_t st);

}  // namespace convbn
