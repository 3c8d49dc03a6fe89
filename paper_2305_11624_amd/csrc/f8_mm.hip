// z = x8 . w8^T + b + add: the product of rows in 8-bit floating point, as they are held.
//
// The matrix instruction multiplies e4m3 numbers and takes a power of two for each row and 32 channels of either operand: a block of 128
// channels gives all of its four the same, and the product needs no other step than a plain one.  For fp32 rows the codes become bf16 numbers in front
// of the bf16 instruction, whose sums are fp32 throughout.
//
// Bound by the matrix pipe (mm_tile.h): 8192 x 4096 -> 8192 in 240 - 250 us, 2.2 PFLOP/s; packing the rows in front of it 17 - 20.  8192 x 4096 -> 4096 with it 154,
// fp32 rows 250.
#include "mm_tile.h"

namespace convbn {

namespace {

template <typename T> struct F8Out {
  F8Mul q;
  __device__ __forceinline__ F8 columns(int n) const { return q.b ? load8<float>(q.b, n, q.N) : F8{}; }
  __device__ __forceinline__ void operator()(i64 m, int n, const F8& b, F8 v) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) v.v[i] += b.v[i];
    store8_plus<T>(static_cast<T*>(q.z) + m * q.ldz, q.add ? static_cast<const T*>(q.add) + m * q.ldz : nullptr, n, q.N, v);
  }
};
int chunks_of(int K) { return ceil_div(qrow(K), KB); }

}  // namespace

size_t f8mul_scratch(i64 M, int N, int K) { return mm_scratch(mm_plan(M, N, chunks_of(K)), M, round8(N)); }

hipError_t launch_f8mul(const F8Mul& q, void* ws, hipStream_t st) {
  const int Kp = qrow(q.K);
  MmParams p = {};
  p.a = {q.qx, Kp, 0, Kp};
  p.b = {q.qw, Kp, 0, Kp};
  p.sa = q.sx; p.sb = q.sw; p.srow = f8srow(q.K);
  p.I = q.M; p.J = q.N;
  p.nch = p.plane_ch = chunks_of(q.K);
  const MmPlan pl = mm_plan(q.M, q.N, p.nch);
  if (q.dtype == CONVBN_BF16) return mm_launch<OpF8, false, false, false, 1>(p, pl, static_cast<float*>(ws), F8Out<bf16_t>{q}, st);
  return mm_launch<OpF8Wide, false, false, false, 1>(p, pl, static_cast<float*>(ws), F8Out<float>{q}, st);
}

}  // namespace convbn
