// Gradients of the 8-bit product from the kept codes: dx = dz . (sw qw) + add, dW = dz^T . (sx qx), db = column sums of dz.
#include "quant.h"

namespace convbn {

namespace {

// C[i][j] = sum_r A(i, r) s[r] q[r][j], 32 x 32 outputs a workgroup, 32 of the reduced index at a time.  TRANS: A(i, r) = dz[r][i].
template <typename T, bool TRANS>
__global__ __launch_bounds__(256) void qgrad_kernel(i64 I, int J, i64 R, const T* __restrict__ dz, i64 ldz, const int8_t* __restrict__ q,
                                                    const float* __restrict__ s, T* C, i64 ldc, const T* add) {
  __shared__ float A[32][33], Bq[32][33];
  const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
  const i64 i0 = (i64)blockIdx.x * 32;
  const int j0 = blockIdx.y * 32, Jp = qrow(J);
  float acc[4] = {};
  for (i64 r0 = 0; r0 < R; r0 += 32) {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int y = ty + 8 * t;
      if (TRANS) A[y][tx] = r0 + y < R && i0 + tx < I ? to_f32(dz[(r0 + y) * ldz + i0 + tx]) : 0.f;   // [r][i]
      else A[tx][y] = i0 + y < I && r0 + tx < R ? to_f32(dz[(i0 + y) * ldz + r0 + tx]) : 0.f;
      Bq[y][tx] = r0 + y < R && j0 + tx < J ? (float)q[(r0 + y) * Jp + j0 + tx] * s[r0 + y] : 0.f;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < 32; ++r)
#pragma unroll
      for (int t = 0; t < 4; ++t) acc[t] += A[r][ty + 8 * t] * Bq[r][tx];
    __syncthreads();
  }
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const i64 i = i0 + ty + 8 * t;
    if (i >= I || j0 + tx >= J) continue;
    const i64 o = i * ldc + j0 + tx;
    C[o] = from_f32<T>(acc[t] + (add ? to_f32(add[o]) : 0.f));
  }
}

template <typename T> __global__ __launch_bounds__(256) void qcolsum_kernel(i64 M, int N, const T* __restrict__ dz, i64 ldz, float* db) {
  __shared__ float part[4][64];
  const int n = blockIdx.x * 64 + (threadIdx.x & 63), w = threadIdx.x >> 6;
  float s = 0.f;
  if (n < N)
    for (i64 m = w; m < M; m += 4) s += to_f32(dz[m * ldz + n]);
  part[w][threadIdx.x & 63] = s;
  __syncthreads();
  if (w == 0 && n < N) db[n] = part[0][threadIdx.x] + part[1][threadIdx.x] + part[2][threadIdx.x] + part[3][threadIdx.x];
}

template <typename T> hipError_t grad_t(const QGrad& p, hipStream_t st) {
  const T* dz = static_cast<const T*>(p.dz);
  if (p.dx && p.M)
    qgrad_kernel<T, false><<<dim3((unsigned)((p.M + 31) / 32), ceil_div(p.K, 32)), 256, 0, st>>>(
        p.M, p.K, p.N, dz, p.ldz, (const int8_t*)p.qw, p.sw, (T*)p.dx, p.ldx, (const T*)p.add);
  if (p.dW)
    qgrad_kernel<T, true><<<dim3(ceil_div(p.N, 32), ceil_div(p.K, 32)), 256, 0, st>>>(
        p.N, p.K, p.M, dz, p.ldz, (const int8_t*)p.qx, p.sx, (T*)p.dW, p.K, nullptr);
  if (p.db) qcolsum_kernel<T><<<ceil_div(p.N, 64), 256, 0, st>>>(p.M, p.N, dz, p.ldz, p.db);
  return hipGetLastError();
}

}  // namespace

size_t qgrad_scratch(const QGrad&) { return 0; }
hipError_t launch_qgrad(const QGrad& p, void*, hipStream_t st) {
  return p.dtype == CONVBN_BF16 ? grad_t<bf16_t>(p, st) : grad_t<float>(p, st);
}

}  // namespace convbn
