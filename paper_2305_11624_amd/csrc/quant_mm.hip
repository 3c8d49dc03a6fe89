// z = sx sw (qx . qw) + b + add: the product of 8-bit integers with a scale for each row of either operand.
#include "quant.h"

namespace convbn {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

// A wave's 32 x 32 outputs, operands straight from memory: lane l holds 16 codes of row l % 32 (both operands' channels run
// together, 32 a step).
template <typename T> __global__ __launch_bounds__(256) void qmul_kernel(QMul p) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const i64 m0 = (i64)blockIdx.x * 64 + (wave & 1) * 32;
  const int n0 = blockIdx.y * 64 + (wave >> 1) * 32;
  const int Kp = qrow(p.K), half = (lane >> 5) * 16;
  const i64 m = m0 + (lane & 31);
  const int n = n0 + (lane & 31);
  const int8_t* a = static_cast<const int8_t*>(p.qx) + (m < p.M ? m : 0) * Kp;
  const int8_t* w = static_cast<const int8_t*>(p.qw) + (i64)(n < p.N ? n : 0) * Kp;
  i32x16 acc = {};
  for (int k = half; k < Kp + half; k += 32) {
    i32x4 av = {}, wv = {};
    if (k < Kp) {
      av = *reinterpret_cast<const i32x4*>(a + k);
      wv = *reinterpret_cast<const i32x4*>(w + k);
    }
    acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(av, wv, acc, 0, 0, 0);
  }
  if (n >= p.N) return;
  const float sw = p.sw[n], b = p.b ? p.b[n] : 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const i64 mm = m0 + 8 * (i >> 2) + 4 * (lane >> 5) + (i & 3);
    if (mm >= p.M) continue;
    float v = (float)acc[i] * (p.sx[mm] * sw) + b;
    if (p.add) v += to_f32(static_cast<const T*>(p.add)[mm * p.ldz + n]);
    static_cast<T*>(p.z)[mm * p.ldz + n] = from_f32<T>(v);
  }
}

}  // namespace

hipError_t launch_qmul(const QMul& p, hipStream_t st) {
  const dim3 grid((unsigned)((p.M + 63) / 64), ceil_div(p.N, 64));
  if (p.dtype == CONVBN_BF16) qmul_kernel<bf16_t><<<grid, 256, 0, st>>>(p);
  else qmul_kernel<float><<<grid, 256, 0, st>>>(p);
  return hipGetLastError();
}

}  // namespace convbn
