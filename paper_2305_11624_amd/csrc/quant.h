// 8-bit rows: what the kernels of quant_rows.hip, quant_mm.hip and quant_grad.hip share, and their launchers.
#pragma once
#include "common.h"

namespace convbn {

typedef long long i64;

// Bytes from one row of codes to the next: whole 16-byte pieces, zero past the last channel.
inline __host__ __device__ int qrow(int channels) { return (channels + 15) & ~15; }

// ---- rows (quant_rows.hip): ld* in elements ----
hipError_t launch_qpack(int dtype, i64 rows, int K, i64 ld, const void* x, void* codes, float* scales, hipStream_t st);
hipError_t launch_qunpack(int dtype, i64 rows, int K, i64 ld, const void* codes, const float* scales, void* x, hipStream_t st);
// h_codes / h_scales, y, y_codes / y_scales: null = not wanted
hipError_t launch_qgate_fwd(int dtype, int kind, i64 rows, int K, i64 ldh, i64 ldy, const void* h, void* h_codes, float* h_scales,
                            void* y, void* y_codes, float* y_scales, hipStream_t st);
hipError_t launch_qgate_bwd(int dtype, int kind, i64 rows, int K, i64 ldh, i64 ldy, const void* h_codes, const float* h_scales,
                            const void* dy, void* dh, hipStream_t st);

// ---- products ----
// z [M][N] (ldz apart) = sx sw (qx . qw) + b + add
struct QMul {
  i64 M, ldz;
  int K, N, dtype;
  const void* qx; const float* sx; const void* qw; const float* sw; const float* b; const void* add;
  void* z;
};
size_t qmul_scratch(i64 M, int N, int K);
hipError_t launch_qmul(const QMul& p, void* ws, hipStream_t st);

// dx [M][K] = dz . (sw qw) + add, dW [N][K] = dz^T . (sx qx), db = column sums of dz; dx, dW, db nullable
struct QGrad {
  i64 M, ldx, ldz;
  int K, N, dtype;
  const void* qx; const float* sx; const void* qw; const float* sw; const void* dz; const void* add;
  void* dx; void* dW; float* db;
};
size_t qgrad_scratch(const QGrad& p);
hipError_t launch_qgrad(const QGrad& p, void* ws, hipStream_t st);

// api.hip: keeps the message for convbn_last_error and returns the code
convbn_status set_error(convbn_status code, const char* fmt, ...);

}  // namespace convbn
