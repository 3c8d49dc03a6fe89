// A head behind the backbone: launchers of the 8-bit floating-point product, the gated product and group norm.
#pragma once
#include "quant.h"

namespace convbn {

// ---- rows in 8-bit floating point: codes as in quant.h, scale bytes e + 127 a block of 128 channels ----
constexpr int BLK = 128;
inline __host__ __device__ int f8srow(int channels) { return (channels + 4 * BLK - 1) / (4 * BLK) * 4; }   // bytes from a row of scales to the next
hipError_t launch_f8_pack(int dtype, i64 rows, int K, i64 ld, const void* x, void* codes, void* scales, hipStream_t st);
hipError_t launch_f8_unpack(int dtype, i64 rows, int K, i64 ld, const void* codes, const void* scales, void* x, hipStream_t st);

// z [M][N] (ldz apart) = x8 . w8^T + b + add
struct F8Mul {
  i64 M, ldz;
  int K, N, dtype;
  const uint8_t* qx; const uint8_t* sx; const uint8_t* qw; const uint8_t* sw; const float* b; const void* add;
  void* z;
};
size_t f8mul_scratch(i64 M, int N, int K);
hipError_t launch_f8mul(const F8Mul& p, void* ws, hipStream_t st);
// The same for few rows (few.hip), which it packs itself: x != null, codes and scales null = not kept
bool f8few_taken(i64 M, int K);
hipError_t launch_f8few(const F8Mul& p, const void* x, i64 ldx, void* codes, void* scales, hipStream_t st);

// dx [M][K] = dz . w8 + add, dW [N][K] = dz^T . x8, db = column sums of dz; dx, dW, db nullable
struct F8Grad {
  i64 M, ldx, ldz;
  int K, N, dtype;
  const uint8_t* qx; const uint8_t* sx; const uint8_t* qw; const uint8_t* sw; const void* dz; const void* add;
  void* dx; void* dW; float* db;
};
size_t f8grad_scratch(const F8Grad& p);
hipError_t launch_f8grad(const F8Grad& p, void* ws, hipStream_t st);

// ---- gated product: x [M][K], W [2 N][K], y [M][N], h [M][2 N] ----
struct Glu {
  i64 M, ldx, ldz;
  int K, N, dtype, gate;
  bool kept;                                          // backward is given h: the workspace has no room for it
  const void* x; const void* W; const float* b;
  void* y; float* h;                                  // forward
  const float* hk; const void* dy; const void* add;    // backward (hk: the kept h, or null)
  void* dx; void* dW; float* db;
};
bool glu_in_place(int dtype, int K, i64 ld);   // bf16 rows that are read where they are, from 16 bytes on
bool glu_few_taken(i64 M, int K, int dtype);   // few rows (few.hip): no workspace
hipError_t launch_glu_few(const Glu& p, hipStream_t st);
size_t glu_scratch(const Glu& p, int pass);
hipError_t launch_glu_fwd(const Glu& p, void* ws, hipStream_t st);
hipError_t launch_glu_bwd(const Glu& p, void* ws, hipStream_t st);

// ---- group norm ----
struct Norm {
  i64 M, P, ldx, ldy;
  int C, groups, dtype, f;
  float eps;
  const void* x; const float* gamma; const float* beta;
  void* y; float* stats;                    // forward; backward reads stats
  const void* dy; const void* add;
  void* dx; float* dgamma; float* dbeta;
};
size_t norm_scratch(const Norm& p, int pass);
hipError_t launch_norm_fwd(const Norm& p, void* ws, hipStream_t st);
hipError_t launch_norm_bwd(const Norm& p, void* ws, hipStream_t st);

}  // namespace convbn
