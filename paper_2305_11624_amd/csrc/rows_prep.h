// Operands of the products of mm_tile.h, and the passes over them in front of a product: padded copies, fp32 numbers in three bf16 parts, column
// sums, what 8-bit floating-point codes stand for.  All are bound by memory, or, small, by their launch, so that several go in one.
#pragma once
#include "f8_code.h"

namespace convbn {

// An operand: rows of `width` bytes, a multiple of 16, `ld` bytes apart; several planes (parts of fp32 numbers) `plane` bytes apart
struct RowsOp { const uint8_t* p; i64 ld, plane; i64 width; };

// Rows of whole 16-byte pieces with zeros past the last number, for operands that are not read where they are; fp32 numbers in four planes, for
// products with others in four
struct RowsCopy { i64 rows, ld; int width; const void* x; bf16_t* out; };   // (out null: none)
hipError_t launch_rows_copies(int dtype, const RowsCopy& a, const RowsCopy& b, hipStream_t st);


// What codes stand for, as bf16 rows of K rounded up to 8 with zeros past K
struct F8Widen { i64 rows; int K; const uint8_t* q; const uint8_t* s; bf16_t* out; };   // (out null: none)

// Column sums: slices of the rows add up theirs, 16 rows at a time, and a later launch joins the slices in order
constexpr int SUM_ROWS = 16;
struct SumJob { const float* part; int slices, N; float* out; };   // part: [slices][N]; out null: nothing to join
// Some 2048 workgroups, of 32 rows or more (64 slices at most: their sums have to be joined); unsummed rows as finely as that takes
inline int row_slices(i64 M, int N) {
  i64 s = ceil_div(2048, ceil_div(N, 256));
  if (s > M / 32) s = M / 32;
  return (int)(s < 1 ? 1 : s < 64 ? s : 64);
}

namespace {

inline int round8(int n) { return (n + 7) & ~7; }
__device__ __forceinline__ i64 row_of(i64 i, unsigned pieces) { return i >> 32 ? i / pieces : (i64)((unsigned)i / pieces); }

// Workgroup wg of wgs, of NT threads
template <typename T, int NT> __device__ __forceinline__ void rows_copy(const RowsCopy& p, unsigned wg, unsigned wgs) {
  const int W8 = (p.width + 7) & ~7, pieces = W8 / 8;
  const i64 total = p.rows * pieces, plane = p.rows * W8;
  for (i64 i = (i64)wg * NT + threadIdx.x; i < total; i += (i64)wgs * NT) {
    const i64 row = row_of(i, pieces);
    const int k = (int)(i - row * pieces) * 8;
    const F8 v = load8<T>(static_cast<const T*>(p.x) + row * p.ld, k, p.width);
    if constexpr (sizeof(T) == 2) {
      store8<bf16_t>(p.out + row * W8, k, W8, v);
    } else {
      const Parts4 part = split3_near(v);
#pragma unroll
      for (int x = 0; x < 4; ++x) *reinterpret_cast<u32x4*>(p.out + x * plane + row * W8 + k) = part.p[x];
    }
  }
}
template <int NT> __device__ __forceinline__ void f8_widen_rows(const F8Widen& p, unsigned wg, unsigned wgs) {
  const int K8 = (p.K + 7) & ~7, Kp = qrow(p.K), Sp = f8srow(p.K), pieces = K8 / 8;
  const i64 total = p.rows * pieces;
  for (i64 i = (i64)wg * NT + threadIdx.x; i < total; i += (i64)wgs * NT) {
    const i64 row = row_of(i, pieces);
    const int k = (int)(i - row * pieces) * 8;
    const uint2 c = *reinterpret_cast<const uint2*>(p.q + row * Kp + k);   // (zeros past K)
    store8<bf16_t>(p.out + row * K8, k, K8, f8_decode8(c, scale_of_byte(p.s[row * Sp + k / BLK])));
  }
}
template <int NT> unsigned piece_blocks(i64 rows, int width, const void* out) {
  const i64 n = (rows * (round8(width) / 8) + NT - 1) / NT;
  return (unsigned)(out ? n < 1 ? 1 : n < 32768 ? n : 32768 : 0);
}
// Sums of 256 columns over SUM_ROWS threads each, a thread eight of them
__device__ __forceinline__ void meet_sums(const F8& sum, float (*meet)[256 + 8], int n0, int N, float* out) {
  const int c = (threadIdx.x & 31) * 8, r = threadIdx.x >> 5, at = threadIdx.x, col = n0 + at;
  __syncthreads();
#pragma unroll
  for (int e = 0; e < 8; ++e) meet[r][c + e] = sum.v[e];
  __syncthreads();
  if (at < 256 && col < N) {
    float v = 0.f;
#pragma unroll
    for (int i = 0; i < SUM_ROWS; ++i) v += meet[i][at];
    out[col] = v;
  }
}
__device__ __forceinline__ void join_sums(const SumJob& p, int n) {
  if (n >= p.N) return;
  float v = 0.f;
#pragma unroll 8
  for (int s = 0; s < p.slices; ++s) v += p.part[(i64)s * p.N + n];
  p.out[n] = v;
}

}  // namespace

}  // namespace convbn
