// Passes over operands in front of a product: padded copies, fp32 numbers in three bf16 parts, column sums, what 8-bit floating-point codes stand for.
// All are bound by memory, or, small, by their launch; two operands share one.
#include "rows_prep.h"

namespace convbn {

namespace {

int round8(int n) { return (n + 7) & ~7; }
__device__ __forceinline__ i64 row_of(i64 i, unsigned pieces) { return i >> 32 ? i / pieces : (i64)((unsigned)i / pieces); }

template <typename T> __global__ __launch_bounds__(256) void rows_copy_kernel(RowsCopy a, RowsCopy b, unsigned first) {
  const bool is_a = blockIdx.x < first;
  const RowsCopy p = is_a ? a : b;
  const unsigned wg = is_a ? blockIdx.x : blockIdx.x - first, wgs = is_a ? first : gridDim.x - first;
  const int W8 = (p.width + 7) & ~7, pieces = W8 / 8;
  const i64 total = p.rows * pieces, plane = p.rows * W8;
  for (i64 i = (i64)wg * 256 + threadIdx.x; i < total; i += (i64)wgs * 256) {
    const i64 row = row_of(i, pieces);
    const int k = (int)(i - row * pieces) * 8;
    const F8 v = load8<T>(static_cast<const T*>(p.x) + row * p.ld, k, p.width);
    if constexpr (sizeof(T) == 2) {
      store8<bf16_t>(p.out + row * W8, k, W8, v);
    } else {
      F8 part[3];
      split3(v, part);
#pragma unroll
      for (int x = 0; x < 3; ++x) store8<bf16_t>(p.out + x * plane + row * W8, k, W8, part[x]);
    }
  }
}
unsigned copy_blocks(const RowsCopy& a) {
  const i64 n = (a.rows * (round8(a.width) / 8) + 255) / 256;
  return (unsigned)(a.out ? n < 1 ? 1 : n < 32768 ? n : 32768 : 0);
}

__global__ __launch_bounds__(256) void f8_widen_kernel(F8Widen a, F8Widen b, unsigned first) {
  const bool is_a = blockIdx.x < first;
  const F8Widen p = is_a ? a : b;
  const unsigned wg = is_a ? blockIdx.x : blockIdx.x - first, wgs = is_a ? first : gridDim.x - first;
  const int K8 = (p.K + 7) & ~7, Kp = qrow(p.K), Sp = f8srow(p.K), pieces = K8 / 8;
  const i64 total = p.rows * pieces;
  for (i64 i = (i64)wg * 256 + threadIdx.x; i < total; i += (i64)wgs * 256) {
    const i64 row = row_of(i, pieces);
    const int k = (int)(i - row * pieces) * 8;
    const uint2 c = *reinterpret_cast<const uint2*>(p.q + row * Kp + k);   // (zeros past K)
    store8<bf16_t>(p.out + row * K8, k, K8, f8_decode8(c, scale_of_byte(p.s[row * Sp + k / BLK])));
  }
}

struct SumArgs { i64 M, ldz, per; int N; const void* dz; bf16_t* copy; float* sums; };
// A workgroup takes 256 columns, a thread eight of them and every 16th row of a slice.
template <typename T> __global__ __launch_bounds__(32 * SUM_ROWS) void rows_sums_kernel(SumArgs p) {
  __shared__ float meet[SUM_ROWS][256 + 8];
  const int c = (threadIdx.x & 31) * 8, r = threadIdx.x >> 5, n = blockIdx.x * 256 + c, N8 = (p.N + 7) & ~7;
  const i64 beg = (i64)blockIdx.y * p.per, end = beg + p.per < p.M ? beg + p.per : p.M, plane = p.M * N8;
  F8 sum = {};
  if (n < p.N) {
#pragma unroll 4
    for (i64 m = beg + r; m < end; m += SUM_ROWS) {
      const F8 v = load8<T>(static_cast<const T*>(p.dz) + m * p.ldz, n, p.N);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum.v[e] += v.v[e];
      if (!p.copy) continue;
      if constexpr (sizeof(T) == 2) {
        store8<bf16_t>(p.copy + m * N8, n, N8, v);
      } else {
        F8 part[3];
        split3(v, part);
#pragma unroll
        for (int x = 0; x < 3; ++x) store8<bf16_t>(p.copy + x * plane + m * N8, n, N8, part[x]);
      }
    }
  }
  if (!p.sums) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) meet[r][c + e] = sum.v[e];
  __syncthreads();
  const int at = threadIdx.x, col = blockIdx.x * 256 + at;
  if (at < 256 && col < p.N) {
    float v = 0.f;
#pragma unroll
    for (int i = 0; i < SUM_ROWS; ++i) v += meet[i][at];
    p.sums[(i64)blockIdx.y * p.N + col] = v;
  }
}
__global__ __launch_bounds__(256) void sums_kernel(const float* part, int slices, int N, float* out) {
  const int n = blockIdx.x * 256 + threadIdx.x;
  if (n >= N) return;
  float v = 0.f;
#pragma unroll 8
  for (int s = 0; s < slices; ++s) v += part[(i64)s * N + n];
  out[n] = v;
}
}  // namespace

hipError_t launch_rows_copies(int dtype, const RowsCopy& a, const RowsCopy& b, hipStream_t st) {
  const unsigned na = copy_blocks(a), nb = copy_blocks(b);
  if (!(na + nb)) return hipSuccess;
  if (dtype == CONVBN_BF16) rows_copy_kernel<bf16_t><<<na + nb, 256, 0, st>>>(a, b, na);
  else rows_copy_kernel<float><<<na + nb, 256, 0, st>>>(a, b, na);
  return hipGetLastError();
}


// Some 2048 workgroups, of 32 rows or more (64 slices at most: their sums have to be joined)
int row_slices(i64 M, int N) {
  i64 s = ceil_div(2048, ceil_div(N, 256));
  if (s > M / 32) s = M / 32;
  return (int)(s < 1 ? 1 : s < 64 ? s : 64);
}

hipError_t launch_sums(const float* part, int slices, int N, float* out, hipStream_t st) {
  sums_kernel<<<ceil_div(N, 256), 256, 0, st>>>(part, slices, N, out);
  return hipGetLastError();
}
hipError_t launch_rows_sums(int dtype, i64 M, int N, i64 ldz, const void* dz, bf16_t* copy, float* part, float* out, hipStream_t st) {
  const int slices = row_slices(M, N);
  const SumArgs a = {M, ldz, (M + slices - 1) / slices, N, dz, copy, !out ? nullptr : slices > 1 ? part : out};
  const dim3 grid(ceil_div(N, 256), slices);
  if (dtype == CONVBN_BF16) rows_sums_kernel<bf16_t><<<grid, 32 * SUM_ROWS, 0, st>>>(a);
  else rows_sums_kernel<float><<<grid, 32 * SUM_ROWS, 0, st>>>(a);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess && out && slices > 1 ? launch_sums(part, slices, N, out, st) : e;
}

hipError_t launch_f8_widen(const F8Widen& a, const F8Widen& b, hipStream_t st) {
  auto blocks = [](const F8Widen& w) {
    const i64 n = (w.rows * (round8(w.K) / 8) + 255) / 256;
    return (unsigned)(w.out ? n < 1 ? 1 : n < 32768 ? n : 32768 : 0);
  };
  const unsigned na = blocks(a), nb = blocks(b);
  if (!(na + nb)) return hipSuccess;
  f8_widen_kernel<<<na + nb, 256, 0, st>>>(a, b, na);
  return hipGetLastError();
}

}  // namespace convbn
