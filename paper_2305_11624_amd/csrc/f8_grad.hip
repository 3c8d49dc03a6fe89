// Gradients of the 8-bit floating-point product from the kept codes: dx = dz . w8 + add, dW = dz^T . x8, db = column sums of dz.
//
// What a code stands for is a bf16 number, so the codes are written out as such, once, and the products are plain ones of bf16 operands that lie across
// the sum; fp32 dz meets them in three bf16 parts that add up to it.  One pass does all that comes in front: the codes of x and of the weight, a copy of dz
// where it is not read in place, its column sums.  That pass is bound by memory (8192 x 4096 and 4096 x 4096 codes 25 us, 154 MB), the products as mm_tile.h says (214 and
// 208 us, 1280 and 1320 TFLOP/s; fp32 dz, three products each, 1320 in all); 1568 x 2048 -> 512, all three gradients, is four launches' worth of waiting.
#include "grads.h"

namespace convbn {

namespace {

struct Plan { size_t dz, x, w, part, sums, total; };
int pairs_of(int dtype) { return dtype == CONVBN_BF16 ? 1 : 3; }
Plan plan_of(const F8Grad& p) {
  Plan s = {};
  const int pairs = pairs_of(p.dtype), N8 = round8(p.N), K8 = round8(p.K);
  s.dz = qgrad_reads_in_place(p.dtype, p.N, p.ldz) ? 0 : align_up((size_t)pairs * p.M * N8 * 2, 256);
  s.x = align_up((size_t)p.M * K8 * 2, 256);
  s.w = align_up((size_t)p.N * K8 * 2, 256);
  s.part = grads_scratch(p.M, p.N, p.K, pairs);
  s.sums = align_up((size_t)row_slices(p.M, p.N) * p.N * 4, 256);
  s.total = s.dz + s.x + s.w + s.part + s.sums;
  return s;
}

// dz: workgroups of 256 columns and a slice of the rows, a thread eight columns of every 16th row
constexpr int NT = 32 * SUM_ROWS;
struct Dz { i64 M, ldz, per; int N, across, blocks; const void* dz; bf16_t* copy; float* sums; };
template <typename T> __global__ __launch_bounds__(NT) void f8_prep_kernel(Dz p, F8Widen x, unsigned nx, F8Widen w) {
  __shared__ float meet[SUM_ROWS][256 + 8];
  if ((int)blockIdx.x >= p.blocks) {
    const unsigned wg = blockIdx.x - p.blocks;
    if (wg < nx) f8_widen_rows<NT>(x, wg, nx);
    else f8_widen_rows<NT>(w, wg - nx, gridDim.x - p.blocks - nx);
    return;
  }
  const int slice = (int)blockIdx.x / p.across, n0 = ((int)blockIdx.x - slice * p.across) * 256, n = n0 + (threadIdx.x & 31) * 8;
  const int r = threadIdx.x >> 5, N8 = (p.N + 7) & ~7;
  const i64 beg = (i64)slice * p.per, end = beg + p.per < p.M ? beg + p.per : p.M, plane = p.M * N8;
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
        for (int i = 0; i < 3; ++i) store8<bf16_t>(p.copy + i * plane + m * N8, n, N8, part[i]);
      }
    }
  }
  if (p.sums) meet_sums(sum, meet, n0, p.N, p.sums + (i64)slice * p.N);
}

__global__ __launch_bounds__(256) void f8_widen_kernel(F8Widen x, unsigned nx, F8Widen w) {
  if (blockIdx.x < nx) f8_widen_rows<256>(x, blockIdx.x, nx);
  else f8_widen_rows<256>(w, blockIdx.x - nx, gridDim.x - nx);
}

template <typename T> hipError_t grad_t(const F8Grad& p, char* ws, hipStream_t st) {
  const Plan s = plan_of(p);
  const int N8 = round8(p.N), K8 = round8(p.K), slices = row_slices(p.M, p.N);
  bf16_t* const dz = reinterpret_cast<bf16_t*>(ws);
  bf16_t* const x = reinterpret_cast<bf16_t*>(ws + s.dz);
  bf16_t* const w = reinterpret_cast<bf16_t*>(ws + s.dz + s.x);
  float* const sums = reinterpret_cast<float*>(ws + s.dz + s.x + s.w + s.part);
  const bool copies = s.dz && p.M && (p.dx || p.dW);
  Dz d = {p.M, p.ldz, (p.M + slices - 1) / slices, p.N, ceil_div(p.N, 256), 0, p.dz, copies ? dz : nullptr, !p.db ? nullptr : slices > 1 ? sums : p.db};
  if (copies || p.db) d.blocks = d.across * slices;
  const F8Widen fx = {p.M, p.K, p.qx, p.sx, p.dW && p.M ? x : nullptr}, fw = {p.N, p.K, p.qw, p.sw, p.dx && p.M ? w : nullptr};
  if (d.blocks) {
    const unsigned nx = piece_blocks<NT>(p.M, p.K, fx.out), nw = piece_blocks<NT>(p.N, p.K, fw.out);
    f8_prep_kernel<T><<<d.blocks + nx + nw, NT, 0, st>>>(d, fx, nx, fw);
  } else {   // (codes alone: a kernel of fewer registers; both gradients of 8192 x 4096 x 4096 8 us sooner)
    const unsigned nx = piece_blocks<256>(p.M, p.K, fx.out), nw = piece_blocks<256>(p.N, p.K, fw.out);
    if (nx + nw) f8_widen_kernel<<<nx + nw, 256, 0, st>>>(fx, nx, fw);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  Grads g = {};
  g.M = p.M; g.N = p.N; g.K = p.K; g.ldx = p.ldx; g.pairs = pairs_of(p.dtype); g.dtype = p.dtype;
  g.a = s.dz ? RowsOp{(const uint8_t*)dz, 2 * N8, 2 * p.M * N8, 2 * N8} : RowsOp{(const uint8_t*)p.dz, 2 * p.ldz, 0, 2 * N8};
  g.w = {(const uint8_t*)w, 2 * K8, 0, 2 * K8};
  g.x = {(const uint8_t*)x, 2 * K8, 0, 2 * K8};
  g.dx = p.dx; g.add = p.add; g.dW = p.dW;
  g.sum = {sums, slices, p.N, slices > 1 ? p.db : nullptr};
  return launch_grads(g, reinterpret_cast<float*>(ws + s.dz + s.x + s.w), st);
}

}  // namespace

size_t f8grad_scratch(const F8Grad& p) { return plan_of(p).total; }
hipError_t launch_f8grad(const F8Grad& p, void* ws, hipStream_t st) {
  return p.dtype == CONVBN_BF16 ? grad_t<bf16_t>(p, static_cast<char*>(ws), st) : grad_t<float>(p, static_cast<char*>(ws), st);
}

}  // namespace convbn
