// Gradients of the 8-bit floating-point product from the kept codes: dx = dz . w8 + add, dW = dz^T . x8, db = column sums of dz.
//
// What a code stands for is a bf16 number, so the codes are written out as such, once, and the products are plain ones of bf16 operands that lie across
// the sum; fp32 dz meets them in three bf16 parts that add up to it.
#include "mm_tile.h"
#include "rows_prep.h"

namespace convbn {

namespace {

struct Plan {
  MmPlan dx, dw;
  size_t dz, x, w, part, sums, total;
};
Plan plan_of(const F8Grad& p) {
  Plan s = {};
  const int planes = p.dtype == CONVBN_BF16 ? 1 : 3, N8 = round8(p.N), K8 = round8(p.K);
  s.dx = mm_plan(p.M, p.K, planes * chunks(p.N));
  s.dw = mm_plan(p.N, p.K, planes * chunks(p.M));
  s.dz = qgrad_reads_in_place(p.dtype, p.N, p.ldz) ? 0 : align_up((size_t)planes * p.M * N8 * 2, 256);
  s.x = align_up((size_t)p.M * K8 * 2, 256);
  s.w = align_up((size_t)p.N * K8 * 2, 256);
  s.part = mm_scratch(s.dx, p.M, K8) + mm_scratch(s.dw, p.N, K8);
  s.sums = align_up((size_t)row_slices(p.M, p.N) * p.N * 4, 256);
  s.total = s.dz + s.x + s.w + s.part + s.sums;
  return s;
}

template <typename T> hipError_t grad_t(const F8Grad& p, char* ws, hipStream_t st) {
  constexpr int PAIRS = sizeof(T) == 2 ? 1 : 3;
  const Plan s = plan_of(p);
  const int N8 = round8(p.N), K8 = round8(p.K);
  const bool want_dx = p.dx && p.M;
  bf16_t* const dz = reinterpret_cast<bf16_t*>(ws);
  bf16_t* const x = reinterpret_cast<bf16_t*>(ws + s.dz);
  bf16_t* const w = reinterpret_cast<bf16_t*>(ws + s.dz + s.x);
  float* const part = reinterpret_cast<float*>(ws + s.dz + s.x + s.w);
  float* const sums = reinterpret_cast<float*>(ws + s.dz + s.x + s.w + s.part);
  const bool copies = s.dz && p.M && (p.dx || p.dW);
  hipError_t e = hipSuccess;
  if (copies || p.db) e = launch_rows_sums(p.dtype, p.M, p.N, p.ldz, p.dz, copies ? dz : nullptr, sums, p.db, st);
  if (e == hipSuccess)
    e = launch_f8_widen({p.M, p.K, p.qx, p.sx, p.dW && p.M ? x : nullptr}, {p.N, p.K, p.qw, p.sw, want_dx ? w : nullptr}, st);
  const RowsOp rows = s.dz ? RowsOp{(const uint8_t*)dz, 2 * N8, 2 * p.M * N8, 2 * N8} : RowsOp{(const uint8_t*)p.dz, 2 * p.ldz, 0, 2 * N8};
  if (e == hipSuccess && want_dx) {
    MmParams m = {};
    m.a = rows; m.b = {(const uint8_t*)w, 2 * K8, 0, 2 * K8};
    m.I = p.M; m.J = p.K; m.R = p.N;
    m.plane_ch = chunks(p.N);
    m.nch = PAIRS * m.plane_ch;
    e = mm_launch<OpBf16, false, true, false, PAIRS>(m, s.dx, part, GradOut<T>{p.dx, p.add, p.ldx, p.K}, st);
  }
  if (e == hipSuccess && p.dW) {
    MmParams m = {};
    m.a = rows; m.b = {(const uint8_t*)x, 2 * K8, 0, 2 * K8};
    m.I = p.N; m.J = p.K; m.R = p.M;
    m.plane_ch = chunks(p.M);
    m.nch = PAIRS * m.plane_ch;
    e = mm_launch<OpBf16, true, true, false, PAIRS>(m, s.dw, part + mm_scratch(s.dx, p.M, K8) / 4, GradOut<T>{p.dW, nullptr, p.K, p.K}, st);
  }
  return e;
}

}  // namespace

size_t f8grad_scratch(const F8Grad& p) { return plan_of(p).total; }
hipError_t launch_f8grad(const F8Grad& p, void* ws, hipStream_t st) {
  return p.dtype == CONVBN_BF16 ? grad_t<bf16_t>(p, static_cast<char*>(ws), st) : grad_t<float>(p, static_cast<char*>(ws), st);
}

}  // namespace convbn
