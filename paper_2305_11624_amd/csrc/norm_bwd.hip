// Group norm: backward (norm_impl.h has the kernels).
#include "norm_impl.h"

namespace convbn {

hipError_t launch_norm_bwd(const Norm& n, void* ws, hipStream_t st) {
  Plan s = plan_of(n, true);
  s.p.part = static_cast<double2*>(ws);
  const bool params = n.dgamma || n.dbeta;
  float* const sums = reinterpret_cast<float*>(static_cast<char*>(ws) + s.part);
  s.p.sums = params ? sums : nullptr;
  const hipError_t e = n.M ? run_norm<true>(s, st) : hipSuccess;
  if (e != hipSuccess || !params) return e;
  norm_join_kernel<<<ceil_div(n.C, 16), 1024, 0, st>>>(sums, n.M ? s.p.slices * s.p.segs : 0, n.C, n.dgamma, n.dbeta);
  return hipGetLastError();
}

}  // namespace convbn
