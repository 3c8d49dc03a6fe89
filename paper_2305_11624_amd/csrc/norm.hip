// Group norm: workspace, forward (norm_impl.h has the kernels).
#include "norm_impl.h"

namespace convbn {

size_t norm_scratch(const Norm& p, int pass) { return plan_of(p, pass == CONVBN_PASS_BWD).total; }

hipError_t launch_norm_fwd(const Norm& n, void* ws, hipStream_t st) {
  if (!n.M) return hipSuccess;
  Plan s = plan_of(n, false);
  s.p.part = static_cast<double2*>(ws);
  return run_norm<false>(s, st);
}

}  // namespace convbn
