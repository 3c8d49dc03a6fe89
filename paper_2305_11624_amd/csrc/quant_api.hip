// C ABI of the 8-bit rows: argument checks, workspace and launch sequences.  Host code only enqueues.
#include "row_checks.h"

using namespace convbn;

namespace {

QGrad grad_of(const convbn_qdesc* d, i64 ldx, i64 ldz) {
  QGrad g = {};
  g.M = d->M; g.ldx = ldx; g.ldz = ldz; g.K = d->K; g.N = d->N; g.dtype = d->dtype;
  g.add = (d->act & CONVBN_ACT_ADD_IN) ? d->add_in : nullptr;
  return g;
}
// Forward workspace: the product's, then codes and scales that the call does not hand out
size_t mul_ws(const convbn_qdesc* d) { return qfew_taken(d->M, d->N, d->K) ? 0 : qmul_scratch(d->M, d->N, d->K); }
size_t codes_ws(const convbn_qdesc* d) { return align_up((size_t)d->M * qrow(d->K), 256); }
size_t fwd_ws(const convbn_qdesc* d) {
  if (qfew_taken(d->M, d->N, d->K) && qfew_packs(d->M, d->N, d->K)) return 0;
  return mul_ws(d) + codes_ws(d) + align_up((size_t)d->M * 4, 256);
}

}  // namespace

extern "C" {

size_t convbn_qrow_bytes(int32_t channels) { return channels < 1 || channels > 1 << 30 ? 0 : (size_t)qrow(channels); }

convbn_status convbn_qpack(const convbn_qdesc* desc, const void* x, void* codes, float* scales, void* stream) {
  i64 ld;
  TRY_STATUS(check_rows(desc, &ld));
  REQUIRE_ROWS(x, elem(desc)); REQUIRE_ROWS(codes, 16); REQUIRE_ROWS(scales, 4);
  LAUNCH(launch_qpack(desc->dtype, desc->M, desc->K, ld, x, codes, scales, (hipStream_t)stream));
  return CONVBN_OK;
}

convbn_status convbn_qunpack(const convbn_qdesc* desc, const void* codes, const float* scales, void* x, void* stream) {
  i64 ld;
  TRY_STATUS(check_rows(desc, &ld));
  REQUIRE_ROWS(codes, 16); REQUIRE_ROWS(scales, 4); REQUIRE_ROWS(x, elem(desc));
  LAUNCH(launch_qunpack(desc->dtype, desc->M, desc->K, ld, codes, scales, x, (hipStream_t)stream));
  return CONVBN_OK;
}

size_t convbn_qlinear_workspace_bytes(const convbn_qdesc* desc, int pass) {
  i64 ldx, ldz;
  if (check_linear(desc, &ldx, &ldz) != CONVBN_OK) return 0;
  return pass == CONVBN_PASS_FWD ? fwd_ws(desc) : qgrad_scratch(grad_of(desc, ldx, ldz));
}

convbn_status convbn_qlinear_fwd(const convbn_qdesc* desc, const void* x, void* codes, float* scales, const void* w_codes,
                                 const float* w_scales, const float* b, void* z, void* ws, size_t ws_bytes, void* stream) {
  i64 ldx, ldz;
  TRY_STATUS(check_linear(desc, &ldx, &ldz));
  OPTIONAL(x, elem(desc));
  if (!x) { REQUIRE_ROWS(codes, 16); REQUIRE_ROWS(scales, 4); }
  OPTIONAL(codes, 16); OPTIONAL(scales, 4);
  TRY_STATUS(both("codes and scales", codes, scales));
  REQUIRE(w_codes, 16); REQUIRE(w_scales, 4); OPTIONAL(b, 4); REQUIRE_ROWS(z, elem(desc));
  OPTIONAL(desc->add_out, elem(desc));
  if (!desc->M) return CONVBN_OK;
  const bool few = qfew_taken(desc->M, desc->N, desc->K), packs = few && x && qfew_packs(desc->M, desc->N, desc->K);
  if (!packs) TRY_STATUS(check_ws(codes ? mul_ws(desc) : fwd_ws(desc), ws, ws_bytes));
  const hipStream_t st = (hipStream_t)stream;
  QMul m = {};
  m.M = desc->M; m.ldz = ldz; m.K = desc->K; m.N = desc->N; m.dtype = desc->dtype;
  m.qw = w_codes; m.sw = w_scales; m.b = b; m.z = z;
  m.add = (desc->act & CONVBN_ACT_ADD_OUT) ? desc->add_out : nullptr;
  if (packs) {
    LAUNCH(launch_qfew(m, x, ldx, codes, scales, st));
    return CONVBN_OK;
  }
  if (!codes) {
    codes = static_cast<char*>(ws) + mul_ws(desc);
    scales = reinterpret_cast<float*>(static_cast<char*>(codes) + codes_ws(desc));
  }
  m.qx = codes; m.sx = scales;
  if (x) LAUNCH(launch_qpack(desc->dtype, desc->M, desc->K, ldx, x, codes, scales, st));
  if (few) LAUNCH(launch_qfew(m, nullptr, 0, nullptr, nullptr, st));
  else LAUNCH(launch_qmul(m, ws, st));
  return CONVBN_OK;
}

convbn_status convbn_qlinear_bwd(const convbn_qdesc* desc, const void* codes, const float* scales, const void* w_codes,
                                 const float* w_scales, const void* dz, void* dx, void* dW, float* db, void* ws, size_t ws_bytes,
                                 void* stream) {
  i64 ldx, ldz;
  TRY_STATUS(check_linear(desc, &ldx, &ldz));
  REQUIRE_ROWS(dz, qgrad_reads_in_place(desc->dtype, desc->N, ldz) && (dx || dW) ? 16 : elem(desc));
  OPTIONAL(dx, elem(desc)); OPTIONAL(dW, elem(desc)); OPTIONAL(db, 4);
  if (!dx && !dW && !db && desc->M) return set_error(CONVBN_ERR_NULL, "no output is asked for");
  if (dW) { REQUIRE_ROWS(codes, 16); REQUIRE_ROWS(scales, 4); }
  if (dx) { REQUIRE(w_codes, 16); REQUIRE(w_scales, 4); }
  OPTIONAL(desc->add_in, elem(desc));
  QGrad g = grad_of(desc, ldx, ldz);
  g.qx = codes; g.sx = scales; g.qw = w_codes; g.sw = w_scales; g.dz = dz; g.dx = dx; g.dW = dW; g.db = db;
  TRY_STATUS(check_ws(qgrad_scratch(g), ws, ws_bytes));
  LAUNCH(launch_qgrad(g, ws, (hipStream_t)stream));
  return CONVBN_OK;
}

convbn_status convbn_qgate_fwd(const convbn_qdesc* desc, const void* h, void* h_codes, float* h_scales, void* y, void* y_codes,
                               float* y_scales, void* stream) {
  i64 ldh, ldy;
  TRY_STATUS(check_gate(desc, &ldh, &ldy));
  REQUIRE_ROWS(h, elem(desc));
  OPTIONAL(h_codes, 16); OPTIONAL(h_scales, 4); OPTIONAL(y, elem(desc)); OPTIONAL(y_codes, 16); OPTIONAL(y_scales, 4);
  TRY_STATUS(both("h_codes and h_scales", h_codes, h_scales));
  TRY_STATUS(both("y_codes and y_scales", y_codes, y_scales));
  if (!y && !y_codes && desc->M) return set_error(CONVBN_ERR_NULL, "no output is asked for");
  LAUNCH(launch_qgate_fwd(desc->dtype, desc->gate, desc->M, desc->K, ldh, ldy, h, h_codes, h_scales, y, y_codes, y_scales,
                          (hipStream_t)stream));
  return CONVBN_OK;
}

convbn_status convbn_qgate_bwd(const convbn_qdesc* desc, const void* h_codes, const float* h_scales, const void* dy, void* dh,
                               void* stream) {
  i64 ldh, ldy;
  TRY_STATUS(check_gate(desc, &ldh, &ldy));
  REQUIRE_ROWS(h_codes, 16); REQUIRE_ROWS(h_scales, 4); REQUIRE_ROWS(dy, elem(desc)); REQUIRE_ROWS(dh, elem(desc));
  LAUNCH(launch_qgate_bwd(desc->dtype, desc->gate, desc->M, desc->K, ldh, ldy, h_codes, h_scales, dy, dh, (hipStream_t)stream));
  return CONVBN_OK;
}

}  // extern "C"
