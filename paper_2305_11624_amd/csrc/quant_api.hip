// C ABI of the 8-bit rows: argument checks, workspace and launch sequences.  Host code only enqueues.
#include "quant.h"

using namespace convbn;

namespace {

constexpr int32_t MAX_SUM = 131072;   // products of two codes stay below 2^14: that many of them fit 32 bits
constexpr int32_t MAX_OUT = 1 << 20;

bool misaligned(const void* p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }

#define TRY_STATUS(expr)                     \
  do {                                       \
    const convbn_status s_ = (expr);         \
    if (s_ != CONVBN_OK) return s_;          \
  } while (0)
#define LAUNCH(expr)                                                                                   \
  do {                                                                                                 \
    const hipError_t e_ = (expr);                                                                      \
    if (e_ != hipSuccess) return set_error(CONVBN_ERR_LAUNCH, "%s: %s", #expr, hipGetErrorString(e_)); \
  } while (0)

convbn_status pointer(const char* name, const void* p, uintptr_t align, bool required) {
  if (!p) return required ? set_error(CONVBN_ERR_NULL, "required pointer '%s' is NULL", name) : CONVBN_OK;
  if (misaligned(p, align)) return set_error(CONVBN_ERR_UNSUPPORTED, "pointer '%s' is not %d-byte aligned", name, (int)align);
  return CONVBN_OK;
}
#define REQUIRE(p, align) TRY_STATUS(pointer(#p, p, align, true))
#define OPTIONAL(p, align) TRY_STATUS(pointer(#p, p, align, false))
#define REQUIRE_ROWS(p, align) TRY_STATUS(pointer(#p, p, align, desc->M > 0))   // (no rows: there may be no memory either)

convbn_status both(const char* names, const void* a, const void* b) {
  if (!a != !b) return set_error(CONVBN_ERR_NULL, "%s are given together or not at all", names);
  return CONVBN_OK;
}

uintptr_t elem(const convbn_qdesc* d) { return d->dtype == CONVBN_BF16 ? 2 : 4; }

// What every call asks of its descriptor; wx, wz: channels of a row that is ldx / ldz apart (0 = the call has none).
convbn_status check(const convbn_qdesc* d, i64 wx, i64 wz, i64* ldx, i64* ldz) {
  const i64 lim = 1LL << 30;
  if (d->M < 0 || d->K < 1) return set_error(CONVBN_ERR_SHAPE, "M must be >= 0 and K >= 1");
  if (d->dtype != CONVBN_F32 && d->dtype != CONVBN_BF16)
    return set_error(CONVBN_ERR_UNSUPPORTED, "dtype %d is not CONVBN_F32 or CONVBN_BF16", d->dtype);
  if (d->reserved) return set_error(CONVBN_ERR_UNSUPPORTED, "reserved must be 0");
  if (d->M > lim || wx > lim || wz > lim)
    return set_error(CONVBN_ERR_UNSUPPORTED, "more than 2^30 rows or channels");
  *ldx = d->ldx ? d->ldx : wx;
  *ldz = d->ldz ? d->ldz : wz;
  if ((wx && *ldx < wx) || (wz && *ldz < wz)) return set_error(CONVBN_ERR_SHAPE, "ldx or ldz is shorter than a row");
  if (*ldx > (1LL << 40) || *ldz > (1LL << 40)) return set_error(CONVBN_ERR_UNSUPPORTED, "ldx or ldz is longer than 2^40");
  return CONVBN_OK;
}

convbn_status check_linear(const convbn_qdesc* d, i64* ldx, i64* ldz) {
  if (!d) return set_error(CONVBN_ERR_NULL, "descriptor is NULL");
  if (d->N < 1) return set_error(CONVBN_ERR_SHAPE, "N must be >= 1");
  TRY_STATUS(check(d, d->K, d->N, ldx, ldz));
  if (d->K > MAX_SUM) return set_error(CONVBN_ERR_UNSUPPORTED, "a sum over more than %d channels", (int)MAX_SUM);
  if (d->N > MAX_OUT) return set_error(CONVBN_ERR_UNSUPPORTED, "more than %d output channels", (int)MAX_OUT);
  const i64 most = 1LL << 38;   // (more than the card holds; tile counts stay far below 2^31)
  if (d->M * d->N > most || d->M * d->K > most) return set_error(CONVBN_ERR_UNSUPPORTED, "a tensor of more than 2^38 elements");
  if (d->act & ~(CONVBN_ACT_ADD_OUT | CONVBN_ACT_ADD_IN))
    return set_error(CONVBN_ERR_UNSUPPORTED, "act %d: only the two addends", d->act);
  if (d->M && (((d->act & CONVBN_ACT_ADD_OUT) && !d->add_out) || ((d->act & CONVBN_ACT_ADD_IN) && !d->add_in)))
    return set_error(CONVBN_ERR_NULL, "act %d asks for an addend that the descriptor does not give", d->act);
  return CONVBN_OK;
}
convbn_status check_rows(const convbn_qdesc* d, i64* ldx) {
  i64 ldz;
  if (!d) return set_error(CONVBN_ERR_NULL, "descriptor is NULL");
  return check(d, d->K, 0, ldx, &ldz);
}
convbn_status check_gate(const convbn_qdesc* d, i64* ldh, i64* ldy) {
  if (!d) return set_error(CONVBN_ERR_NULL, "descriptor is NULL");
  TRY_STATUS(check(d, 2 * (i64)d->K, d->K, ldh, ldy));
  if (d->gate != CONVBN_GATE_SILU && d->gate != CONVBN_GATE_GELU) return set_error(CONVBN_ERR_UNSUPPORTED, "gate %d is unknown", d->gate);
  return CONVBN_OK;
}

convbn_status check_ws(size_t need, void* ws, size_t ws_bytes) {
  if (need == 0) return CONVBN_OK;
  if (!ws) return set_error(CONVBN_ERR_WORKSPACE, "workspace is NULL but %zu bytes are needed", need);
  if (misaligned(ws, 16)) return set_error(CONVBN_ERR_UNSUPPORTED, "workspace is not 16-byte aligned");
  if (ws_bytes < need) return set_error(CONVBN_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", ws_bytes, need);
  return CONVBN_OK;
}

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
