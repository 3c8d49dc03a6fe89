// C ABI of the 8-bit floating-point rows, the gated product and group norm: argument checks, workspace and launch sequences.  Host code only
// enqueues.
#include <math.h>

#include "head.h"
#include "row_checks.h"

using namespace convbn;

namespace {

// ---- 8-bit floating point ----
F8Grad grad_of(const convbn_qdesc* d, i64 ldx, i64 ldz) {
  F8Grad g = {};
  g.M = d->M; g.ldx = ldx; g.ldz = ldz; g.K = d->K; g.N = d->N; g.dtype = d->dtype;
  g.add = (d->act & CONVBN_ACT_ADD_IN) ? d->add_in : nullptr;
  return g;
}
// Forward workspace: the product's, then codes and scales that the call does not hand out
size_t mul_ws(const convbn_qdesc* d) { return f8few_taken(d->M, d->K) ? 0 : f8mul_scratch(d->M, d->N, d->K); }
size_t codes_ws(const convbn_qdesc* d) { return align_up((size_t)d->M * qrow(d->K), 256); }
size_t fwd_ws(const convbn_qdesc* d) { return f8few_taken(d->M, d->K) ? 0 : mul_ws(d) + codes_ws(d) + align_up((size_t)d->M * f8srow(d->K), 256); }

// ---- gated product ----
convbn_status check_glu(const convbn_qdesc* d, Glu* g) {
  TRY_STATUS(check_linear(d, &g->ldx, &g->ldz, CONVBN_ACT_H_KEPT));
  if (d->act & ~(CONVBN_ACT_ADD_IN | CONVBN_ACT_H_KEPT))
    return set_error(CONVBN_ERR_UNSUPPORTED, "act %d: only CONVBN_ACT_ADD_IN and CONVBN_ACT_H_KEPT", d->act);
  if (d->gate != CONVBN_GATE_SILU && d->gate != CONVBN_GATE_GELU) return set_error(CONVBN_ERR_UNSUPPORTED, "gate %d is unknown", d->gate);
  g->M = d->M; g->K = d->K; g->N = d->N; g->dtype = d->dtype; g->gate = d->gate;
  g->add = (d->act & CONVBN_ACT_ADD_IN) ? d->add_in : nullptr;
  g->kept = d->act & CONVBN_ACT_H_KEPT;
  return CONVBN_OK;
}

// ---- group norm ----
convbn_status check_norm(const convbn_norm_desc* d, Norm* n) {
  if (!d) return set_error(CONVBN_ERR_NULL, "descriptor is NULL");
  if (d->M < 0 || d->P < 1 || d->C < 1 || d->groups < 1 || d->C % d->groups)
    return set_error(CONVBN_ERR_SHAPE, "M must be >= 0, P, C and groups >= 1, and C a multiple of groups");
  if (d->dtype != CONVBN_F32 && d->dtype != CONVBN_BF16)
    return set_error(CONVBN_ERR_UNSUPPORTED, "dtype %d is not CONVBN_F32 or CONVBN_BF16", d->dtype);
  if (d->f < CONVBN_NORM_NONE || d->f > CONVBN_NORM_GELU) return set_error(CONVBN_ERR_UNSUPPORTED, "activation %d is unknown", d->f);
  if (!(d->eps > 0.f) || !isfinite(d->eps)) return set_error(CONVBN_ERR_SHAPE, "eps must be above 0 and finite");
  if (d->reserved) return set_error(CONVBN_ERR_UNSUPPORTED, "reserved must be 0");
  if (d->act & ~CONVBN_ACT_ADD_IN) return set_error(CONVBN_ERR_UNSUPPORTED, "act %d: only CONVBN_ACT_ADD_IN", d->act);
  if (d->C > MAX_OUT) return set_error(CONVBN_ERR_UNSUPPORTED, "more than %d channels", (int)MAX_OUT);
  const i64 lim = 1LL << 30;
  if (d->M > lim || d->P > lim || d->M * d->P > lim) return set_error(CONVBN_ERR_UNSUPPORTED, "more than 2^30 pixels");
  if (d->M * d->groups > lim) return set_error(CONVBN_ERR_UNSUPPORTED, "more than 2^30 groups of all images");
  if (d->M * d->P * d->C > 1LL << 38) return set_error(CONVBN_ERR_UNSUPPORTED, "a tensor of more than 2^38 elements");
  n->ldx = d->ldx ? d->ldx : d->C;
  n->ldy = d->ldy ? d->ldy : d->C;
  if (n->ldx < d->C || n->ldy < d->C) return set_error(CONVBN_ERR_SHAPE, "ldx or ldy is shorter than a pixel");
  if (n->ldx > (1LL << 32) || n->ldy > (1LL << 32)) return set_error(CONVBN_ERR_UNSUPPORTED, "ldx or ldy is longer than 2^32");
  if (d->M && (d->act & CONVBN_ACT_ADD_IN) && !d->add_in)
    return set_error(CONVBN_ERR_NULL, "act %d asks for an addend that the descriptor does not give", d->act);
  n->M = d->M; n->P = d->P; n->C = d->C; n->groups = d->groups; n->dtype = d->dtype; n->f = d->f; n->eps = d->eps;
  n->add = (d->act & CONVBN_ACT_ADD_IN) ? d->add_in : nullptr;
  return CONVBN_OK;
}

// The rows that a kernel reads while others of its workgroups write theirs
convbn_status apart(const char* names, const void* out, const void* in) {
  return out == in ? set_error(CONVBN_ERR_UNSUPPORTED, "%s: other workgroups read what this output overwrites", names) : CONVBN_OK;
}

}  // namespace

extern "C" {

size_t convbn_fscale_bytes(int32_t channels) { return channels < 1 || channels > 1 << 30 ? 0 : (size_t)f8srow(channels); }

convbn_status convbn_fpack(const convbn_qdesc* desc, const void* x, void* codes, void* scales, void* stream) {
  i64 ld;
  TRY_STATUS(check_rows(desc, &ld));
  REQUIRE_ROWS(x, elem(desc)); REQUIRE_ROWS(codes, 16); REQUIRE_ROWS(scales, 4);
  LAUNCH(launch_f8_pack(desc->dtype, desc->M, desc->K, ld, x, codes, scales, (hipStream_t)stream));
  return CONVBN_OK;
}

convbn_status convbn_funpack(const convbn_qdesc* desc, const void* codes, const void* scales, void* x, void* stream) {
  i64 ld;
  TRY_STATUS(check_rows(desc, &ld));
  REQUIRE_ROWS(codes, 16); REQUIRE_ROWS(scales, 4); REQUIRE_ROWS(x, elem(desc));
  LAUNCH(launch_f8_unpack(desc->dtype, desc->M, desc->K, ld, codes, scales, x, (hipStream_t)stream));
  return CONVBN_OK;
}

size_t convbn_flinear_workspace_bytes(const convbn_qdesc* desc, int pass) {
  i64 ldx, ldz;
  if (check_linear(desc, &ldx, &ldz) != CONVBN_OK) return 0;
  return pass == CONVBN_PASS_FWD ? fwd_ws(desc) : f8grad_scratch(grad_of(desc, ldx, ldz));
}

convbn_status convbn_flinear_fwd(const convbn_qdesc* desc, const void* x, void* codes, void* scales, const void* w_codes,
                                  const void* w_scales, const float* b, void* z, void* ws, size_t ws_bytes, void* stream) {
  i64 ldx, ldz;
  TRY_STATUS(check_linear(desc, &ldx, &ldz));
  OPTIONAL(x, elem(desc));
  if (!x) { REQUIRE_ROWS(codes, 16); REQUIRE_ROWS(scales, 4); }
  OPTIONAL(codes, 16); OPTIONAL(scales, 4);
  TRY_STATUS(both("codes and scales", codes, scales));
  REQUIRE(w_codes, 16); REQUIRE(w_scales, 4); OPTIONAL(b, 4); REQUIRE_ROWS(z, elem(desc));
  OPTIONAL(desc->add_out, elem(desc));
  if (!desc->M) return CONVBN_OK;
  TRY_STATUS(check_ws(codes ? mul_ws(desc) : fwd_ws(desc), ws, ws_bytes));
  TRY_STATUS(apart("z is x", z, x));
  const hipStream_t st = (hipStream_t)stream;
  F8Mul m = {};
  m.M = desc->M; m.ldz = ldz; m.K = desc->K; m.N = desc->N; m.dtype = desc->dtype;
  m.qw = (const uint8_t*)w_codes; m.sw = (const uint8_t*)w_scales; m.b = b; m.z = z;
  m.add = (desc->act & CONVBN_ACT_ADD_OUT) ? desc->add_out : nullptr;
  if (f8few_taken(desc->M, desc->K)) {
    m.qx = (const uint8_t*)codes; m.sx = (const uint8_t*)scales;
    LAUNCH(launch_f8few(m, x, ldx, codes, scales, st));
    return CONVBN_OK;
  }
  if (!codes) {
    codes = static_cast<char*>(ws) + mul_ws(desc);
    scales = static_cast<char*>(codes) + codes_ws(desc);
  }
  m.qx = (const uint8_t*)codes; m.sx = (const uint8_t*)scales;
  if (x) LAUNCH(launch_f8_pack(desc->dtype, desc->M, desc->K, ldx, x, codes, scales, st));
  LAUNCH(launch_f8mul(m, ws, st));
  return CONVBN_OK;
}

convbn_status convbn_flinear_bwd(const convbn_qdesc* desc, const void* codes, const void* scales, const void* w_codes,
                                  const void* w_scales, const void* dz, void* dx, void* dW, float* db, void* ws, size_t ws_bytes,
                                  void* stream) {
  i64 ldx, ldz;
  TRY_STATUS(check_linear(desc, &ldx, &ldz));
  REQUIRE_ROWS(dz, qgrad_reads_in_place(desc->dtype, desc->N, ldz) && (dx || dW) ? 16 : elem(desc));
  OPTIONAL(dx, elem(desc)); OPTIONAL(dW, elem(desc)); OPTIONAL(db, 4);
  if (!dx && !dW && !db && desc->M) return set_error(CONVBN_ERR_NULL, "no output is asked for");
  if (dW) { REQUIRE_ROWS(codes, 16); REQUIRE_ROWS(scales, 4); }
  if (dx) { REQUIRE(w_codes, 16); REQUIRE(w_scales, 4); }
  OPTIONAL(desc->add_in, elem(desc));
  F8Grad g = grad_of(desc, ldx, ldz);
  g.qx = (const uint8_t*)codes; g.sx = (const uint8_t*)scales; g.qw = (const uint8_t*)w_codes; g.sw = (const uint8_t*)w_scales;
  g.dz = dz; g.dx = dx; g.dW = dW; g.db = db;
  TRY_STATUS(check_ws(f8grad_scratch(g), ws, ws_bytes));
  if (dx && desc->M) TRY_STATUS(apart("dx is dz", dx, dz));
  LAUNCH(launch_f8grad(g, ws, (hipStream_t)stream));
  return CONVBN_OK;
}

size_t convbn_glu_workspace_bytes(const convbn_qdesc* desc, int pass) {
  Glu g = {};
  return check_glu(desc, &g) == CONVBN_OK ? glu_scratch(g, pass) : 0;
}

convbn_status convbn_glu_fwd(const convbn_qdesc* desc, const void* x, const void* W, const float* b, void* y, float* h, void* ws,
                             size_t ws_bytes, void* stream) {
  Glu g = {};
  TRY_STATUS(check_glu(desc, &g));
  REQUIRE_ROWS(x, glu_in_place(g.dtype, g.K, g.ldx) ? 16 : elem(desc));
  REQUIRE(W, glu_in_place(g.dtype, g.K, g.K) ? 16 : elem(desc));
  OPTIONAL(b, 4); REQUIRE_ROWS(y, elem(desc)); OPTIONAL(h, 4);
  if (!desc->M) return CONVBN_OK;
  TRY_STATUS(check_ws(glu_scratch(g, CONVBN_PASS_FWD), ws, ws_bytes));
  TRY_STATUS(apart("y is x", y, x));
  g.x = x; g.W = W; g.b = b; g.y = y; g.h = h;
  LAUNCH(launch_glu_fwd(g, ws, (hipStream_t)stream));
  return CONVBN_OK;
}

convbn_status convbn_glu_bwd(const convbn_qdesc* desc, const void* x, const void* W, const float* b, const float* h, const void* dy,
                             void* dx, void* dW, float* db, void* ws, size_t ws_bytes, void* stream) {
  Glu g = {};
  TRY_STATUS(check_glu(desc, &g));
  REQUIRE_ROWS(x, glu_in_place(g.dtype, g.K, g.ldx) ? 16 : elem(desc));
  REQUIRE(W, glu_in_place(g.dtype, g.K, g.K) ? 16 : elem(desc));
  OPTIONAL(b, 4); REQUIRE_ROWS(dy, elem(desc));
  if (g.kept) REQUIRE_ROWS(h, 4);
  OPTIONAL(h, 4);
  OPTIONAL(dx, elem(desc)); OPTIONAL(dW, elem(desc)); OPTIONAL(db, 4);
  if (!dx && !dW && !db && desc->M) return set_error(CONVBN_ERR_NULL, "no output is asked for");
  OPTIONAL(desc->add_in, elem(desc));
  TRY_STATUS(check_ws(glu_scratch(g, CONVBN_PASS_BWD), ws, ws_bytes));
  if (dx && desc->M) TRY_STATUS(apart("dx is x", dx, x));
  g.x = x; g.W = W; g.b = b; g.hk = h; g.dy = dy; g.dx = dx; g.dW = dW; g.db = db;
  LAUNCH(launch_glu_bwd(g, ws, (hipStream_t)stream));
  return CONVBN_OK;
}

size_t convbn_norm_workspace_bytes(const convbn_norm_desc* desc, int pass) {
  Norm n = {};
  return check_norm(desc, &n) == CONVBN_OK ? norm_scratch(n, pass) : 0;
}

convbn_status convbn_norm_fwd(const convbn_norm_desc* desc, const void* x, const float* gamma, const float* beta, void* y, float* stats,
                              void* ws, size_t ws_bytes, void* stream) {
  Norm n = {};
  TRY_STATUS(check_norm(desc, &n));
  const uintptr_t elem = n.dtype == CONVBN_BF16 ? 2 : 4;
  REQUIRE_ROWS(x, elem); OPTIONAL(gamma, 4); OPTIONAL(beta, 4); REQUIRE_ROWS(y, elem); OPTIONAL(stats, 4);
  if (!n.M) return CONVBN_OK;
  TRY_STATUS(apart("y is x", y, x));
  TRY_STATUS(check_ws(norm_scratch(n, CONVBN_PASS_FWD), ws, ws_bytes));
  n.x = x; n.gamma = gamma; n.beta = beta; n.y = y; n.stats = stats;
  LAUNCH(launch_norm_fwd(n, ws, (hipStream_t)stream));
  return CONVBN_OK;
}

convbn_status convbn_norm_bwd(const convbn_norm_desc* desc, const void* x, const float* gamma, const float* beta, const float* stats,
                              const void* dy, void* dx, float* dgamma, float* dbeta, void* ws, size_t ws_bytes, void* stream) {
  Norm n = {};
  TRY_STATUS(check_norm(desc, &n));
  const uintptr_t elem = n.dtype == CONVBN_BF16 ? 2 : 4;
  REQUIRE_ROWS(x, elem); OPTIONAL(gamma, 4); OPTIONAL(beta, 4); REQUIRE_ROWS(stats, 4); REQUIRE_ROWS(dy, elem);
  OPTIONAL(dx, elem); OPTIONAL(dgamma, 4); OPTIONAL(dbeta, 4);
  if (!dx && !dgamma && !dbeta && desc->M) return set_error(CONVBN_ERR_NULL, "no output is asked for");
  OPTIONAL(desc->add_in, elem);
  TRY_STATUS(check_ws(norm_scratch(n, CONVBN_PASS_BWD), ws, ws_bytes));
  n.x = x; n.gamma = gamma; n.beta = beta; n.stats = const_cast<float*>(stats); n.dy = dy; n.dx = dx; n.dgamma = dgamma; n.dbeta = dbeta;
  LAUNCH(launch_norm_bwd(n, ws, (hipStream_t)stream));
  return CONVBN_OK;
}

}  // extern "C"
