// Argument checks that the calls on rows share (8-bit rows, the gated product, group norm).  Host code only.
#pragma once
#include "quant.h"

namespace convbn {
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

convbn_status check_linear(const convbn_qdesc* d, i64* ldx, i64* ldz, int32_t more_acts = 0) {
  if (!d) return set_error(CONVBN_ERR_NULL, "descriptor is NULL");
  if (d->N < 1) return set_error(CONVBN_ERR_SHAPE, "N must be >= 1");
  TRY_STATUS(check(d, d->K, d->N, ldx, ldz));
  if (d->K > MAX_SUM) return set_error(CONVBN_ERR_UNSUPPORTED, "a sum over more than %d channels", (int)MAX_SUM);
  if (d->N > MAX_OUT) return set_error(CONVBN_ERR_UNSUPPORTED, "more than %d output channels", (int)MAX_OUT);
  const i64 most = 1LL << 38;   // (more than the card holds; tile counts stay far below 2^31)
  if (d->M * d->N > most || d->M * d->K > most) return set_error(CONVBN_ERR_UNSUPPORTED, "a tensor of more than 2^38 elements");
  if (d->act & ~(CONVBN_ACT_ADD_OUT | CONVBN_ACT_ADD_IN | more_acts))
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

}  // namespace
}  // namespace convbn
