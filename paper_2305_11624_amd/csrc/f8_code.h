// e4m3 codes and a block's power of two: device code shared by the kernels of the 8-bit floating-point rows.
#pragma once
#include "head.h"
#include "quant_code.h"

namespace convbn {

constexpr int E_MIN = -116, E_MAX = 120;   // (the smallest code is 2^-9: with e = -116 every value a code stands for is a normal number; a fp32
                                           // maximum never needs more than 120)

// The block's e from its maximum's bits: a = m 2^x <= 1.75 2^(e + 8)
__device__ __forceinline__ int f8_exp(unsigned bits) {
  const int e = (int)((bits + 0x1fffffu) >> 23) - 127 - 8;
  return bits >= INF ? 0 : max(e, E_MIN);
}
__device__ __forceinline__ float two_to(int e) { return __uint_as_float((unsigned)(e + 127) << 23); }
__device__ __forceinline__ float scale_of_byte(unsigned s) { return __uint_as_float(s << 23); }

// Eight codes of a block with maximum `bits`.  The product with a power of two is exact (below the normal range it is far below the smallest
// code); the conversion rounds to nearest, ties to even.  At E_MAX codes stay at 240: 256 2^120 is no fp32 number.
__device__ __forceinline__ uint2 f8_codes8(const F8& f, unsigned bits) {
  const int e = f8_exp(bits);
  const float r = two_to(-e), most = e == E_MAX ? 240.f : 448.f;
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = fminf(fmaxf(f.v[i] * r, -most), most);
  int a = 0, b = 0;
  a = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], a, false);
  a = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], a, true);
  b = __builtin_amdgcn_cvt_pk_fp8_f32(v[4], v[5], b, false);
  b = __builtin_amdgcn_cvt_pk_fp8_f32(v[6], v[7], b, true);
  if (bits >= INF) a = b = 0x7f7f7f7f;
  return make_uint2((unsigned)a, (unsigned)b);
}
__device__ __forceinline__ F8 f8_decode8(uint2 c, float s) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)c.x, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)c.x, true);
  const f32x2 d = __builtin_amdgcn_cvt_pk_f32_fp8((int)c.y, false), e = __builtin_amdgcn_cvt_pk_f32_fp8((int)c.y, true);
  return {{a[0] * s, a[1] * s, b[0] * s, b[1] * s, d[0] * s, d[1] * s, e[0] * s, e[1] * s}};
}
// the bytes of codes8 from channel k on that lie past K
__device__ __forceinline__ uint2 f8_clip(uint2 c, int k, int K) {
  const int n = K - k;
  if (n >= 8) return c;
  const uint64_t v = ((uint64_t)c.y << 32 | c.x) & (n <= 0 ? 0 : ~0ull >> (64 - 8 * n));
  return make_uint2((unsigned)v, (unsigned)(v >> 32));
}
// A maximum over the 16 lanes that hold a block
__device__ __forceinline__ unsigned block_max(unsigned m) {
#pragma unroll
  for (int off = 8; off > 0; off >>= 1) m = max(m, (unsigned)__shfl_xor((int)m, off, 64));
  return m;
}

}  // namespace convbn
