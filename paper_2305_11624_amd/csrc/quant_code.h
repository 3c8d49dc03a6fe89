// A row's scale and codes, and eight channels of a row at a time: device code shared by the kernels that pack.
#pragma once
#include "quant.h"

namespace convbn {

constexpr float TINY = 1.504632769e-36f;   // 2^-119: below, 127 / a and a / 127 leave the normal range; the row counts as zeros
constexpr unsigned ABS = 0x7fffffffu, INF = 0x7f800000u;

struct F8 { float v[8]; };

template <typename T> struct Raw8;
template <> struct Raw8<bf16_t> { uint4 a; };
template <> struct Raw8<float> { uint4 a, b; };

__device__ __forceinline__ F8 widen(const Raw8<bf16_t>& r) {
  return {{bf16_lo(r.a.x), bf16_hi(r.a.x), bf16_lo(r.a.y), bf16_hi(r.a.y), bf16_lo(r.a.z), bf16_hi(r.a.z), bf16_lo(r.a.w), bf16_hi(r.a.w)}};
}
__device__ __forceinline__ F8 widen(const Raw8<float>& r) {
  return {{__uint_as_float(r.a.x), __uint_as_float(r.a.y), __uint_as_float(r.a.z), __uint_as_float(r.a.w), __uint_as_float(r.b.x),
           __uint_as_float(r.b.y), __uint_as_float(r.b.z), __uint_as_float(r.b.w)}};
}

// Channels k .. k+7 of a row of K (zeros past the end).  AL: every row starts on 16 bytes.
template <typename T, bool AL> __device__ __forceinline__ F8 load8(const T* __restrict__ row, int k, int K) {
  if (AL && k + 8 <= K) {
    const Raw8<T> r = *reinterpret_cast<const Raw8<T>*>(row + k);
    return widen(r);
  }
  F8 f;
#pragma unroll
  for (int i = 0; i < 8; ++i) f.v[i] = k + i < K ? to_f32(row[k + i]) : 0.f;
  return f;
}
template <typename T, bool AL> __device__ __forceinline__ void store8(T* __restrict__ row, int k, int K, const F8& f) {
  if (AL && k + 8 <= K) {
    if constexpr (sizeof(T) == 2) {
      *reinterpret_cast<uint4*>(row + k) = make_uint4(pack_bf16x2(f.v[0], f.v[1]), pack_bf16x2(f.v[2], f.v[3]),
                                                      pack_bf16x2(f.v[4], f.v[5]), pack_bf16x2(f.v[6], f.v[7]));
    } else {
      float4* p = reinterpret_cast<float4*>(row + k);
      p[0] = make_float4(f.v[0], f.v[1], f.v[2], f.v[3]);
      p[1] = make_float4(f.v[4], f.v[5], f.v[6], f.v[7]);
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (k + i < K) row[k + i] = from_f32<T>(f.v[i]);
}

__device__ __forceinline__ unsigned amax8(const F8& f) {   // (compared as whole numbers: a NaN is the largest of all)
  unsigned m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(f.v[i]) & ABS);
  return m;
}

// Scale and 127 / a of a row from its maximum's bits
struct Scale { float s, r; };
__device__ __forceinline__ Scale scale_of(unsigned bits) {
  if (bits >= INF) return {__uint_as_float(0x7fc00000u), 0.f};
  const float a = __uint_as_float(bits);
  if (a < TINY) return {0.f, 0.f};
  float s = a / 127.f;
  if (s * 127.f >= INFINITY) s = __uint_as_float(__float_as_uint(s) - 1);   // (rounded up at the very top: a row's maximum reads back finite)
  return {s, 127.f / a};
}

// 8 codes: adding 1.5 * 2^23 to |v| <= 127.0001 rounds it to a whole number, ties to even, and leaves it in the low byte.  The
// product is rounded before that (the definition): no fused multiply-add here.
__device__ __forceinline__ uint2 codes8(const F8& f, float r) {
#pragma clang fp contract(off)
  unsigned q[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float v = f.v[i] * r;
    q[i] = __float_as_uint(v + 12582912.f);
  }
  if (r == 0.f) return make_uint2(0, 0);
  auto four = [](unsigned a, unsigned b, unsigned c, unsigned d) {
    return (a & 255u) | (b & 255u) << 8 | (c & 255u) << 16 | d << 24;
  };
  return make_uint2(four(q[0], q[1], q[2], q[3]), four(q[4], q[5], q[6], q[7]));
}
__device__ __forceinline__ F8 decode8(uint2 c, float s) {
  F8 f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f.v[i] = (float)(int8_t)(c.x >> (8 * i)) * s;
    f.v[4 + i] = (float)(int8_t)(c.y >> (8 * i)) * s;
  }
  return f;
}


}  // namespace convbn
