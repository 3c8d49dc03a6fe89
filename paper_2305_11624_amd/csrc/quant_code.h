// A row's scale and codes, and eight channels of a row at a time: device code shared by the kernels that pack.
#pragma once
#include "quant.h"

namespace convbn {

constexpr float TINY = 1.504632769e-36f;   // 2^-119: below, 127 / a and a / 127 leave the normal range; the row counts as zeros
constexpr unsigned ABS = 0x7fffffffu, INF = 0x7f800000u;

struct F8 { float v[8]; };

// Eight channels of a row wherever it starts: one or two 16-byte accesses that need the alignment of an element only (the hardware takes
// any; rows of odd length cost little more than aligned ones)
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
template <typename T> struct Raw8;
template <> struct __attribute__((packed, aligned(2), may_alias)) Raw8<bf16_t> { u32x4 a; };
template <> struct __attribute__((packed, aligned(4), may_alias)) Raw8<float> { u32x4 a, b; };

__device__ __forceinline__ F8 widen(const Raw8<bf16_t>& r) {
  const u32x4 a = r.a;
  return {{bf16_lo(a[0]), bf16_hi(a[0]), bf16_lo(a[1]), bf16_hi(a[1]), bf16_lo(a[2]), bf16_hi(a[2]), bf16_lo(a[3]), bf16_hi(a[3])}};
}
__device__ __forceinline__ F8 widen(const Raw8<float>& r) {
  const u32x4 a = r.a, b = r.b;
  return {{__uint_as_float(a[0]), __uint_as_float(a[1]), __uint_as_float(a[2]), __uint_as_float(a[3]), __uint_as_float(b[0]),
           __uint_as_float(b[1]), __uint_as_float(b[2]), __uint_as_float(b[3])}};
}
template <typename T> __device__ __forceinline__ Raw8<T> narrow(const F8& f) {
  Raw8<T> r;
  if constexpr (sizeof(T) == 2) {
    r.a = (u32x4){pack_bf16x2(f.v[0], f.v[1]), pack_bf16x2(f.v[2], f.v[3]), pack_bf16x2(f.v[4], f.v[5]), pack_bf16x2(f.v[6], f.v[7])};
  } else {
    r.a = (u32x4){__float_as_uint(f.v[0]), __float_as_uint(f.v[1]), __float_as_uint(f.v[2]), __float_as_uint(f.v[3])};
    r.b = (u32x4){__float_as_uint(f.v[4]), __float_as_uint(f.v[5]), __float_as_uint(f.v[6]), __float_as_uint(f.v[7])};
  }
  return r;
}

// Channels k .. k+7 of a row of K (zeros past the end)
template <typename T> __device__ __forceinline__ F8 load8(const T* __restrict__ row, int k, int K) {
  if (k + 8 <= K) return widen(*reinterpret_cast<const Raw8<T>*>(row + k));
  F8 f;
#pragma unroll
  for (int i = 0; i < 8; ++i) f.v[i] = k + i < K ? to_f32(row[k + i]) : 0.f;
  return f;
}
// STREAM: past the L2 caches
template <typename T, bool STREAM = false> __device__ __forceinline__ void store8(T* __restrict__ row, int k, int K, const F8& f) {
  if (k + 8 <= K) {
    const Raw8<T> r = narrow<T>(f);
    if constexpr (STREAM) {
      typedef u32x4 __attribute__((aligned(2), may_alias)) Piece;
      __builtin_nontemporal_store(r.a, reinterpret_cast<Piece*>(row + k));
      if constexpr (sizeof(T) == 4) __builtin_nontemporal_store(r.b, reinterpret_cast<Piece*>(row + k + 4));
    } else {
      *reinterpret_cast<Raw8<T>*>(row + k) = r;
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (k + i < K) row[k + i] = from_f32<T>(f.v[i]);
}
// ... a product's result: the addend, if any, comes on top (it may be the same memory).  Results leave the caches to the operands.  us, kept there
// and streamed, up product, gate and down product forward and backward: 25088 x 512 -> 2 x 1024 484 and 458, 8192 x 4096 -> 2 x 8192 3913 and 3877, 1568 x
// 2048 -> 2 x 8192 517 and 498; forward alone, where the next kernel reads them at once, 1568 x 512 -> 2 x 2048 32.3 and 30.8, 1568 x 2048 -> 2 x
// 8192 133 and 135.
template <typename T> __device__ __forceinline__ void store8_plus(T* row, const T* add, int k, int K, F8 f) {
  if (add) {
    if (k + 8 <= K) {
      const F8 a = widen(*reinterpret_cast<const Raw8<T>*>(add + k));
#pragma unroll
      for (int i = 0; i < 8; ++i) f.v[i] += a.v[i];
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (k + i < K) f.v[i] += to_f32(add[k + i]);
    }
  }
  store8<T, true>(row, k, K, f);
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

// The order of sum * s_x * s_w.  The scales' own product can leave the range where the result does not (two rows below 2^-60, a mask's value against
// a large weight: zero sums became NaN), so the sum, a whole number below 2^31, meets one scale first: the row's, after which it is at least
// 2^-126 and, as long as that scale is at most 2^96, finite.  Above, the row's comes last: if the sum overflows with the other, the result does.
__device__ __forceinline__ bool scale_last(float sx) { return sx > 0x1p96f; }

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
