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

// f(g) and f'(g), for rows of T
template <typename T, int KIND> __device__ __forceinline__ void gate_of(float g, float* f, float* df) {
  if constexpr (KIND == CONVBN_GATE_SILU && sizeof(T) == 4) {
    // p = 1 / (1 + e^-g) and 1 - p from e^-|g|, which neither overflows nor cancels: a few ulp each at either sign
    const float e = expf(-fabsf(g)), r = __builtin_amdgcn_rcpf(1.f + e), er = e * r;   // (1 ulp, between 1 and 2)
    const float p = g < 0.f ? er : r, q = g < 0.f ? r : er;
    *f = g * p;
    *df = p * (1.f + g * q);
  } else if constexpr (KIND == CONVBN_GATE_SILU) {
    // (the hardware's 2^x and reciprocal, 1 ulp each, and an exponent that is rounded: p is right to 2^-23 (1 + |g|), 2^-16 where it is smallest,
    // far inside the 2^-9 of the result)
    const float p = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(g * -1.44269504088896341f));
    *f = g * p;
    *df = p * (1.f + g * (1.f - p));
  } else {
    // The distribution's tail beyond |g| is e^(-g^2 / 2) times a smooth function, here t Q(t) with t = 1 / (1 + 0.27 |g|) and Q the polynomial of
    // degree 8 with the least relative error for |g| <= 16 (2.4e-8; a weighted least-squares fit in 64 bits): right to (17 + 1.5 g^2) 2^-24
    // at either sign, where 1 + erf(g / sqrt 2) cancels for negative g (a tenth at -5).  f and f' share the exponential.
    const float a = fabsf(g), t = __builtin_amdgcn_rcpf(fmaf(0.27f, a, 1.f)), e = __builtin_amdgcn_exp2f(a * a * -0.72134752044448170f);
    float Q = 0.0290384758f;
    Q = fmaf(Q, t, -0.126874059f);
    Q = fmaf(Q, t, 0.170616165f);
    Q = fmaf(Q, t, -0.0701961815f);
    Q = fmaf(Q, t, 0.108534291f);
    Q = fmaf(Q, t, 0.0717343763f);
    Q = fmaf(Q, t, 0.101895072f);
    Q = fmaf(Q, t, 0.107530445f);
    Q = fmaf(Q, t, 0.107721426f);
    const float tail = t * Q * e, p = g < 0.f ? tail : 1.f - tail;
    *f = g * p;
    *df = p + g * e * 0.39894228040143268f;
  }
}

// ---- bf16 operands whose rows lie across the reduced index: LDS, transposing loads, fp32 numbers in parts ----
typedef short s16x4 __attribute__((ext_vector_type(4)));

// 64-byte pieces of a row of W channels in LDS are exchanged by the row's low bits, so that the pieces of four rows that half a wave reads
// with the transposing load lie on distinct banks
template <int W> __device__ __forceinline__ int turn(int r) { return W >= 128 ? r & 3 : (r >> 1) & 1; }

__device__ __forceinline__ bf16x8 read_tr8(const unsigned char* p, int rows4) {   // 8 rows of this lane's column; rows4: bytes of 4 rows
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p));
  const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p + rows4));
  typedef short s16x8 __attribute__((ext_vector_type(8)));
  return __builtin_bit_cast(bf16x8, (s16x8){a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]});
}

// v in three parts of 8 bits each, which add up to it; infinities and NaN are the first whole
__device__ __forceinline__ void split3(const F8& f, F8 (&part)[3]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float v = f.v[e];
    const bool whole = (__float_as_uint(v) & INF) == INF;
#pragma unroll
    for (int i = 0; i < 3; ++i) {   // the 8 leading bits, what is left of it, and the rest of that: each exact
      const float t = whole ? (i ? 0.f : v) : __uint_as_float(__float_as_uint(v) & 0xffff0000u);
      part[i].v[e] = t;
      v -= t;
    }
  }
}

// ... for products of two such numbers, of whose pairs of parts the last three are left out.  The first two parts are rounded to nearest: of numbers in [1, 2) the others
// are at most 2^-8 and 2^-17, and what is left out of a product is at most 2^-24 of it, of either sign (leading bits would leave out 2^-21, always towards zero).
// The fourth is the first once more, zero in place of infinities and NaN: lower parts meet it, whose zeros would make NaN of an infinity.
struct Parts4 { u32x4 p[4]; };   // eight bf16 numbers each
__device__ __forceinline__ Parts4 split3_near(const F8& f) {
  constexpr float MOST = 0x1.fep127f;   // bf16's largest number
  Parts4 o;
  float sum = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) sum += fabsf(f.v[e]);
  const bool plain = sum <= MOST;   // (no infinity, no NaN, nothing that is rounded to an infinity)
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float v[2] = {f.v[2 * e], f.v[2 * e + 1]};
#pragma unroll
    for (int i = 0; i < 3; ++i) {   // (each difference is exact, and the last a bf16 number)
      o.p[i][e] = pack_bf16x2(v[0], v[1]);
      v[0] -= bf16_lo(o.p[i][e]);
      v[1] -= bf16_hi(o.p[i][e]);
    }
  }
  o.p[3] = o.p[0];
  if (!plain) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float v = f.v[e];
      const bool whole = (__float_as_uint(v) & INF) == INF;
      unsigned t[4];
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        const unsigned near = pack_bf16x2(fminf(fmaxf(v, -MOST), MOST), 0.f) & 0xffffu;
        t[i] = !whole ? near : i ? 0u : pack_bf16x2(f.v[e], 0.f) & 0xffffu;
        v -= bf16_lo(near);
        if (i == 0) t[3] = whole ? 0u : near;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) o.p[i][e / 2] = e & 1 ? (o.p[i][e / 2] & 0xffffu) | t[i] << 16 : (o.p[i][e / 2] & 0xffff0000u) | t[i];
    }
  }
  return o;
}

}  // namespace convbn
