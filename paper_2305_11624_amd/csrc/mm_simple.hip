// The products of the 8-bit floating-point rows and of the gated block, plainly: tiles of 64 x 64 through LDS, fp32 multiply-adds.
#include "f8_code.h"

namespace convbn {

namespace {

constexpr int T = 64, RC = 16;

// C(i, j) = sum_r A(i, r) B(j, r), for one or two B; out(i, j, sums)
template <int NB, class A, class B, class OUT>
__global__ __launch_bounds__(256) void mm_kernel(i64 I, int J, i64 R, A a, B b, OUT out) {
  __shared__ float la[RC][T + 1], lb[NB][RC][T + 1];
  const int tid = threadIdx.x, ti = tid & 15, tj = tid >> 4, ntj = (J + T - 1) / T;
  const i64 i0 = (i64)(blockIdx.x / ntj) * T;
  const int j0 = (int)(blockIdx.x % ntj) * T;
  float acc[NB][4][4] = {};
  for (i64 r0 = 0; r0 < R; r0 += RC) {
    for (int x = tid; x < T * RC; x += 256) {
      const int r = x % RC, at = x / RC;
      la[r][at] = i0 + at < I && r0 + r < R ? a(i0 + at, r0 + r) : 0.f;
      for (int n = 0; n < NB; ++n) lb[n][r][at] = j0 + at < J && r0 + r < R ? b(n, j0 + at, r0 + r) : 0.f;
    }
    __syncthreads();
    for (int r = 0; r < RC; ++r)
      for (int n = 0; n < NB; ++n)
        for (int x = 0; x < 4; ++x)
          for (int y = 0; y < 4; ++y) acc[n][x][y] += la[r][ti + 16 * x] * lb[n][r][tj + 16 * y];
    __syncthreads();
  }
  for (int x = 0; x < 4; ++x)
    for (int y = 0; y < 4; ++y) {
      const i64 i = i0 + ti + 16 * x;
      const int j = j0 + tj + 16 * y;
      float v[NB];
      for (int n = 0; n < NB; ++n) v[n] = acc[n][x][y];
      if (i < I && j < J) out(i, j, v);
    }
}
template <int NB, class A, class B, class OUT> hipError_t mm(i64 I, int J, i64 R, A a, B b, OUT out, hipStream_t st) {
  if (!I || !J) return hipSuccess;
  mm_kernel<NB><<<(unsigned)((I + T - 1) / T * ((J + T - 1) / T)), 256, 0, st>>>(I, J, R, a, b, out);
  return hipGetLastError();
}
template <class V> __global__ void sums_kernel(i64 M, int N, V v, float* out) {
  const int n = blockIdx.x * 64 + threadIdx.x;
  if (n >= N) return;
  float s = 0.f;
  for (i64 m = 0; m < M; ++m) s += v(m, n);
  out[n] = s;
}

__device__ float f8_value(const uint8_t* q, const uint8_t* s, int Kp, int Sp, i64 row, i64 k) {
  return f8_decode8(make_uint2(q[row * Kp + k], 0), scale_of_byte(s[row * Sp + k / BLK])).v[0];
}

template <typename E> hipError_t f8mul_t(const F8Mul& p, hipStream_t st) {
  const int Kp = qrow(p.K), Sp = f8srow(p.K);
  return mm<1>(p.M, p.N, p.K, [=] __device__(i64 m, i64 k) { return f8_value(p.qx, p.sx, Kp, Sp, m, k); },
               [=] __device__(int, i64 n, i64 k) { return f8_value(p.qw, p.sw, Kp, Sp, n, k); },
               [=] __device__(i64 m, int n, const float* v) {
                 float z = v[0] + (p.b ? p.b[n] : 0.f);
                 if (p.add) z += to_f32(static_cast<const E*>(p.add)[m * p.ldz + n]);
                 static_cast<E*>(p.z)[m * p.ldz + n] = from_f32<E>(z);
               }, st);
}
template <typename E> hipError_t f8grad_t(const F8Grad& p, hipStream_t st) {
  const int Kp = qrow(p.K), Sp = f8srow(p.K);
  auto dz = [=] __device__(i64 m, i64 n) { return to_f32(static_cast<const E*>(p.dz)[m * p.ldz + n]); };
  hipError_t e = hipSuccess;
  if (p.dx)
    e = mm<1>(p.M, p.K, p.N, dz, [=] __device__(int, i64 k, i64 n) { return f8_value(p.qw, p.sw, Kp, Sp, n, k); },
              [=] __device__(i64 m, int k, const float* v) {
                float z = v[0];
                if (p.add) z += to_f32(static_cast<const E*>(p.add)[m * p.ldx + k]);
                static_cast<E*>(p.dx)[m * p.ldx + k] = from_f32<E>(z);
              }, st);
  if (p.dW && e == hipSuccess)
    e = mm<1>(p.N, p.K, p.M, [=] __device__(i64 n, i64 m) { return dz(m, n); },
              [=] __device__(int, i64 k, i64 m) { return f8_value(p.qx, p.sx, Kp, Sp, m, k); },
              [=] __device__(i64 n, int k, const float* v) { static_cast<E*>(p.dW)[n * p.K + k] = from_f32<E>(v[0]); }, st);
  if (p.db && e == hipSuccess) {
    sums_kernel<<<ceil_div(p.N, 64), 64, 0, st>>>(p.M, p.N, dz, p.db);
    e = hipGetLastError();
  }
  return e;
}

template <typename E, int KIND> hipError_t glu_fwd_t(const Glu& p, float* dh, hipStream_t st) {
  const int F = p.N;
  return mm<2>(p.M, F, p.K, [=] __device__(i64 m, i64 k) { return to_f32(static_cast<const E*>(p.x)[m * p.ldx + k]); },
               [=] __device__(int n, i64 j, i64 k) { return to_f32(static_cast<const E*>(p.W)[(j + (i64)n * F) * p.K + k]); },
               [=] __device__(i64 m, int j, const float* v) {
                 const float g = v[0] + (p.b ? p.b[j] : 0.f), u = v[1] + (p.b ? p.b[F + j] : 0.f);
                 float f, df;
                 gate_of<E, KIND>(g, &f, &df);
                 if (p.y) static_cast<E*>(p.y)[m * p.ldz + j] = from_f32<E>(f * u);
                 if (p.h) {
                   static_cast<E*>(p.h)[m * 2 * F + j] = from_f32<E>(g);
                   static_cast<E*>(p.h)[m * 2 * F + F + j] = from_f32<E>(u);
                 }
                 if (dh) {
                   const float dy = to_f32(static_cast<const E*>(p.dy)[m * p.ldz + j]);
                   dh[m * 2 * F + j] = dy * u * df;
                   dh[m * 2 * F + F + j] = dy * f;
                 }
               }, st);
}
template <typename E, int KIND> __global__ void dgate_kernel(Glu p, float* dh) {
  const int F = p.N;
  for (i64 x = (i64)blockIdx.x * 256 + threadIdx.x; x < p.M * F; x += (i64)gridDim.x * 256) {
    const i64 m = x / F;
    const int j = (int)(x - m * F);
    const E* h = static_cast<const E*>(p.hk) + m * 2 * F;
    float f, df;
    gate_of<E, KIND>(to_f32(h[j]), &f, &df);
    const float dy = to_f32(static_cast<const E*>(p.dy)[m * p.ldz + j]);
    dh[m * 2 * F + j] = dy * to_f32(h[F + j]) * df;
    dh[m * 2 * F + F + j] = dy * f;
  }
}
template <typename E, int KIND> hipError_t glu_bwd_t(const Glu& p, float* dh, hipStream_t st) {
  hipError_t e = hipSuccess;
  if (!p.hk) e = glu_fwd_t<E, KIND>(p, dh, st);
  else if (p.M) dgate_kernel<E, KIND><<<2048, 256, 0, st>>>(p, dh);
  if (e != hipSuccess) return e;
  const i64 F2 = 2 * (i64)p.N;
  if (p.dx)
    e = mm<1>(p.M, p.K, F2, [=] __device__(i64 m, i64 j) { return dh[m * F2 + j]; },
              [=] __device__(int, i64 k, i64 j) { return to_f32(static_cast<const E*>(p.W)[j * p.K + k]); },
              [=] __device__(i64 m, int k, const float* v) {
                float z = v[0];
                if (p.add) z += to_f32(static_cast<const E*>(p.add)[m * p.ldx + k]);
                static_cast<E*>(p.dx)[m * p.ldx + k] = from_f32<E>(z);
              }, st);
  if (p.dW && e == hipSuccess)
    e = mm<1>(F2, p.K, p.M, [=] __device__(i64 j, i64 m) { return dh[m * F2 + j]; },
              [=] __device__(int, i64 k, i64 m) { return to_f32(static_cast<const E*>(p.x)[m * p.ldx + k]); },
              [=] __device__(i64 j, int k, const float* v) { static_cast<E*>(p.dW)[j * p.K + k] = from_f32<E>(v[0]); }, st);
  if (p.db && e == hipSuccess) {
    sums_kernel<<<ceil_div((int)F2, 64), 64, 0, st>>>(p.M, (int)F2, [=] __device__(i64 m, i64 j) { return dh[m * F2 + j]; }, p.db);
    e = hipGetLastError();
  }
  return e;
}
template <class F> hipError_t by_gate(const Glu& p, F&& f) {
  auto with = [&](auto t) { return p.gate == CONVBN_GATE_SILU ? f(t, std::integral_constant<int, 0>{}) : f(t, std::integral_constant<int, 1>{}); };
  return p.dtype == CONVBN_BF16 ? with(bf16_t{}) : with(float{});
}

}  // namespace

size_t f8mul_scratch(i64, int, int) { return 0; }
hipError_t launch_f8mul(const F8Mul& p, void*, hipStream_t st) { return p.dtype == CONVBN_BF16 ? f8mul_t<bf16_t>(p, st) : f8mul_t<float>(p, st); }
size_t f8grad_scratch(const F8Grad&) { return 0; }
hipError_t launch_f8grad(const F8Grad& p, void*, hipStream_t st) { return p.dtype == CONVBN_BF16 ? f8grad_t<bf16_t>(p, st) : f8grad_t<float>(p, st); }

bool glu_in_place(int dtype, int K, i64 ld) { return dtype == CONVBN_BF16 && K % 8 == 0 && ld % 8 == 0 && ld <= 1 << 20; }
size_t glu_scratch(const Glu& p, int pass) { return pass == CONVBN_PASS_FWD ? 0 : align_up((size_t)p.M * 2 * p.N * 4, 256); }
hipError_t launch_glu_fwd(const Glu& p, void*, hipStream_t st) {
  return by_gate(p, [&](auto t, auto k) { return glu_fwd_t<decltype(t), k.value>(p, nullptr, st); });
}
hipError_t launch_glu_bwd(const Glu& p, void* ws, hipStream_t st) {
  return by_gate(p, [&](auto t, auto k) { return glu_bwd_t<decltype(t), k.value>(p, static_cast<float*>(ws), st); });
}

}  // namespace convbn
