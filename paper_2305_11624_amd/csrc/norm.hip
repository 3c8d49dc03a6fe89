// Group norm with an activation, channels last, forward and backward: a workgroup an image and group.
#include "f8_code.h"

namespace convbn {

namespace {

constexpr int NT = 256;

__device__ __forceinline__ float block_sum(float v, float* lds) {
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  float s = 0.f;
  for (int w = 0; w < NT / 64; ++w) s += lds[w];
  return s;
}
template <typename T, int F> __device__ __forceinline__ void act_of(float z, float* f, float* df) {
  if constexpr (F == CONVBN_NORM_NONE) { *f = z; *df = 1.f; }
  else if constexpr (F == CONVBN_NORM_RELU) { *f = z > 0.f ? z : 0.f * z; *df = z > 0.f ? 1.f : 0.f; }
  else gate_of<T, F == CONVBN_NORM_SILU ? CONVBN_GATE_SILU : CONVBN_GATE_GELU>(z, f, df);
}

template <typename T, int F> __global__ __launch_bounds__(NT) void norm_fwd_kernel(Norm p) {
  __shared__ float lds[NT / 64];
  const int cg = p.C / p.groups, g = blockIdx.x % p.groups;
  const i64 m = blockIdx.x / p.groups, n = p.P * cg;
  const T* x = static_cast<const T*>(p.x) + m * p.P * p.ldx + g * cg;
  float s = 0.f;
  for (i64 i = threadIdx.x; i < n; i += NT) s += to_f32(x[i / cg * p.ldx + i % cg]);
  const float mean = block_sum(s, lds) / (float)n;
  s = 0.f;
  for (i64 i = threadIdx.x; i < n; i += NT) {
    const float d = to_f32(x[i / cg * p.ldx + i % cg]) - mean;
    s += d * d;
  }
  const float r = 1.f / sqrtf(block_sum(s, lds) / (float)n + p.eps);
  if (p.stats && threadIdx.x == 0) {
    p.stats[2 * (i64)blockIdx.x] = mean;
    p.stats[2 * (i64)blockIdx.x + 1] = r;
  }
  T* y = static_cast<T*>(p.y) + m * p.P * p.ldy + g * cg;
  for (i64 i = threadIdx.x; i < n; i += NT) {
    const int c = (int)(i % cg);
    const float z = (to_f32(x[i / cg * p.ldx + c]) - mean) * r * (p.gamma ? p.gamma[g * cg + c] : 1.f) + (p.beta ? p.beta[g * cg + c] : 0.f);
    float f, df;
    act_of<T, F>(z, &f, &df);
    y[i / cg * p.ldy + c] = from_f32<T>(f);
  }
}

template <typename T, int F> __global__ __launch_bounds__(NT) void norm_bwd_kernel(Norm p, float* sums) {
  __shared__ float lds[NT / 64];
  const int cg = p.C / p.groups, g = blockIdx.x % p.groups;
  const i64 m = blockIdx.x / p.groups, n = p.P * cg;
  const T* x = static_cast<const T*>(p.x) + m * p.P * p.ldx + g * cg;
  const T* dy = static_cast<const T*>(p.dy) + m * p.P * p.ldy + g * cg;
  const float mean = p.stats[2 * (i64)blockIdx.x], r = p.stats[2 * (i64)blockIdx.x + 1];
  auto at = [&](i64 px, int c, float* xhat) {
    const float ga = p.gamma ? p.gamma[g * cg + c] : 1.f;
    *xhat = (to_f32(x[px * p.ldx + c]) - mean) * r;
    float f, df;
    act_of<T, F>(*xhat * ga + (p.beta ? p.beta[g * cg + c] : 0.f), &f, &df);
    return to_f32(dy[px * p.ldy + c]) * df;
  };
  float s1 = 0.f, s2 = 0.f;
  for (int c = 0; c < cg; ++c) {
    float a = 0.f, b = 0.f;
    for (i64 px = threadIdx.x; px < p.P; px += NT) {
      float xhat;
      const float dz = at(px, c, &xhat);
      a += dz;
      b += dz * xhat;
    }
    a = block_sum(a, lds);
    b = block_sum(b, lds);
    const float ga = p.gamma ? p.gamma[g * cg + c] : 1.f;
    s1 += ga * a;
    s2 += ga * b;
    if (threadIdx.x == 0) {
      sums[(m * p.C + g * cg + c) * 2] = b;
      sums[(m * p.C + g * cg + c) * 2 + 1] = a;
    }
  }
  if (!p.dx) return;
  s1 /= (float)n;
  s2 /= (float)n;
  T* dx = static_cast<T*>(p.dx) + m * p.P * p.ldx + g * cg;
  const T* add = p.add ? static_cast<const T*>(p.add) + m * p.P * p.ldx + g * cg : nullptr;
  for (i64 i = threadIdx.x; i < n; i += NT) {
    const int c = (int)(i % cg);
    float xhat;
    const float dz = at(i / cg, c, &xhat);
    float v = r * (dz * (p.gamma ? p.gamma[g * cg + c] : 1.f) - s1 - xhat * s2);
    if (add) v += to_f32(add[i / cg * p.ldx + c]);
    dx[i / cg * p.ldx + c] = from_f32<T>(v);
  }
}
__global__ __launch_bounds__(64) void norm_join_kernel(Norm p, const float* sums) {
  const int c = blockIdx.x * 64 + threadIdx.x;
  if (c >= p.C) return;
  float a = 0.f, b = 0.f;
  for (i64 m = 0; m < p.M; ++m) {
    a += sums[(m * p.C + c) * 2];
    b += sums[(m * p.C + c) * 2 + 1];
  }
  if (p.dgamma) p.dgamma[c] = a;
  if (p.dbeta) p.dbeta[c] = b;
}

template <class F> hipError_t by_type(const Norm& p, F&& f) {
  using std::integral_constant;
  auto with = [&](auto t) {
    switch (p.f) {
      case CONVBN_NORM_RELU: return f(t, integral_constant<int, CONVBN_NORM_RELU>{});
      case CONVBN_NORM_SILU: return f(t, integral_constant<int, CONVBN_NORM_SILU>{});
      case CONVBN_NORM_GELU: return f(t, integral_constant<int, CONVBN_NORM_GELU>{});
    }
    return f(t, integral_constant<int, CONVBN_NORM_NONE>{});
  };
  return p.dtype == CONVBN_BF16 ? with(bf16_t{}) : with(float{});
}

}  // namespace

size_t norm_scratch(const Norm& p, int pass) { return pass == CONVBN_PASS_FWD ? 0 : align_up((size_t)p.M * p.C * 8, 256); }
hipError_t launch_norm_fwd(const Norm& p, void*, hipStream_t st) {
  if (!p.M) return hipSuccess;
  return by_type(p, [&](auto t, auto f) {
    norm_fwd_kernel<decltype(t), f.value><<<(unsigned)(p.M * p.groups), NT, 0, st>>>(p);
    return hipGetLastError();
  });
}
hipError_t launch_norm_bwd(const Norm& p, void* ws, hipStream_t st) {
  float* sums = static_cast<float*>(ws);
  hipError_t e = hipSuccess;
  if (p.M)
    e = by_type(p, [&](auto t, auto f) {
      norm_bwd_kernel<decltype(t), f.value><<<(unsigned)(p.M * p.groups), NT, 0, st>>>(p, sums);
      return hipGetLastError();
    });
  if (e != hipSuccess || !(p.dgamma || p.dbeta)) return e;
  norm_join_kernel<<<ceil_div(p.C, 64), 64, 0, st>>>(p, sums);
  return hipGetLastError();
}

}  // namespace convbn
