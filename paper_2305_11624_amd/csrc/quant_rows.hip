// Rows in 8 bits: packing, reading back, and the gate between two products with its backward pass.
//
// A row is taken by a group of LPR lanes (a part of a wave, a wave, or the workgroup), each holding VPL pieces of 8 channels in
// registers from the one read of the row to the store of its codes: the maximum has to be known before the first code is.  Rows that
// are too long for that (VPL = 0) are read twice, the second time from the caches.  Many rows are bound by memory (100352 x 256: 15 us,
// 5.1 TB/s); few rows by the way there and back, so they take as many lanes as there are pieces, up to 1024
// (49 x 2048: 2.7 us for a launch).  The gate reads and writes 8 bytes for each bf16 element of y, forward and backward, and memory bounds
// it: 8192 x 8192, 537 MB, forward 113 us, 4.8 TB/s, backward 90 us, 6.0 TB/s (a part of what it reads is still in the last-level cache); GELU,
// with twice the operations, 117 and 94.  fp32 rows: 940 MB each way, 165 us, 5.7 TB/s, with either f.
#include "quant_code.h"

namespace convbn {

namespace {

constexpr int NT = 256;
// N maxima over the LPR lanes of a row (all of them call this together).
constexpr int threads_of(int LPR) { return LPR > NT ? LPR : NT; }
template <int LPR, int N> __device__ __forceinline__ void group_max(unsigned (&m)[N], unsigned (&lds)[N][16]) {
#pragma unroll
  for (int off = (LPR < 64 ? LPR : 64) / 2; off > 0; off >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) m[i] = max(m[i], (unsigned)__shfl_xor((int)m[i], off, 64));
  if constexpr (LPR > 64) {
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) lds[i][threadIdx.x >> 6] = m[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int w = 0; w < LPR / 64; ++w) m[i] = max(m[i], lds[i][w]);
    __syncthreads();   // (the next row's maxima go to the same place)
  }
}

struct RowArgs { i64 rows, ld; int K; const void* x; void* out; uint8_t* codes; float* scales; };

template <typename T, int LPR, int VPL>
__global__ __launch_bounds__(threads_of(LPR)) void qpack_kernel(RowArgs p) {
  __shared__ unsigned lds[1][16];
  constexpr int RPB = threads_of(LPR) / LPR;
  const int lane = threadIdx.x % LPR, row0 = threadIdx.x / LPR;
  const int K = p.K, Kp = qrow(K);
  for (i64 b = blockIdx.x; b * RPB < p.rows; b += gridDim.x) {   // (whole groups: every lane reaches group_max)
    const i64 row = b * RPB + row0;
    const bool in = row < p.rows;
    const T* x = static_cast<const T*>(p.x) + (in ? row : 0) * p.ld;
    uint8_t* codes = p.codes + (in ? row : 0) * Kp;
    F8 f[VPL ? VPL : 1];
    unsigned m[1] = {0};
    if constexpr (VPL > 0) {
#pragma unroll
      for (int v = 0; v < VPL; ++v) f[v] = load8<T>(x, (v * LPR + lane) * 8, in ? K : 0);
#pragma unroll
      for (int v = 0; v < VPL; ++v) m[0] = max(m[0], amax8(f[v]));
    } else {
      for (int k = lane * 8; k < K; k += LPR * 8) m[0] = max(m[0], amax8(load8<T>(x, k, K)));
    }
    group_max<LPR>(m, lds);
    const Scale sc = scale_of(m[0]);
    if (!in) continue;
    if (lane == 0) p.scales[row] = sc.s;
    if constexpr (VPL > 0) {
#pragma unroll
      for (int v = 0; v < VPL; ++v) {
        const int k = (v * LPR + lane) * 8;
        if (k < Kp) *reinterpret_cast<uint2*>(codes + k) = codes8(f[v], sc.r);
      }
    } else {
      for (int k = lane * 8; k < Kp; k += LPR * 8) *reinterpret_cast<uint2*>(codes + k) = codes8(load8<T>(x, k, K), sc.r);
    }
  }
}

__device__ __forceinline__ i64 row_of(i64 i, unsigned pieces) { return i >> 32 ? i / pieces : (i64)((unsigned)i / pieces); }

template <typename T>
__global__ __launch_bounds__(NT) void qunpack_kernel(RowArgs p, unsigned pieces) {
  const int K = p.K, Kp = qrow(K);
  const i64 total = p.rows * pieces;
  for (i64 i = (i64)blockIdx.x * NT + threadIdx.x; i < total; i += (i64)gridDim.x * NT) {
    const i64 row = row_of(i, pieces);
    const int k = (int)(i - row * pieces) * 8;
    const uint2 c = *reinterpret_cast<const uint2*>(p.codes + row * Kp + k);
    store8<T>(static_cast<T*>(p.out) + row * p.ld, k, K, decode8(c, p.scales[row]));
  }
}

struct GateArgs {
  i64 rows, ldh, ldy;
  int K;
  const void* h; void* y; uint8_t* hc; float* hs; uint8_t* yc; float* ys;   // forward
  const void* dy; void* dh;                                                  // backward
};

template <typename T, int KIND, int LPR, int VPL>
__global__ __launch_bounds__(threads_of(LPR)) void qgate_fwd_kernel(GateArgs p) {
  __shared__ unsigned lds_h[2][16], lds_y[1][16];
  constexpr int RPB = threads_of(LPR) / LPR, NV = VPL ? VPL : 1;
  const int lane = threadIdx.x % LPR, row0 = threadIdx.x / LPR;
  const int K = p.K, Kp = qrow(K);
  for (i64 b = blockIdx.x; b * RPB < p.rows; b += gridDim.x) {
    const i64 row = b * RPB + row0;
    const bool in = row < p.rows;
    const i64 at = in ? row : 0;
    const T* h = static_cast<const T*>(p.h) + at * p.ldh;
    auto make = [](const F8& g, const F8& u) {
      F8 y;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float f, df;
        gate_of<T, KIND>(g.v[i], &f, &df);
        y.v[i] = f * u.v[i];
      }
      return y;
    };
    F8 g[NV], u[NV], y[NV];
    unsigned mh[2] = {0, 0}, my[1] = {0};
    auto look = [&](const F8& a, const F8& b2, const F8& c) {
      if (p.hc) { mh[0] = max(mh[0], amax8(a)); mh[1] = max(mh[1], amax8(b2)); }
      if (p.yc) my[0] = max(my[0], amax8(c));
    };
    if constexpr (VPL > 0) {
      const int Kin = in ? K : 0;
#pragma unroll
      for (int v = 0; v < VPL; ++v) {
        g[v] = load8<T>(h, (v * LPR + lane) * 8, Kin);
        u[v] = load8<T>(h + K, (v * LPR + lane) * 8, Kin);
      }
#pragma unroll
      for (int v = 0; v < VPL; ++v) {
        y[v] = make(g[v], u[v]);
        look(g[v], u[v], y[v]);
      }
    } else {
      for (int k = lane * 8; k < K; k += LPR * 8) {
        g[0] = load8<T>(h, k, K);
        u[0] = load8<T>(h + K, k, K);
        look(g[0], u[0], make(g[0], u[0]));
      }
    }
    if (p.hc) group_max<LPR>(mh, lds_h);
    if (p.yc) group_max<LPR>(my, lds_y);
    const Scale sg = scale_of(mh[0]), su = scale_of(mh[1]), sy = scale_of(my[0]);
    if (!in) continue;
    if (lane == 0) {
      if (p.hc) { p.hs[2 * row] = sg.s; p.hs[2 * row + 1] = su.s; }
      if (p.yc) p.ys[row] = sy.s;
    }
    auto out = [&](int k, const F8& a, const F8& b2, const F8& c) {
      if (k >= Kp) return;
      if (p.hc) {
        *reinterpret_cast<uint2*>(p.hc + 2 * row * Kp + k) = codes8(a, sg.r);
        *reinterpret_cast<uint2*>(p.hc + (2 * row + 1) * Kp + k) = codes8(b2, su.r);
      }
      if (p.yc) *reinterpret_cast<uint2*>(p.yc + row * Kp + k) = codes8(c, sy.r);
      if (p.y) store8<T>(static_cast<T*>(p.y) + row * p.ldy, k, K, c);
    };
    if constexpr (VPL > 0) {
#pragma unroll
      for (int v = 0; v < VPL; ++v) out((v * LPR + lane) * 8, g[v], u[v], y[v]);
    } else {
      for (int k = lane * 8; k < Kp; k += LPR * 8) {
        g[0] = load8<T>(h, k, K);
        u[0] = load8<T>(h + K, k, K);
        out(k, g[0], u[0], make(g[0], u[0]));
      }
    }
  }
}

template <typename T, int KIND>
__global__ __launch_bounds__(NT) void qgate_bwd_kernel(GateArgs p, unsigned pieces) {
  const int K = p.K, Kp = qrow(K);
  const i64 total = p.rows * pieces;
  for (i64 i = (i64)blockIdx.x * NT + threadIdx.x; i < total; i += (i64)gridDim.x * NT) {
    const i64 row = row_of(i, pieces);
    const int k = (int)(i - row * pieces) * 8;
    const F8 g = decode8(*reinterpret_cast<const uint2*>(p.hc + 2 * row * Kp + k), p.hs[2 * row]);
    const F8 u = decode8(*reinterpret_cast<const uint2*>(p.hc + (2 * row + 1) * Kp + k), p.hs[2 * row + 1]);
    const F8 dy = load8<T>(static_cast<const T*>(p.dy) + row * p.ldy, k, K);
    F8 dg, du;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float f, df;
      gate_of<T, KIND>(g.v[e], &f, &df);
      dg.v[e] = dy.v[e] * u.v[e] * df;
      du.v[e] = dy.v[e] * f;
    }
    T* dh = static_cast<T*>(p.dh) + row * p.ldh;
    store8<T>(dh, k, K, dg);
    store8<T>(dh + K, k, K, du);
  }
}

int blocks_of(i64 work) { return (int)(work < 1 << 20 ? work : 1 << 20); }   // (launches stay below 2^32 threads)

}  // namespace

// Calls f(LPR, VPL) with the group for rows of K channels: with few rows (at most two a compute unit) one piece a lane as far as that goes, else
// few lanes and more pieces in flight for each.  us, forward gate: 4 rows of 8192 with 256 lanes 7.0,
// with 1024 4.9; 8192 rows of 8192 with 256 lanes of four pieces 121, with 512 of two 113, with 1024 of one 149.
template <class F> static hipError_t by_row_length(i64 rows, int K, F&& f) {
  const int pieces = ceil_div(K, 8);
  using std::integral_constant;
#define QROW(LPR, VPL) \
  if (pieces <= (LPR) * (VPL)) return f(integral_constant<int, LPR>{}, integral_constant<int, VPL>{})
  QROW(8, 1); QROW(16, 1); QROW(32, 1); QROW(64, 1);
  if (rows <= 512) { QROW(256, 1); QROW(512, 1); QROW(1024, 1); }
  QROW(64, 2); QROW(256, 1); QROW(256, 2); QROW(512, 2); QROW(1024, 2);
#undef QROW
  return f(integral_constant<int, 256>{}, integral_constant<int, 0>{});
}

template <typename T> static hipError_t pack_t(const RowArgs& a, hipStream_t st) {
  return by_row_length(a.rows, a.K, [&](auto lpr, auto vpl) {
    constexpr int nt = threads_of(lpr.value);
    const int grid = blocks_of((a.rows + nt / lpr.value - 1) / (nt / lpr.value));
    qpack_kernel<T, lpr.value, vpl.value><<<grid, nt, 0, st>>>(a);
    return hipGetLastError();
  });
}

hipError_t launch_qpack(int dtype, i64 rows, int K, i64 ld, const void* x, void* codes, float* scales, hipStream_t st) {
  if (!rows) return hipSuccess;
  const RowArgs a = {rows, ld, K, x, nullptr, (uint8_t*)codes, scales};
  if (dtype == CONVBN_BF16) return pack_t<bf16_t>(a, st);
  return pack_t<float>(a, st);
}

hipError_t launch_qunpack(int dtype, i64 rows, int K, i64 ld, const void* codes, const float* scales, void* x, hipStream_t st) {
  if (!rows) return hipSuccess;
  const RowArgs a = {rows, ld, K, nullptr, x, (uint8_t*)codes, (float*)scales};
  const unsigned pieces = ceil_div(K, 8);
  const int grid = blocks_of((rows * pieces + NT - 1) / NT);
  if (dtype == CONVBN_BF16) qunpack_kernel<bf16_t><<<grid, NT, 0, st>>>(a, pieces);
  else qunpack_kernel<float><<<grid, NT, 0, st>>>(a, pieces);
  return hipGetLastError();
}

template <typename T, int KIND> static hipError_t gate_fwd_t(const GateArgs& a, hipStream_t st) {
  return by_row_length(a.rows, a.K, [&](auto lpr, auto vpl) {
    constexpr int nt = threads_of(lpr.value);
    const int grid = blocks_of((a.rows + nt / lpr.value - 1) / (nt / lpr.value));
    qgate_fwd_kernel<T, KIND, lpr.value, vpl.value><<<grid, nt, 0, st>>>(a);
    return hipGetLastError();
  });
}
template <typename T, int KIND> static hipError_t gate_bwd_t(const GateArgs& a, hipStream_t st) {
  const unsigned pieces = ceil_div(a.K, 8);
  qgate_bwd_kernel<T, KIND><<<blocks_of((a.rows * pieces + NT - 1) / NT), NT, 0, st>>>(a, pieces);
  return hipGetLastError();
}
// Calls f(T, KIND) with the gate's types
template <class F> static hipError_t by_gate(int dtype, int kind, F&& f) {
  auto with = [&](auto t) { return kind == CONVBN_GATE_SILU ? f(t, std::integral_constant<int, 0>{}) : f(t, std::integral_constant<int, 1>{}); };
  return dtype == CONVBN_BF16 ? with(bf16_t{}) : with(float{});
}

hipError_t launch_qgate_fwd(int dtype, int kind, i64 rows, int K, i64 ldh, i64 ldy, const void* h, void* h_codes, float* h_scales,
                            void* y, void* y_codes, float* y_scales, hipStream_t st) {
  if (!rows) return hipSuccess;
  GateArgs a = {rows, ldh, ldy, K, h, y, (uint8_t*)h_codes, h_scales, (uint8_t*)y_codes, y_scales, nullptr, nullptr};
  return by_gate(dtype, kind, [&](auto t, auto k) { return gate_fwd_t<decltype(t), k.value>(a, st); });
}
hipError_t launch_qgate_bwd(int dtype, int kind, i64 rows, int K, i64 ldh, i64 ldy, const void* h_codes, const float* h_scales,
                            const void* dy, void* dh, hipStream_t st) {
  if (!rows) return hipSuccess;
  GateArgs a = {rows, ldh, ldy, K, nullptr, nullptr, (uint8_t*)h_codes, (float*)h_scales, nullptr, nullptr, dy, dh};
  return by_gate(dtype, kind, [&](auto t, auto k) { return gate_bwd_t<decltype(t), k.value>(a, st); });
}

}  // namespace convbn
