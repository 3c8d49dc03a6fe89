// The gated product y = f(x Wg^T + bg) (x Wu^T + bu) and its gradients.
//
// Forward is one product: a tile takes 32 rows of Wg and the same 32 of Wu in turn, so that a wave holds g and u of the same numbers of y when
// the sum is done, and neither goes to memory unless it is kept.  Backward turns g, u and dy into dh = [dg | du] in one pass, which sums dh's columns too,
// and multiplies it with W and with x as they lie.
//
// Bound by the matrix pipe (mm_tile.h): 8192 x 4096 -> 8192 forward 955 us, 1150 TFLOP/s; dx and dW 848 and 857, 1300 each; dh in front of them 172, 940 MB read
// and written at 5.4 TB/s.  The projections are kept in 32 bits: kept in bf16 that pass takes 122, and the gradients are off by a third more
// (relative 2-norm against 64 bits 0.003 instead of 0.0023, where dh in bf16 and the result's own rounding make 0.0023).
//
// F32: operands are split into three bf16 parts that add up to all 24 bits, and six products of parts are summed in fp32; the others add up to at most 2^-24 of
// a product, of either sign.  8192 x 2048 -> 4096 forward 1350 us (a library's fp32 product alone 1850), backward 2770; one row 2048 -> 8192 28.7, 134 MB.
#include "grads.h"
#include "mm_tile.h"

namespace convbn {

namespace {

int planes_of(int dtype) { return dtype == CONVBN_BF16 ? 1 : 4; }

// ---- forward ----
template <typename T, int KIND> struct GluOut {
  Glu q;
  struct Cols { F8 g, u; };
  __device__ __forceinline__ Cols columns(int n) const {
    return q.b ? Cols{load8<float>(q.b, n, q.N), load8<float>(q.b + q.N, n, q.N)} : Cols{};
  }
  __device__ __forceinline__ void operator()(i64 m, int n, const Cols& b, F8 g, F8 u) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      g.v[i] += b.g.v[i];
      u.v[i] += b.u.v[i];
    }
    if (q.h) {
      float* h = q.h + m * 2 * q.N;   // (halves of a lane's 32 bytes are two stores: the caches make lines of them)
      store8<float>(h, n, q.N, g);
      store8<float>(h + q.N, n, q.N, u);
    }
    if (q.y) {
      F8 y;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float f, df;
        gate_of<T, KIND>(g.v[i], &f, &df);
        y.v[i] = f * u.v[i];
      }
      store8<T, true>(static_cast<T*>(q.y) + m * q.ldz, n, q.N, y);
    }
  }
};

// ---- in front of the gradients: dh and its column sums, copies of x and W where they are not read in place ----
// dh: workgroups of 256 columns of either half and a slice of the rows, a thread eight columns of every 16th row.
constexpr int NT = 32 * SUM_ROWS;
struct DGate {
  i64 M, ldz, per;
  int N, W2, across, blocks;
  const float* h; const void* dy;
  bf16_t* dh; i64 plane;      // null: not wanted
  float* sums;                // [slices][2 N] or null
};
template <typename T, int KIND> __global__ __launch_bounds__(NT) void glu_prep_kernel(DGate p, RowsCopy x, unsigned nx, RowsCopy w) {
  __shared__ float meet[SUM_ROWS][256 + 8];
  if ((int)blockIdx.x >= p.blocks) {
    const unsigned wg = blockIdx.x - p.blocks;
    if (wg < nx) rows_copy<T, NT>(x, wg, nx);
    else rows_copy<T, NT>(w, wg - nx, gridDim.x - p.blocks - nx);
    return;
  }
  const int slice = (int)blockIdx.x / p.across, n0 = ((int)blockIdx.x - slice * p.across) * 256, n = n0 + (threadIdx.x & 31) * 8;
  const i64 beg = (i64)slice * p.per, end = beg + p.per < p.M ? beg + p.per : p.M;
  F8 sum[2] = {};
  if (n < p.N) {
#pragma unroll 2
    for (i64 m = beg + (threadIdx.x >> 5); m < end; m += SUM_ROWS) {
      const float* h = p.h + m * 2 * p.N;
      const F8 g = load8<float>(h, n, p.N), u = load8<float>(h + p.N, n, p.N), dy = load8<T>(static_cast<const T*>(p.dy) + m * p.ldz, n, p.N);
      F8 d[2];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float f, df;
        gate_of<T, KIND>(g.v[i], &f, &df);
        d[0].v[i] = dy.v[i] * u.v[i] * df;
        d[1].v[i] = dy.v[i] * f;
      }
#pragma unroll
      for (int y = 0; y < 2; ++y) {
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[y].v[i] += d[y].v[i];
        if (!p.dh) continue;
        bf16_t* out = p.dh + m * p.W2 + y * p.N;
        const int width = y ? p.W2 - p.N : p.N;   // (u's last piece clears what is behind it: products read whole rows)
        const int behind = y && n + 8 >= p.N ? width : 0;
        if constexpr (sizeof(T) == 2) {
          store8<bf16_t>(out, n, width, d[y]);
          for (int c = n + 8; c < behind; ++c) out[c] = bf16_t(0.f);
        } else {
          const Parts4 part = split3_near(d[y]);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            store8<bf16_t>(out + i * p.plane, n, width, widen(Raw8<bf16_t>{part.p[i]}));
            for (int c = n + 8; c < behind; ++c) out[i * p.plane + c] = bf16_t(0.f);
          }
        }
      }
    }
  }
  if (!p.sums) return;
#pragma unroll
  for (int y = 0; y < 2; ++y) meet_sums(sum[y], meet, n0, p.N, p.sums + (i64)slice * 2 * p.N + y * p.N);
}

// ---- gradients ----
// What a call needs of the workspace, in this order, and its operands
struct Plan {
  MmPlan fwd;
  int slices;
  size_t h, dh, x, W, part, sums, total;
};
Plan plan_of(const Glu& p, bool bwd) {
  Plan s = {};
  const int pl = planes_of(p.dtype), pairs = pl == 1 ? 1 : 6, K8 = round8(p.K), W2 = round8(2 * p.N);
  s.fwd = mm_plan(p.M, 2 * (i64)p.N, pairs * chunks(K8));
  s.x = glu_in_place(p.dtype, p.K, p.ldx) ? 0 : align_up((size_t)pl * p.M * K8 * 2, 256);
  s.W = glu_in_place(p.dtype, p.K, p.K) ? 0 : align_up((size_t)pl * 2 * p.N * K8 * 2, 256);
  s.part = mm_scratch(s.fwd, p.M, 2 * round8(p.N));
  if (bwd) {
    s.slices = row_slices(p.M, p.N);
    s.h = p.kept ? 0 : align_up((size_t)p.M * 2 * p.N * 4, 256);
    s.dh = align_up((size_t)pl * p.M * W2 * 2, 256);
    const size_t both = grads_scratch(p.M, 2 * (i64)p.N, p.K, pairs);
    s.part = s.part > both ? s.part : both;
    s.sums = align_up((size_t)s.slices * 2 * p.N * 4, 256);
  }
  s.total = s.h + s.dh + s.x + s.W + s.part + s.sums;
  return s;
}

// x and W as the products read them, after launch_rows_copies
struct Operands { RowsOp x, W; RowsCopy cx, cw; };
Operands operands_of(const Glu& p, const Plan& s, char* ws, bool want_x, bool want_W) {
  Operands o = {};
  const int K8 = round8(p.K);
  bf16_t* const x = reinterpret_cast<bf16_t*>(ws + s.h + s.dh);
  bf16_t* const W = reinterpret_cast<bf16_t*>(ws + s.h + s.dh + s.x);
  if (s.x && want_x) o.cx = {p.M, p.ldx, p.K, p.x, x};
  if (s.W && want_W) o.cw = {2 * (i64)p.N, p.K, p.K, p.W, W};
  o.x = s.x ? RowsOp{(const uint8_t*)x, 2 * K8, 2 * p.M * K8, 2 * K8} : RowsOp{(const uint8_t*)p.x, 2 * p.ldx, 0, 2 * K8};
  o.W = s.W ? RowsOp{(const uint8_t*)W, 2 * K8, 4 * (i64)p.N * K8, 2 * K8} : RowsOp{(const uint8_t*)p.W, 2 * K8, 0, 2 * K8};
  return o;
}

template <typename T, int KIND> hipError_t project(const Glu& p, const Plan& s, const Operands& o, char* ws, hipStream_t st) {
  if (glu_few_taken(p.M, p.K, p.dtype)) return launch_glu_few(p, st);
  constexpr int PAIRS = sizeof(T) == 2 ? 1 : 6;
  MmParams m = {};
  m.a = o.x; m.b = o.W;
  m.I = p.M; m.J = p.N;
  m.plane_ch = chunks(round8(p.K));
  m.nch = PAIRS * m.plane_ch;
  return mm_launch<OpBf16, false, false, true, PAIRS>(m, s.fwd, reinterpret_cast<float*>(ws + s.h + s.dh + s.x + s.W), GluOut<T, KIND>{p}, st);
}

template <typename T, int KIND> hipError_t fwd_t(const Glu& p, char* ws, hipStream_t st) {
  if (glu_few_taken(p.M, p.K, p.dtype)) return launch_glu_few(p, st);
  const Plan s = plan_of(p, false);
  const Operands o = operands_of(p, s, ws, true, true);
  const hipError_t e = launch_rows_copies(p.dtype, o.cx, o.cw, st);
  return e == hipSuccess ? project<T, KIND>(p, s, o, ws, st) : e;
}

template <typename T, int KIND> hipError_t bwd_t(const Glu& p, char* ws, hipStream_t st) {
  const Plan s = plan_of(p, true);
  const bool again = !p.hk && p.M, want_dx = p.dx && p.M, want_dW = p.dW && p.M;
  const Operands o = operands_of(p, s, ws, again || want_dW, again || want_dx);
  const float* h = p.hk;
  if (again) {
    Glu q = p;
    q.y = nullptr;
    q.h = reinterpret_cast<float*>(ws);
    hipError_t e = launch_rows_copies(p.dtype, o.cx, o.cw, st);
    if (e == hipSuccess) e = project<T, KIND>(q, s, o, ws, st);
    if (e != hipSuccess) return e;
    h = q.h;
  }
  float* const sums = reinterpret_cast<float*>(ws + s.h + s.dh + s.x + s.W + s.part);
  const int W2 = round8(2 * p.N);
  bf16_t* const dh = reinterpret_cast<bf16_t*>(ws + s.h);
  // (rows that are not summed go in slices of a turn each)
  const int slices = p.db ? s.slices : (int)(p.M > SUM_ROWS << 16 ? 1 << 16 : (p.M + SUM_ROWS - 1) / SUM_ROWS);
  DGate d = {p.M, p.ldz, slices ? (p.M + slices - 1) / slices : 0, p.N, W2, ceil_div(p.N, 256), 0, h, p.dy, want_dx || want_dW ? dh : nullptr, p.M * W2,
             !p.db ? nullptr : slices > 1 ? sums : p.db};
  d.blocks = d.across * slices;
  const RowsCopy cx = again ? RowsCopy{} : o.cx, cw = again ? RowsCopy{} : o.cw;
  const unsigned nx = piece_blocks<NT>(cx.rows, cx.width, cx.out), nw = piece_blocks<NT>(cw.rows, cw.width, cw.out), blocks = d.blocks + nx + nw;
  if (blocks) glu_prep_kernel<T, KIND><<<blocks, NT, 0, st>>>(d, cx, nx, cw);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  Grads g = {};
  g.M = p.M; g.N = 2 * (i64)p.N; g.K = p.K; g.ldx = p.ldx; g.pairs = sizeof(T) == 2 ? 1 : 6; g.dtype = p.dtype;
  g.a = {(const uint8_t*)dh, 2 * W2, 2 * p.M * W2, 2 * W2};
  g.w = o.W; g.x = o.x;
  g.dx = p.dx; g.add = p.add; g.dW = p.dW;
  g.sum = {sums, slices, 2 * p.N, p.db && slices > 1 ? p.db : nullptr};
  return launch_grads(g, reinterpret_cast<float*>(ws + s.h + s.dh + s.x + s.W), st);
}

// Calls f(T, KIND) with the gate's types
template <class F> hipError_t by_gate(const Glu& p, F&& f) {
  auto with = [&](auto t) { return p.gate == CONVBN_GATE_SILU ? f(t, std::integral_constant<int, 0>{}) : f(t, std::integral_constant<int, 1>{}); };
  return p.dtype == CONVBN_BF16 ? with(bf16_t{}) : with(float{});
}

}  // namespace

bool glu_in_place(int dtype, int K, i64 ld) { return dtype == CONVBN_BF16 && K % 8 == 0 && ld % 8 == 0 && ld <= 1 << 20; }
size_t glu_scratch(const Glu& p, int pass) {
  return pass == CONVBN_PASS_FWD && glu_few_taken(p.M, p.K, p.dtype) ? 0 : plan_of(p, pass == CONVBN_PASS_BWD).total;
}
hipError_t launch_glu_fwd(const Glu& p, void* ws, hipStream_t st) {
  return by_gate(p, [&](auto t, auto k) { return fwd_t<decltype(t), k.value>(p, static_cast<char*>(ws), st); });
}
hipError_t launch_glu_bwd(const Glu& p, void* ws, hipStream_t st) {
  return by_gate(p, [&](auto t, auto k) { return bwd_t<decltype(t), k.value>(p, static_cast<char*>(ws), st); });
}

}  // namespace convbn
