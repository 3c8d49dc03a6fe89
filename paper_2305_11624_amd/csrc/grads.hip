// The two products of a backward pass, dx = a . w + add and dW = a^T . x: operands that lie across the sum, on the tiles of mm_tile.h.
//
// Where neither product fills the chip, both are one launch: the second need not wait for the last workgroup of the first.
#include "grads.h"
#include "mm_tile.h"

namespace convbn {

namespace {

// Rows ld apart, an addend laid out like them on top
template <typename T> struct GradOut {
  void* c; const void* add;
  i64 ld;
  int J;
  struct None {};
  __device__ __forceinline__ None columns(int) const { return {}; }
  __device__ __forceinline__ void operator()(i64 i, int j, const None&, const F8& v) const {
    store8_plus<T>(static_cast<T*>(c) + i * ld, add ? static_cast<const T*>(add) + i * ld : nullptr, j, J, v);
  }
};

// Both products in one launch, then what is left to do
template <class X, class W, int PAIRS, typename T>
__global__ __launch_bounds__(X::NT) void grads_pair_kernel(MmParams x, GradOut<T> ox, MmParams w, GradOut<T> ow, int first) {
  static_assert(X::NT == W::NT, "one launch");
  extern __shared__ __align__(16) unsigned char smem[];
  if ((int)blockIdx.x < first) mm_tile<X, false, true, false, PAIRS, EITHER>(x, (int)blockIdx.x, smem, ox);
  else mm_tile<W, true, true, false, PAIRS, EITHER>(w, (int)blockIdx.x - first, smem, ow);
}
template <typename T>
__global__ __launch_bounds__(256) void grads_join_kernel(MmParams x, GradOut<T> ox, unsigned nx, MmParams w, GradOut<T> ow, unsigned nw, SumJob sum) {
  if (blockIdx.x < nx) mm_join<false>(x, ox, blockIdx.x, nx);
  else if (blockIdx.x < nx + nw) mm_join<false>(w, ow, blockIdx.x - nx, nw);
  else join_sums(sum, (int)(blockIdx.x - nx - nw) * 256 + (int)threadIdx.x);
}

using Small = MmCfg<OpBf16, 64, 32, 32, 8, 2>;
using Mid = MmCfg<OpBf16, 128, 32, 64, 8, 1>;

template <class X, class W, int PAIRS, typename T> hipError_t pair(const MmParams& x, const GradOut<T>& ox, const MmParams& w, const GradOut<T>& ow, hipStream_t st) {
  constexpr int LDS = X::LDS > W::LDS ? X::LDS : W::LDS;
  static LdsLimitOnce once;
  auto* k = &grads_pair_kernel<X, W, PAIRS, T>;
  const hipError_t e = set_lds_limit_once(once, (const void*)k, LDS);
  if (e != hipSuccess) return e;
  k<<<mm_grid(x) + mm_grid(w), X::NT, LDS, st>>>(x, ox, w, ow, mm_grid(x));
  return hipGetLastError();
}

// The products one after the other, or both in one launch of workgroups that are alone on their compute units: where there is one for each, or
// where both would be such anyway.  (More of them, of unlike lengths, do not fill the chip any better: dx and dW of 1568 x 512 -> 2 x 2048 in tiles of 64 and 128
// together 36 us, one after the other 31.)
struct Plans { MmPlan dx, dw; bool one; };
Plans plans_of(i64 M, i64 N, int K, int pairs, bool both) {
  const int cx = pairs * chunks(N), cw = pairs * chunks(M);
  Plans pl = {mm_plan(M, K, cx), mm_plan(N, K, cw), false};
  if (!both || !M) return pl;
  auto alone = [](const MmPlan& p, i64 I, i64 J) { return p.tile <= 128 && mm_tiles(I, J, p.tile) * p.splits <= MM_CUS; };
  pl.one = alone(pl.dx, M, K) && alone(pl.dw, N, K);
  double best = pl.dx.us + pl.dw.us;
  for (int tx = 64; tx <= 128; tx *= 2)
    for (int sx = 1; sx <= 16 && sx <= cx; sx *= 2)
      for (int tw = 64; tw <= 128; tw *= 2)
        for (int sw = 1; sw <= 16 && sw <= cw; sw *= 2) {
          const int px = ceil_div(cx, sx), nx = ceil_div(cx, px), pw = ceil_div(cw, sw), nw = ceil_div(cw, pw);
          if (mm_tiles(M, K, tx) * nx + mm_tiles(N, K, tw) * nw > MM_CUS) continue;
          const double ux = mm_alone_us(tx, px), uw = mm_alone_us(tw, pw);
          const double join = (nx > 1 || nw > 1 ? 4.2 : 0) + 2e-6 * ((nx > 1 ? nx * (double)M : 0) + (nw > 1 ? nw * (double)N : 0)) * K;
          const double us = 2 + (ux > uw ? ux : uw) + join;
          if (us < best) {
            best = us;
            pl = {{tx, nx, px, us}, {tw, nw, pw, us}, true};
          }
        }
  return pl;
}

template <typename T, int PAIRS> hipError_t grads_t(const Grads& g, float* part, hipStream_t st) {
  const bool dx = g.dx && g.M, dw = g.dW;
  const Plans pl = plans_of(g.M, g.N, g.K, PAIRS, dx && dw);
  MmParams x = {}, w = {};
  x.a = w.a = g.a;
  x.b = g.w; w.b = g.x;
  x.I = g.M; x.R = g.N;
  w.I = g.N; w.R = g.M;
  x.J = w.J = g.K;
  x.plane_ch = chunks(g.N); x.nch = PAIRS * x.plane_ch;
  w.plane_ch = chunks(g.M); w.nch = PAIRS * w.plane_ch;
  mm_place(&x, pl.dx, part, false);
  mm_place(&w, pl.dw, part + mm_scratch(pl.dx, g.M, round8(g.K)) / 4, false);
  const GradOut<T> ox = {g.dx, g.add, g.ldx, g.K}, ow = {g.dW, nullptr, g.K, g.K};
  hipError_t e = hipSuccess;
  if (pl.one) {
    if (pl.dx.tile == 64) e = pl.dw.tile == 64 ? pair<Small, Small, PAIRS>(x, ox, w, ow, st) : pair<Small, Mid, PAIRS>(x, ox, w, ow, st);
    else e = pl.dw.tile == 64 ? pair<Mid, Small, PAIRS>(x, ox, w, ow, st) : pair<Mid, Mid, PAIRS>(x, ox, w, ow, st);
  } else {
    if (dx) e = mm_by_tile<OpBf16, false, true, false, PAIRS>(pl.dx.tile, x, ox, st);
    if (e == hipSuccess && dw) e = mm_by_tile<OpBf16, true, true, false, PAIRS>(pl.dw.tile, w, ow, st);
  }
  if (e != hipSuccess) return e;
  const unsigned nx = dx && pl.dx.splits > 1 ? join_blocks(x) : 0, nw = dw && pl.dw.splits > 1 ? join_blocks(w) : 0;
  const unsigned ns = g.sum.out ? ceil_div(g.sum.N, 256) : 0;
  if (nx + nw + ns) grads_join_kernel<T><<<nx + nw + ns, 256, 0, st>>>(x, ox, nx, w, ow, nw, g.sum);
  return hipGetLastError();
}

}  // namespace

size_t grads_scratch(i64 M, i64 N, int K, int pairs) {   // (either way)
  size_t most = 0;
  for (bool both : {false, true}) {
    const Plans pl = plans_of(M, N, K, pairs, both);
    const size_t n = mm_scratch(pl.dx, M, round8(K)) + mm_scratch(pl.dw, N, round8(K));
    most = n > most ? n : most;
  }
  return most;
}
hipError_t launch_grads(const Grads& g, float* part, hipStream_t st) {
  if (g.dtype == CONVBN_BF16) return grads_t<bf16_t, 1>(g, part, st);
  return g.pairs == 3 ? grads_t<float, 3>(g, part, st) : grads_t<float, 6>(g, part, st);
}

}  // namespace convbn
