// z = sx sw (qx . qw) + b + add: the product of 8-bit integers with a scale for each row of either operand.
//
// Both operands' channels run together, which is what the matrix instruction wants; they pass through LDS as rows of 128 codes whose
// 16-byte pieces are exchanged by bits 1-3 of the row, so that 16 lanes reading a column of pieces meet distinct banks.  Sums over
// channels that are split between workgroups stay whole numbers: any order gives the same.
//
// 8192 x 4096 x 8192: 233 - 252 us (2180 - 2355 TOP/s), a little faster than the library's rate at 8192^3 (2036 - 2094).  The matrix pipe is busy for
// 57 % of the time: with one workgroup of 256 x 256 a compute unit, what is left is the copies behind each chunk's barrier, the epilogue (134 MB
// out, 26 us at a copy's rate) and the drain of the last round.  Small products (1568 x 2048 x 512: 7 us) are bound by the way to memory:
// four waves a SIMD, each with few chunks.
#include "quant_code.h"

namespace convbn {

namespace {

typedef int i32x16 __attribute__((ext_vector_type(16)));

constexpr int KC = 128;                 // channels at a time: a whole cache line a row

struct MulParams {
  QMul m;
  int Kp, nch, splits, per;   // chunks of KC, chunks of a split
  int nti, ntj;
  int* part;                  // [splits][M][N], where there are several
};

// Eight channels n .. n+7 of row m: scaled, with bias and addend, rounded once
template <typename T>
__device__ __forceinline__ void finish8(const QMul& q, i64 m, int n, const int (&acc)[8], float sx, const float (&sw)[8], const float (&b)[8]) {
  F8 f;
  // (no branch: one by the row's scale in front of a store takes 22144 x 192 -> 3840 from 66 to 68 - 70 us, wherever it stands, the third factor to 67)
  const float first = scale_last(sx) ? 1.f : sx, last = scale_last(sx) ? sx : 1.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) f.v[i] = (float)acc[i] * first * sw[i] * last + b[i];
  store8_plus<T>(static_cast<T*>(q.z) + m * q.ldz, q.add ? static_cast<const T*>(q.add) + m * q.ldz : nullptr, n, q.N, f);
}

// G groups of waves divide the workgroup's channels (one wave on a SIMD waits for its own reads and copies most of the time); their sums meet
// on the way out.  Each has a ring of NB halves, a half being KC channels of its tile's rows of x or of the weight: chunk c's are halves 2 c and
// 2 c + 1 of the sequence, and while it is multiplied halves 2 c + NB - 2 and 2 c + NB - 1 are copied.  (Five halves for 256 x 256 tiles, all of LDS, so
// that copies are in flight across the barrier: 8192 x 4096 x 8192 240.7 us, with four 237.7.)
template <int TI_, int WI, int WJ, int NB_, int G> struct MulCfg {
  static constexpr int NB = NB_, WAVES = (TI_ / WI) * (TI_ / WJ), NT = 64 * WAVES * G, HALF = TI_ * KC;   // WAVES: of a group
  static constexpr int CPH = TI_ / 8 / WAVES;   // copies a wave and half, 8 rows each
  static constexpr int PITCH = WJ * 4 + 16, OUT = G * WAVES * 32 * PITCH;   // sums of 32 rows a wave on their way out
  static constexpr int LDS = G * NB * HALF > OUT ? G * NB * HALF : OUT;
  static_assert(TI_ % (16 * WAVES) == 0 && NB >= 4 && NB % 2 == 0 && LDS <= 160 * 1024, "whole pairs of copies");
};

template <typename T, int TI, int WI, int WJ, int NB, int G, bool SPLIT>
__global__ __launch_bounds__((TI / WI) * (TI / WJ) * 64 * G) void qmul_kernel(MulParams p) {
  using Cfg = MulCfg<TI, WI, WJ, NB, G>;
  constexpr int TJ = TI, FI = WI / 32, FJ = WJ / 32, CPH = Cfg::CPH;
  extern __shared__ __align__(16) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 63, all = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int group = all / Cfg::WAVES, wave = all % Cfg::WAVES;
  unsigned char* const ring = smem + group * NB * Cfg::HALF;
  TileAt t;
  if (!tile_at((int)blockIdx.x, p.nti, p.ntj, p.splits, &t)) return;
  const int split = t.split, j0 = t.j * TJ;
  const i64 i0 = (i64)t.i * TI;
  const int w_beg = split * p.per, w_end = min(p.nch, w_beg + p.per), share = (w_end - w_beg + G - 1) / G;
  const int c_beg = w_beg + group * share, c_end = min(w_end, c_beg + share);   // (all groups take `share` turns)

  // ---- copies: lane l puts 16 codes into piece l % 8 of row l / 8; rows past the end lie past the buffer
  const int rows_a = (int)(p.m.M - i0 < TI ? p.m.M - i0 : TI);
  const int rows_b = min(p.m.N - j0, TJ);
  const i32x4 ra = make_desc(static_cast<const uint8_t*>(p.m.qx) + i0 * p.Kp, rows_a * p.Kp);
  const i32x4 rb = make_desc(static_cast<const uint8_t*>(p.m.qw) + (i64)j0 * p.Kp, rows_b * p.Kp);
  const int g16 = ((lane & 7) ^ (lane >> 4)) * 16;   // (a wave's odd copies: ^ 64)
  unsigned off[CPH];
#pragma unroll
  for (int i = 0; i < CPH; ++i) off[i] = (unsigned)((wave * CPH + i) * 8 + (lane >> 3)) * (unsigned)p.Kp + (g16 ^ (i & 1) * 64);
  const unsigned lds0 = lds_off(ring) + wave * CPH * 1024;
  // (chunks past the end are copied as zeros: every wave has the same copies in flight)
  auto issue = [&](bool weight, int c, int slot, int from, int to) {
    const unsigned k = (unsigned)c * KC;
    const bool in[2] = {c < c_end && (int)k + g16 < p.Kp, c < c_end && (int)k + (g16 ^ 64) < p.Kp};
#pragma unroll
    for (int i = 0; i < CPH; ++i)
      if (i >= from && i < to) dma16(weight ? rb : ra, in[i & 1] ? off[i] + k : OOB, lds0 + slot * Cfg::HALF + i * 1024);
  };

  const int wi = (wave % (TI / WI)) * WI, wj = (wave / (TI / WI)) * WJ, kb = lane >> 5;
  auto at = [&](int first, int step, int f) {   // 16 codes of row l % 32, from 32 step + 16 (l / 32)
    const int row = first + f * 32 + (lane & 31);
    return row * KC + (((step * 2 + kb) ^ ((row >> 1) & 7)) << 4);
  };
  i32x16 acc[FI][FJ];
#pragma unroll
  for (int i = 0; i < FI; ++i)
#pragma unroll
    for (int j = 0; j < FJ; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0;

#pragma unroll
  for (int h = 0; h < NB - 2; ++h) issue(h & 1, c_beg + h / 2, h, 0, CPH);
  int slot = 0;   // of this chunk's rows of x
  for (int c = c_beg; c < c_beg + share; ++c) {
    landed<CPH * (NB - 4)>();   // this chunk's copies, for all waves; and all have read the chunk before
    auto wrap = [](int s) { return s >= NB ? s - NB : s; };
    const unsigned char* cura = ring + slot * Cfg::HALF;
    const unsigned char* curb = ring + wrap(slot + 1) * Cfg::HALF;
    const int first = wrap(slot + NB - 2), second = wrap(slot + NB - 1);
    slot = wrap(slot + 2);
#pragma unroll
    for (int s = 0; s < KC / 32; ++s) {
      // the copies, spread over the chunk's multiplies: all of them behind the barrier keep the waves from their first multiplies
      // (8192 x 4096 x 8192: 246 us; over the first half of the chunk 240, over all of it 237; 128 x 128 tiles, 1568 x 8192 x 2048:
      // 43, 42 and 45)
      constexpr int OVER = TI == 256 ? 2 : 1;   // steps that a half's copies take
      if (s < OVER) issue(false, c + NB / 2 - 1, first, s * CPH / OVER, (s + 1) * CPH / OVER);
      else if (s < 2 * OVER) issue(true, c + NB / 2 - 1, second, (s - OVER) * CPH / OVER, (s - OVER + 1) * CPH / OVER);
      i32x4 af[FI], bf[FJ];
#pragma unroll
      for (int f = 0; f < FI; ++f) af[f] = *reinterpret_cast<const i32x4*>(cura + at(wi, s, f));
#pragma unroll
      for (int f = 0; f < FJ; ++f) bf[f] = *reinterpret_cast<const i32x4*>(curb + at(wj, s, f));
#pragma unroll
      for (int i = 0; i < FI; ++i)
#pragma unroll
        for (int j = 0; j < FJ; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(bf[j], af[i], acc[i][j], 0, 0, 0);
    }
  }
  landed<0>();

  // ---- out, 32 rows of this wave at a time: a lane holds row l % 32 and, for each e / 4, four channels 8 (e / 4) + 4 (l / 32) ..;
  // through LDS they become whole rows (8 bytes a row straight from the registers: 30 % of the pass at 8192 x 4096 x 8192)
  constexpr int LPR = WJ / 8;   // lanes a row, 8 channels each
  unsigned char* mine = smem + all * 32 * Cfg::PITCH;
  auto meet = [] {
    if constexpr (G > 1) __syncthreads();
    else __builtin_amdgcn_wave_barrier();
  };
  const int col = (lane % LPR) * 8, n = j0 + wj + col;
  float sw[8], b[8];
  if constexpr (!SPLIT) {
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      sw[x] = n + x < p.m.N ? p.m.sw[n + x] : 0.f;
      b[x] = p.m.b && n + x < p.m.N ? p.m.b[n + x] : 0.f;
    }
  }
  const bool vec = p.m.N % 4 == 0;   // (of the partial sums)
#pragma unroll
  for (int i = 0; i < FI; ++i) {
#pragma unroll
    for (int j = 0; j < FJ; ++j)
#pragma unroll
      for (int e = 0; e < 16; e += 4)
        *reinterpret_cast<i32x4*>(mine + (lane & 31) * Cfg::PITCH + (j * 32 + 8 * (e >> 2) + 4 * kb) * 4) =
            (i32x4){acc[i][j][e], acc[i][j][e + 1], acc[i][j][e + 2], acc[i][j][e + 3]};
    meet();
    constexpr int RPI = 64 / LPR;   // rows at a time, a group after the other
#pragma unroll
    for (int r0 = 0; r0 < 32; r0 += RPI * G) {
      const int row = r0 + group * RPI + lane / LPR;
      const i64 m = i0 + wi + i * 32 + row;
      int v[8] = {};
#pragma unroll
      for (int o = 0; o < G; ++o)
#pragma unroll
        for (int h = 0; h < 8; h += 4) {
          const i32x4 w = *reinterpret_cast<const i32x4*>(smem + ((o * Cfg::WAVES + wave) * 32 + row) * Cfg::PITCH + (col + h) * 4);
          v[h] += w[0]; v[h + 1] += w[1]; v[h + 2] += w[2]; v[h + 3] += w[3];
        }
      if (m >= p.m.M || n >= p.m.N) continue;
      if constexpr (SPLIT) {
        int* o = p.part + (split * p.m.M + m) * p.m.N + n;
        if (vec && n + 8 <= p.m.N) {
          *reinterpret_cast<int4*>(o) = make_int4(v[0], v[1], v[2], v[3]);
          *reinterpret_cast<int4*>(o + 4) = make_int4(v[4], v[5], v[6], v[7]);
        } else {
#pragma unroll
          for (int x = 0; x < 8; ++x)
            if (n + x < p.m.N) o[x] = v[x];
        }
      } else {
        finish8<T>(p.m, m, n, v, p.m.sx[m], sw, b);
      }
    }
    meet();
  }
}

template <typename T> __global__ __launch_bounds__(256) void qmul_join_kernel(MulParams p) {
  const int oct = (p.m.N + 7) >> 3;
  const i64 total = p.m.M * oct;
  const bool pvec = p.m.N % 8 == 0;
  for (i64 x = (i64)blockIdx.x * 256 + threadIdx.x; x < total; x += (i64)gridDim.x * 256) {
    const i64 m = x / oct;
    const int n = (int)(x - m * oct) * 8;
    int v[8] = {};
    for (int s = 0; s < p.splits; ++s) {
      const int* o = p.part + (s * p.m.M + m) * p.m.N + n;
      if (pvec) {
        const int4 w = *reinterpret_cast<const int4*>(o), u = *reinterpret_cast<const int4*>(o + 4);
        v[0] += w.x; v[1] += w.y; v[2] += w.z; v[3] += w.w; v[4] += u.x; v[5] += u.y; v[6] += u.z; v[7] += u.w;
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (n + i < p.m.N) v[i] += o[i];
      }
    }
    float sw[8], b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      sw[i] = n + i < p.m.N ? p.m.sw[n + i] : 0.f;
      b[i] = p.m.b && n + i < p.m.N ? p.m.b[n + i] : 0.f;
    }
    finish8<T>(p.m, m, n, v, p.m.sx[m], sw, b);
  }
}

constexpr int CUS = 256;

// The cheapest of tiles of 64, 128 and 256, and of 1 to 64 parts of the channel sum, by what was measured in us: a launch 2, every round of
// workgroups 2, 3 or 6 and, for each chunk, 0.18, 0.47 or 1.85 with a workgroup alone on its compute unit, 0.37 or 1.2 with two (64, 128);
// parts cost another launch and their sums' way through memory.  With one group of waves a tile,
// 1568 x 2048 x 512: 64 whole 8.6 (with two 6.7), in two parts 14.1, 128 whole 13.3; 64 x 8192 x 2048: 64 whole 20.6, in four parts 13.3;
// 1568 x 8192 x 2048: 64 51.9, 128 39.5 (36.2 with twice the waves); 100352 x 64 x 256: 64 39.4, 128 23.3;
// 16384 x 1024 x 1024: 128 30.3, 256 26.
struct Plan { int tile, splits, per; };
Plan plan_of(i64 M, int N, int K) {
  const int nch = ceil_div(qrow(K), KC);
  Plan pl = {64, 1, nch};
  if (M == 0) return pl;
  auto tiles = [&](i64 t) { return ((M + t - 1) / t) * ((N + t - 1) / t); };
  double best = 1e30;
  for (int tile = 64; tile <= 256; tile *= 2)
    for (int s = 1; s <= 64 && s <= nch; s *= 2) {
      const int per = ceil_div(nch, s), parts = ceil_div(nch, per);
      const double w = (double)tiles(tile) * parts;
      const bool alone = w <= CUS;
      const double rounds = (double)(i64)(tile == 256 ? (w + 255) / 256 : (w + 511) / 512);
      const double chunk = tile == 256 ? 1.85 : tile == 128 ? (alone ? 0.47 : 1.2) : alone ? 0.18 : 0.37;
      const double us = 2 + rounds * ((tile == 256 ? 6 : tile == 128 ? 3 : 2) + chunk * per) + (parts > 1 ? 4.2 + 2e-6 * parts * (double)M * N : 0);
      if (us < best) {
        best = us;
        pl = {tile, parts, per};
      }
    }
  return pl;
}

template <typename T, int TI, int WI, int WJ, int NB, int G, bool SPLIT> hipError_t launch_tiles(const MulParams& p, hipStream_t st) {
  using Cfg = MulCfg<TI, WI, WJ, NB, G>;
  static LdsLimitOnce once;
  auto* k = &qmul_kernel<T, TI, WI, WJ, NB, G, SPLIT>;
  const hipError_t e = set_lds_limit_once(once, (const void*)k, Cfg::LDS);
  if (e != hipSuccess) return e;
  k<<<(p.nti * p.ntj * p.splits + 7) / 8 * 8, Cfg::NT, Cfg::LDS, st>>>(p);
  return hipGetLastError();
}
template <typename T, bool SPLIT> hipError_t by_tile(int tile, const MulParams& p, hipStream_t st) {
  const bool alone = p.nti * p.ntj * p.splits <= CUS;   // one workgroup a compute unit: its copies are all that hides the way to memory
  if (tile == 256) return launch_tiles<T, 256, 64, 128, 4, 1, SPLIT>(p, st);
  if (tile == 128) return alone ? launch_tiles<T, 128, 32, 64, 8, 1, SPLIT>(p, st) : launch_tiles<T, 128, 64, 64, 4, 1, SPLIT>(p, st);
  return alone ? launch_tiles<T, 64, 32, 32, 8, 2, SPLIT>(p, st) : launch_tiles<T, 64, 32, 32, 8, 1, SPLIT>(p, st);
}
template <typename T> hipError_t mul_t(const MulParams& p, int tile, hipStream_t st) {
  if (p.splits == 1) return by_tile<T, false>(tile, p, st);
  const hipError_t e = by_tile<int, true>(tile, p, st);
  if (e != hipSuccess) return e;
  const i64 blocks = (p.m.M * ((p.m.N + 7) >> 3) + 255) / 256;
  qmul_join_kernel<T><<<(int)(blocks < 65536 ? blocks : 65536), 256, 0, st>>>(p);
  return hipGetLastError();
}

}  // namespace

size_t qmul_scratch(i64 M, int N, int K) {
  const Plan pl = plan_of(M, N, K);
  return pl.splits > 1 ? align_up((size_t)pl.splits * M * N * 4, 256) : 0;
}

hipError_t launch_qmul(const QMul& q, void* ws, hipStream_t st) {
  const Plan pl = plan_of(q.M, q.N, q.K);
  MulParams p = {q, qrow(q.K), ceil_div(qrow(q.K), KC), pl.splits, pl.per, (int)((q.M + pl.tile - 1) / pl.tile), ceil_div(q.N, pl.tile), (int*)ws};
  return q.dtype == CONVBN_BF16 ? mul_t<bf16_t>(p, pl.tile, st) : mul_t<float>(p, pl.tile, st);
}

}  // namespace convbn
