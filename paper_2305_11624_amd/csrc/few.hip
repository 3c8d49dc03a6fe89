// Few rows (single tokens, small batches) through the 8-bit floating-point product and the gated product: bound by the one read of the weight.
//
// A workgroup owns T output channels and its waves divide the input channels, so that the whole chip streams the weight with every load in
// flight at once; there is nothing to join between workgroups.  The matrix instruction is 16 x 16 x 32, channels of the weight against rows
// of x.  Where there are at most T = 8, 4, 2 or 1 rows it runs block-diagonal: its 16 weight rows are T channels at 16 / T places of the
// reduction, its 16 columns T rows of x at the same places, and the T x T blocks on the diagonal are added up at the end.  That way few rows still give many
// workgroups, and a load takes 1024 / T bytes of each weight row in a run.  One row, 2048 -> 8192: gated, 67 MB in 12.6 us, 5.3 TB/s, the rate of a large
// copy; in 8 bits 17 MB in 7.2 us, 2.4 TB/s, of which a launch is 2 - 3.
//
// x lies in LDS as bf16 numbers, put there by every workgroup for itself while its first weights are on the way (a launch of its own would take longer
// than the whole product): rounded to 8 bits as the packed form is, as it is, or, fp32, in three parts that add up to it (and the first once more, where it is finite).  e4m3 weights become bf16 numbers in
// registers, fp32 ones three parts, and sums are fp32 throughout.
#include "f8_code.h"
#include "mm_tile.h"

namespace convbn {

namespace {

// What the weight is held as: bytes and channels of a lane's piece, streams (the gated product has two), parts
struct F8Weight { static constexpr bool F8 = true; static constexpr int CH = 16, STREAMS = 1, PARTS = 1, UNROLL = 8; };
struct BfWeight { static constexpr bool F8 = false; static constexpr int CH = 8, STREAMS = 2, PARTS = 1, UNROLL = 6; using T = bf16_t; };
struct FpWeight { static constexpr bool F8 = false; static constexpr int CH = 8, STREAMS = 2, PARTS = 4, UNROLL = 4; using T = float; };

struct FewParams {
  F8Mul f; Glu g;                   // one of them
  const void* x; i64 ldx;           // null: f.qx, f.sx
  uint8_t* codes; uint8_t* scales;  // where packed rows go if they are kept (null: nowhere)
  i64 M;
  int K, N, T, steps;               // steps of 4 CH * 16 / T channels
  int pitch;                        // of x in LDS, elements
};

// Channels k .. k+7 of a row of the weight, zeros past the end
template <typename T> __device__ __forceinline__ Raw8<T> weight8(const T* row, int k, int K) {
  if (k + 8 <= K) return *reinterpret_cast<const Raw8<T>*>(row + k);
  return narrow<T>(load8<T>(row, k, K));
}

template <class W, typename T, int KIND> __global__ __launch_bounds__(512) void few_kernel(FewParams p) {
  constexpr int CH = W::CH, S = W::STREAMS, U = W::UNROLL, PARTS = W::PARTS;
  extern __shared__ __align__(16) unsigned char smem[];   // x [PARTS][M][pitch]; later sums [waves][S][256]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), waves = blockDim.x >> 6;
  const int n0 = blockIdx.x * p.T, M = (int)p.M, K = p.K, Kp = qrow(K), Sp = f8srow(K);
  const int r = lane & 15, in_part = r & (p.T - 1), part = r / p.T, stride = 4 * CH * 16 / p.T;
  const int k0 = part * 4 * CH + (lane >> 4) * CH, n = n0 + in_part;
  const int width = W::F8 ? Kp : K;

  // ---- weights: U pieces of each stream on the way
  i32x4 q8[U];
  unsigned s8[U];
  using WT = std::conditional_t<W::F8, bf16_t, T>;
  Raw8<WT> w[S][W::F8 ? 1 : U];
  auto fetch = [&](int s0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = (s0 + u * waves) * stride + k0;
      const bool in = n < p.N && k < width;
      if constexpr (W::F8) {
        q8[u] = in ? *reinterpret_cast<const i32x4*>(p.f.qw + (i64)n * Kp + k) : (i32x4){0, 0, 0, 0};
        s8[u] = in ? p.f.sw[(i64)n * Sp + k / BLK] : 127u;
      } else {
#pragma unroll
        for (int x = 0; x < S; ++x)
          w[x][u] = in ? weight8<T>(static_cast<const T*>(p.g.W) + ((i64)x * p.N + n) * K, k, K) : narrow<T>(F8{});
      }
    }
  };
  fetch(wave);

  // ---- x into LDS: pieces of eight channels, zeros past the end
  bf16_t* const xs = reinterpret_cast<bf16_t*>(smem);
  const int wide = p.pitch - 8, pieces = wide / 8;   // (a multiple of 16 for rows that are packed here: their blocks are 16 lanes)
  auto put = [&](int row, int k, const F8& v) { *reinterpret_cast<u32x4*>(xs + row * p.pitch + k) = narrow<bf16_t>(v).a; };
  for (int i = tid; i < M * pieces; i += blockDim.x) {
    const int m = i / pieces, k = (i - m * pieces) * 8;
    if constexpr (W::F8) {
      F8 v = {};
      if (p.x) {
        const F8 f = k < K ? load8<T>(static_cast<const T*>(p.x) + m * p.ldx, k, K) : F8{};
        const unsigned bits = block_max(amax8(f));
        const uint2 c = f8_clip(f8_codes8(f, bits), k, K);
        const int e = f8_exp(bits);
        if (p.codes && blockIdx.x == 0) {
          if (k < Kp) *reinterpret_cast<uint2*>(p.codes + (i64)m * Kp + k) = c;
          if ((k & (BLK - 1)) == 0) p.scales[(i64)m * Sp + k / BLK] = (uint8_t)(e + 127);
        }
        v = f8_decode8(c, two_to(e));
      } else if (k < Kp) {
        v = f8_decode8(*reinterpret_cast<const uint2*>(p.f.qx + (i64)m * Kp + k), scale_of_byte(p.f.sx[(i64)m * Sp + k / BLK]));
      }
      put(m, k, v);
    } else {
      const F8 f = k < K ? load8<T>(static_cast<const T*>(p.x) + m * p.ldx, k, K) : F8{};
      if constexpr (PARTS == 1) {
        put(m, k, f);
      } else {
        const Parts4 q = split3_near(f);
#pragma unroll
        for (int y = 0; y < PARTS; ++y) *reinterpret_cast<u32x4*>(xs + (y * M + m) * p.pitch + k) = q.p[y];
      }
    }
  }
  if (W::F8 && p.x && p.codes && blockIdx.x == 0) {   // scales past the last block, as packing leaves them
    const int blocks = wide / BLK, pad = Sp - blocks;
    for (int i = tid; i < M * pad; i += blockDim.x) p.scales[(i64)(i / pad) * Sp + blocks + i % pad] = 127;
  }
  __syncthreads();

  f32x4 acc[S];
#pragma unroll
  for (int x = 0; x < S; ++x) acc[x] = (f32x4){0.f, 0.f, 0.f, 0.f};
  for (int s0 = wave; s0 < p.steps; s0 += U * waves) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = (s0 + u * waves) * stride + k0;
      auto rows = [&](int y, int at) {   // eight channels of this lane's row of x
        bf16x8 v = {};
        if (in_part < M && k < wide) v = *reinterpret_cast<const bf16x8*>(xs + (y * M + in_part) * p.pitch + k + at);
        return v;
      };
      if constexpr (W::F8) {
        bf16x8 wv[2];
        f8_widen(q8[u], scale_of_byte(s8[u]), wv);
#pragma unroll
        for (int h = 0; h < 2; ++h) acc[0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv[h], rows(0, 8 * h), acc[0], 0, 0, 0);
      } else if constexpr (PARTS == 1) {
        const bf16x8 xv = rows(0, 0);
#pragma unroll
        for (int x = 0; x < S; ++x) {
          const u32x4 a = w[x][u].a;
          acc[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), xv, acc[x], 0, 0, 0);
        }
      } else {
        const bf16x8 xv[PARTS] = {rows(0, 0), rows(1, 0), rows(2, 0), rows(3, 0)};
#pragma unroll
        for (int x = 0; x < S; ++x) {
          const Parts4 q = split3_near(widen(w[x][u]));
          bf16x8 wv[PARTS];
#pragma unroll
          for (int y = 0; y < PARTS; ++y) wv[y] = __builtin_bit_cast(bf16x8, q.p[y]);
#pragma unroll
          for (int pr = 0; pr < 6; ++pr)
            acc[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv[Parts<6>::B >> (2 * pr) & 3], xv[Parts<6>::A >> (2 * pr) & 3], acc[x], 0, 0, 0);
        }
      }
    }
    if (s0 + U * waves < p.steps) fetch(s0 + U * waves);
  }
  __syncthreads();   // (the sums take x's place)
  // a lane holds column l % 16 (a row of x), weight rows 4 (l / 16) ..
  float* const sums = reinterpret_cast<float*>(smem);
#pragma unroll
  for (int x = 0; x < S; ++x)
#pragma unroll
    for (int i = 0; i < 4; ++i) sums[((wave * S + x) * 16 + (lane & 15)) * 16 + 4 * (lane >> 4) + i] = acc[x][i];
  __syncthreads();
  for (int o = tid; o < M * p.T; o += blockDim.x) {
    const int m = o / p.T, c = o & (p.T - 1), j = n0 + c;
    if (j >= p.N) continue;
    float v[S] = {};
    for (int wv = 0; wv < waves; ++wv)
      for (int q = 0; q < 16; q += p.T)
#pragma unroll
        for (int x = 0; x < S; ++x) v[x] += sums[((wv * S + x) * 16 + q + m) * 16 + q + c];
    if constexpr (W::F8) {
      float z = v[0] + (p.f.b ? p.f.b[j] : 0.f);
      if (p.f.add) z += to_f32(static_cast<const T*>(p.f.add)[m * p.f.ldz + j]);
      static_cast<T*>(p.f.z)[m * p.f.ldz + j] = from_f32<T>(z);
    } else {
      const float g = v[0] + (p.g.b ? p.g.b[j] : 0.f), u = v[S - 1] + (p.g.b ? p.g.b[p.N + j] : 0.f);
      if (p.g.h) {
        const i64 at = (i64)m * 2 * p.N + j;
        p.g.h[at] = g;
        p.g.h[at + p.N] = u;
      }
      float f, df;
      gate_of<T, KIND>(g, &f, &df);
      if (p.g.y) static_cast<T*>(p.g.y)[m * p.g.ldz + j] = from_f32<T>(f * u);
    }
  }
}

// Rows this way, as long as every workgroup's own x takes no more LDS than this; fp32 rows, which the tiles want copies of, more.  us, this and
// the tiles, gated and 8 bits: one row 2048 -> 8192 12.6 and 12.8, 7.2 and 9.6; one row 4096 -> 1024 7.0 and 12.6, 5.9 and 10.2; 16 rows 512 -> 4096 5.0 and 5.7, 5.9
// and 6.9; with twice as much 8 rows 4096 -> 4096 17.3 and 16.6, 14.4 and 12.8.
constexpr int MOST = 16;
constexpr int lds_x(int parts) { return (parts == 1 ? 34 : 90) * 1024; }
int pitch_of(int K, bool f8) { return (f8 ? (K + BLK - 1) / BLK * BLK : (K + 15) & ~15) + 8; }   // (8 more: rows on other banks)
bool fits(i64 M, int K, int parts, bool f8) { return M > 0 && M <= MOST && (i64)M * pitch_of(K, f8) * 2 * parts <= lds_x(parts); }

template <class W, typename T, int KIND> hipError_t launch(FewParams p, hipStream_t st) {
  p.pitch = pitch_of(p.K, W::F8);
  p.T = 16;
  // as few channels a workgroup as the rows allow until there is one for each compute unit, and 2048 waves in all.  us, gated and 8 bits, T and waves: one
  // row 2048 -> 8192 16 of 4 12.9 and 7.1, 16 of 8 12.6 and 8.0, 4 of 4 13.2 and 11.6, 1 of 4 31; one row 4096 -> 1024 4 of 4 6.8 and 5.6, 16 of 4 12.9 and 8.7; 4 rows 2048 -> 2048 8 of 8 6.7
  // and 6.3, 4 of 4 7.2 and 7.6.
  while (p.T / 2 >= p.M && ceil_div(p.N, p.T) < 256) p.T /= 2;
  const int grid = ceil_div(p.N, p.T);
  p.steps = ceil_div(W::F8 ? qrow(p.K) : p.K, 4 * W::CH * 16 / p.T);
  const int waves = grid <= 256 ? 8 : grid >= 512 ? 4 : 2048 / grid;
  const int x = (int)p.M * p.pitch * 2 * W::PARTS, sums = waves * W::STREAMS * 1024;
  static LdsLimitOnce once;
  auto* k = &few_kernel<W, T, KIND>;
  const hipError_t e = set_lds_limit_once(once, (const void*)k, lds_x(W::PARTS) < 64 * 1024 ? 64 * 1024 : lds_x(W::PARTS));
  if (e != hipSuccess) return e;
  k<<<grid, waves * 64, x > sums ? x : sums, st>>>(p);
  return hipGetLastError();
}

}  // namespace

bool f8few_taken(i64 M, int K) { return fits(M, K, 1, true); }
hipError_t launch_f8few(const F8Mul& f, const void* x, i64 ldx, void* codes, void* scales, hipStream_t st) {
  FewParams p = {};
  p.f = f; p.x = x; p.ldx = ldx; p.codes = (uint8_t*)codes; p.scales = (uint8_t*)scales;
  p.M = f.M; p.K = f.K; p.N = f.N;
  return f.dtype == CONVBN_BF16 ? launch<F8Weight, bf16_t, 0>(p, st) : launch<F8Weight, float, 0>(p, st);
}

bool glu_few_taken(i64 M, int K, int dtype) { return fits(M, K, dtype == CONVBN_BF16 ? 1 : FpWeight::PARTS, false); }
hipError_t launch_glu_few(const Glu& g, hipStream_t st) {
  FewParams p = {};
  p.g = g; p.x = g.x; p.ldx = g.ldx;
  p.M = g.M; p.K = g.K; p.N = g.N;
  if (g.dtype == CONVBN_BF16) return g.gate == CONVBN_GATE_SILU ? launch<BfWeight, bf16_t, 0>(p, st) : launch<BfWeight, bf16_t, 1>(p, st);
  return g.gate == CONVBN_GATE_SILU ? launch<FpWeight, float, 0>(p, st) : launch<FpWeight, float, 1>(p, st);
}

}  // namespace convbn
