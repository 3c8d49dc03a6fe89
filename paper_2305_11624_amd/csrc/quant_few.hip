// The 8-bit product for few rows (single tokens, small batches): bound by the one read of the weight.
//
// A workgroup owns T output channels and its waves divide the input channels, so that the whole chip streams the weight with every
// load in flight at once; there is nothing to join between workgroups.  The matrix instruction is 16 x 16 x 64, channels of the weight
// against rows of x.  Where there are at most T = 8, 4, 2 or 1 rows it runs block-diagonal: its 16 weight rows are T channels at 16 / T
// places of the reduction, its 16 columns T rows of x at the same places, and the T x T blocks on the diagonal are added up at the end.
// That way few rows still give many workgroups, and a load takes 64 * 16 / T bytes of each weight row in a run.
//
// One row, 2048 -> 8192: 16.8 MB in 6.0 us, packing and launch included, 2.8 TB/s: the weights' way from memory (about 3.3 us at a copy's rate)
// behind the row's own and its maximum.
//
// x that is not packed yet is packed here, by every workgroup for itself while its first weights are on the way (a launch of its own would
// take longer than the whole product), as long as it is short.
#include "quant_code.h"

namespace convbn {

namespace {

constexpr int unroll_of(int NB) { return NB == 1 ? 8 : 4; }   // weight pieces a lane has in flight (and as many of each block of x)

struct FewParams {
  QMul m;
  const void* x; i64 ldx;           // rows to pack (null: m.qx, m.sx are given)
  uint8_t* codes; float* scales;    // where they go if they are kept (null: nowhere)
  int Kp, T, steps;                 // steps of 64 * 16 / T channels
};

// NB: blocks of 16 rows of x (T == 16 where there are several).  PACK: x comes as T.
template <typename T, int NB, bool PACK>
__global__ __launch_bounds__(1024) void qfew_kernel(FewParams p) {
  constexpr int UNROLL = unroll_of(NB);
  extern __shared__ __align__(16) unsigned char smem[];   // [waves][NB][256] sums; PACK: then codes [M][Kp], scales [16]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), waves = blockDim.x >> 6;
  const int n0 = blockIdx.x * p.T, M = (int)p.m.M;
  const int r = lane & 15, in_part = r & (p.T - 1), part = r / p.T, stride = 64 * 16 / p.T;
  const int k0 = part * 64 + (lane >> 4) * 16;
  const __amdgpu_buffer_rsrc_t rw = make_rsrc(static_cast<const uint8_t*>(p.m.qw) + (i64)n0 * p.Kp, (i64)(p.m.N - n0) * p.Kp);
  const unsigned w_off = (unsigned)in_part * (unsigned)p.Kp + k0;
  const __amdgpu_buffer_rsrc_t rx = make_rsrc(p.m.qx, PACK ? 0 : (i64)M * p.Kp);
  const unsigned x_off = (unsigned)in_part * (unsigned)p.Kp + k0;
  i32x4 w[UNROLL], xv[PACK ? 1 : UNROLL][NB];
  auto fetch = [&](int s0) {
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const int k = (s0 + u * waves) * stride;
      w[u] = __builtin_amdgcn_raw_buffer_load_b128(rw, (int)(k + k0 < p.Kp ? w_off + k : OOB), 0, 0);
      if constexpr (!PACK) {   // (rows past M lie past the buffer)
#pragma unroll
        for (int b = 0; b < NB; ++b)
          xv[u][b] = __builtin_amdgcn_raw_buffer_load_b128(rx, (int)(k + k0 < p.Kp ? x_off + b * 16 * p.Kp + k : OOB), 0, 0);
      }
    }
  };
  fetch(wave);

  int* sums = reinterpret_cast<int*>(smem);
  uint8_t* own = smem + waves * NB * 1024;
  float* own_s = reinterpret_cast<float*>(own + M * p.Kp);
  if constexpr (PACK) {   // rows in turn to groups of `per` waves; their maxima meet where the sums go later
    const int groups = min(waves, M), per = waves / groups;   // (waves beyond groups * per pack nothing)
    const int group = wave / per, first = ((wave % per) * 64 + lane) * 8, hop = per * 512;
    auto piece = [&](int m, int k) {
      const T* x = static_cast<const T*>(p.x) + m * p.ldx;
      return load8<T>(x, k, p.m.K);
    };
    if (group < groups)
      for (int m = group; m < M; m += groups) {
        unsigned mx = 0;
        for (int k = first; k < p.m.K; k += hop) mx = max(mx, amax8(piece(m, k)));
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) mx = max(mx, (unsigned)__shfl_xor((int)mx, off, 64));
        if (lane == 0) sums[m * 16 + wave % per] = (int)mx;
      }
    __syncthreads();
    if (group < groups)
      for (int m = group; m < M; m += groups) {
        unsigned mx = 0;
        for (int i = 0; i < per; ++i) mx = max(mx, (unsigned)sums[m * 16 + i]);
        const Scale sc = scale_of(mx);
        for (int k = first; k < p.Kp; k += hop) {
          const uint2 c = codes8(piece(m, k), sc.r);
          *reinterpret_cast<uint2*>(own + m * p.Kp + k) = c;
          if (p.codes && blockIdx.x == 0) *reinterpret_cast<uint2*>(p.codes + m * p.Kp + k) = c;
        }
        if (first == 0) {
          own_s[m] = sc.s;
          if (p.codes && blockIdx.x == 0) p.scales[m] = sc.s;
        }
      }
    __syncthreads();
  }

  i32x4 acc[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) acc[b] = (i32x4){0, 0, 0, 0};
  for (int s0 = wave; s0 < p.steps; s0 += UNROLL * waves) {
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const int k = (s0 + u * waves) * stride + k0;
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        i32x4 v = {0, 0, 0, 0};
        if constexpr (!PACK) v = xv[u][b];
        else if (in_part < M && k < p.Kp) v = *reinterpret_cast<const i32x4*>(own + in_part * p.Kp + k);
        acc[b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[u], v, acc[b], 0, 0, 0);
      }
    }
    if (s0 + UNROLL * waves < p.steps) fetch(s0 + UNROLL * waves);
  }
  // a lane holds column l % 16 (a row of x), weight rows 4 (l / 16) ..
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int i = 0; i < 4; ++i) sums[((wave * NB + b) * 16 + (lane & 15)) * 16 + 4 * (lane >> 4) + i] = acc[b][i];
  __syncthreads();
  const int rows = NB * (NB > 1 ? 16 : p.T);
  for (int o = tid; o < rows * p.T; o += blockDim.x) {
    const int m = o / p.T, c = o & (p.T - 1), n = n0 + c;
    if (m >= M || n >= p.m.N) continue;
    const int b = m >> 4, mm = m & 15;
    int v = 0;
    for (int wv = 0; wv < waves; ++wv)
      for (int q = 0; q < 16; q += p.T) v += sums[((wv * NB + b) * 16 + q + mm) * 16 + q + c];
    const float sx = PACK ? own_s[m] : p.m.sx[m];
    const float sw = p.m.sw[n], bias = p.m.b ? p.m.b[n] : 0.f;
    float z = scale_last(sx) ? (float)v * sw * sx + bias : (float)v * sx * sw + bias;
    if (p.m.add) z += to_f32(static_cast<const T*>(p.m.add)[m * p.m.ldz + n]);
    static_cast<T*>(p.m.z)[m * p.m.ldz + n] = from_f32<T>(z);
  }
}

// Rows this way.  us, this and the tiles of quant_mm.hip: 4096 x 4096, 24 rows 9.6 and 11.5, 32 rows 9.8 and 12.2; with up to 64, 48 rows took
// 12.9 and 13.6, 64 rows 14.7 and 14.7, 64 rows 8192 -> 2048 21.2 and 16.7.
constexpr int MOST = 32;
// Codes that a workgroup packs for itself: us with the packing inside and as a launch of its own: one row 2048 -> 8192 6.3 and 8.0, one row
// 8192 -> 2048 8.1 and 8.5, 4 rows 4096 -> 4096 9.8 and 8.3, 8 rows 2048 -> 8192 10.2 and 8.1.
constexpr int PACK_BYTES = 1 << 13;

template <typename T, int NB, bool PACK> hipError_t launch_few(const FewParams& p, int grid, int waves, hipStream_t st) {
  const int lds = waves * NB * 1024 + (PACK ? (int)p.m.M * p.Kp + 64 : 0);
  qfew_kernel<T, NB, PACK><<<grid, waves * 64, lds, st>>>(p);
  return hipGetLastError();
}
template <typename T> hipError_t few_t(const FewParams& p, int grid, int waves, hipStream_t st) {
  if (p.x) return launch_few<T, 1, true>(p, grid, waves, st);
  return p.m.M <= 16 ? launch_few<T, 1, false>(p, grid, waves, st) : launch_few<T, 2, false>(p, grid, waves, st);
}

}  // namespace

bool qfew_taken(i64 M, int N, int K) { return M > 0 && M <= MOST; }
bool qfew_packs(i64 M, int N, int K) { return M <= 16 && M * qrow(K) <= PACK_BYTES; }

hipError_t launch_qfew(const QMul& q, const void* x, i64 ldx, void* codes, float* scales, hipStream_t st) {
  FewParams p = {q, x, ldx, (uint8_t*)codes, scales, qrow(q.K), 16, 0};
  // as few channels a workgroup as the rows allow, until there are two workgroups a compute unit
  while (p.T / 2 >= q.M && ceil_div(q.N, p.T) < 512) p.T /= 2;
  const int stride = 64 * 16 / p.T;
  p.steps = ceil_div(p.Kp, stride);
  int waves = ceil_div(p.steps, unroll_of(q.M <= 16 ? 1 : 2));   // a wave's share is one batch of loads, if that gives at most 16 waves
  waves = waves < 4 ? 4 : waves > 16 ? 16 : waves;
  const int grid = ceil_div(q.N, p.T);
  return q.dtype == CONVBN_BF16 ? few_t<bf16_t>(p, grid, waves, st) : few_t<float>(p, grid, waves, st);
}

}  // namespace convbn
