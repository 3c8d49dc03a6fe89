// z = sx sw (qx . qw) + b + add: the product of 8-bit integers with a scale for each row of either operand.
//
// Both operands' channels run together, which is what the matrix instruction wants; they pass through LDS as rows of 128 codes whose
// 16-byte pieces are exchanged by the row's low bits, so that 16 lanes reading a column of pieces meet distinct banks.  Sums over
// channels that are split between workgroups stay whole numbers: any order gives the same.
#include "quant.h"

namespace convbn {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

constexpr unsigned OOB = 0x80000000u;   // beyond any buffer: the load returns zeros
constexpr int KC = 128;                 // channels at a time

__device__ __forceinline__ __amdgpu_buffer_rsrc_t make_rsrc(const void* p, i64 bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (int)(bytes > 0x7ffffff0LL ? 0x7ffffff0LL : bytes), 0x00020000);
}

struct MulParams {
  QMul m;
  int Kp, nch, splits, per;   // chunks of KC, chunks of a split
  int nti, ntj;
  int* part;                  // [splits][M][N], where there are several
};

// Four channels n .. n+3 of row m: scaled, with bias and addend, rounded once
template <typename T> __device__ __forceinline__ void finish4(const QMul& q, i64 m, int n, const int (&acc)[4], float sx, bool vec) {
  T* z = static_cast<T*>(q.z) + m * q.ldz + n;
  const T* add = q.add ? static_cast<const T*>(q.add) + m * q.ldz + n : nullptr;
  float v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool in = n + i < q.N;
    v[i] = (float)acc[i] * (sx * (in ? q.sw[n + i] : 0.f)) + (q.b && in ? q.b[n + i] : 0.f);
  }
  if (vec && n + 4 <= q.N) {
    if constexpr (sizeof(T) == 2) {
      if (add) {
        const uint2 w = *reinterpret_cast<const uint2*>(add);
        v[0] += bf16_lo(w.x); v[1] += bf16_hi(w.x); v[2] += bf16_lo(w.y); v[3] += bf16_hi(w.y);
      }
      *reinterpret_cast<uint2*>(z) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
    } else {
      if (add) {
        const float4 w = *reinterpret_cast<const float4*>(add);
        v[0] += w.x; v[1] += w.y; v[2] += w.z; v[3] += w.w;
      }
      *reinterpret_cast<float4*>(z) = make_float4(v[0], v[1], v[2], v[3]);
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (n + i < q.N) z[i] = from_f32<T>(v[i] + (add ? to_f32(add[i]) : 0.f));
}
template <typename T> __device__ __forceinline__ bool vectors(const QMul& q) {
  return ((uintptr_t)q.z | (uintptr_t)(q.ldz * sizeof(T)) | (uintptr_t)q.add) % (4 * sizeof(T)) == 0;
}

template <int TI, int TJ, int WI, int WJ> struct MulCfg {
  static constexpr int NT = 64 * (TI / WI) * (TJ / WJ), STAGE = (TI + TJ) * KC, LDS = 2 * STAGE;
};

template <typename T, int TI, int TJ, int WI, int WJ, bool SPLIT>
__global__ __launch_bounds__((TI / WI) * (TJ / WJ) * 64) void qmul_kernel(MulParams p) {
  using Cfg = MulCfg<TI, TJ, WI, WJ>;
  constexpr int NT = Cfg::NT, FI = WI / 32, FJ = WJ / 32, PA = TI * 8 / NT, PB = TJ * 8 / NT;
  extern __shared__ __align__(16) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int total = p.nti * p.ntj * p.splits, run = (total + 7) >> 3;   // contiguous runs of tiles to each XCD
  const int id = ((int)blockIdx.x & 7) * run + ((int)blockIdx.x >> 3);
  if (((int)blockIdx.x >> 3) >= run || id >= total) return;
  const int split = id / (p.nti * p.ntj), tile = id - split * (p.nti * p.ntj);
  const i64 i0 = (i64)(tile % p.nti) * TI;
  const int j0 = tile / p.nti * TJ;
  const int c_beg = split * p.per, c_end = min(p.nch, c_beg + p.per);

  const i64 rows_a = p.m.M - i0 < TI ? p.m.M - i0 : TI;
  const int rows_b = min(p.m.N - j0, TJ);
  const __amdgpu_buffer_rsrc_t ra = make_rsrc(static_cast<const uint8_t*>(p.m.qx) + i0 * p.Kp, rows_a * p.Kp);
  const __amdgpu_buffer_rsrc_t rb = make_rsrc(static_cast<const uint8_t*>(p.m.qw) + (i64)j0 * p.Kp, (i64)rows_b * p.Kp);
  // piece w of a chunk: row w / 8, 16 codes from 16 (w % 8); rows past the end lie past the buffer
  const int g = tid & 7, row0 = tid >> 3;
  const unsigned off0 = (unsigned)(row0 * p.Kp + g * 16), step = (unsigned)(NT / 8) * (unsigned)p.Kp;
  const unsigned lds0 = row0 * KC + ((g ^ (row0 & 7)) << 4);
  static_assert(NT / 8 % 8 == 0, "a thread's pieces are exchanged alike");
  i32x4 a_reg[PA], b_reg[PB];
  auto fetch = [&](int c) {
    const unsigned k = (unsigned)c * KC;
    const bool in = (int)k + g * 16 < p.Kp;
#pragma unroll
    for (int t = 0; t < PA; ++t) a_reg[t] = __builtin_amdgcn_raw_buffer_load_b128(ra, (int)(in ? off0 + t * step + k : OOB), 0, 0);
#pragma unroll
    for (int t = 0; t < PB; ++t) b_reg[t] = __builtin_amdgcn_raw_buffer_load_b128(rb, (int)(in ? off0 + t * step + k : OOB), 0, 0);
  };
  auto put = [&](unsigned char* stage) {
#pragma unroll
    for (int t = 0; t < PA; ++t) *reinterpret_cast<i32x4*>(stage + lds0 + t * (NT / 8) * KC) = a_reg[t];
#pragma unroll
    for (int t = 0; t < PB; ++t) *reinterpret_cast<i32x4*>(stage + TI * KC + lds0 + t * (NT / 8) * KC) = b_reg[t];
  };

  const int wi = (wave % (TI / WI)) * WI, wj = (wave / (TI / WI)) * WJ, kb = lane >> 5;
  auto at = [&](int first, int step_, int f) {   // 16 codes of row l % 32, from 32 step + 16 (l / 32)
    const int row = first + f * 32 + (lane & 31);
    return row * KC + (((step_ * 2 + kb) ^ (row & 7)) << 4);
  };
  i32x16 acc[FI][FJ];
#pragma unroll
  for (int i = 0; i < FI; ++i)
#pragma unroll
    for (int j = 0; j < FJ; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0;

  fetch(c_beg);
  put(smem);
  if (c_beg + 1 < c_end) fetch(c_beg + 1);
  __syncthreads();
  for (int c = c_beg; c < c_end; ++c) {
    const unsigned char* cur = smem + ((c - c_beg) & 1) * Cfg::STAGE;
    if (c + 1 < c_end) {
      put(smem + ((c - c_beg + 1) & 1) * Cfg::STAGE);
      if (c + 2 < c_end) fetch(c + 2);
    }
#pragma unroll
    for (int s = 0; s < KC / 32; ++s) {
      i32x4 af[FI], bf[FJ];
#pragma unroll
      for (int f = 0; f < FI; ++f) af[f] = *reinterpret_cast<const i32x4*>(cur + at(wi, s, f));
#pragma unroll
      for (int f = 0; f < FJ; ++f) bf[f] = *reinterpret_cast<const i32x4*>(cur + TI * KC + at(wj, s, f));
#pragma unroll
      for (int i = 0; i < FI; ++i)
#pragma unroll
        for (int j = 0; j < FJ; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(bf[j], af[i], acc[i][j], 0, 0, 0);
    }
    __syncthreads();
  }

  // a lane holds row l % 32 and, for each e / 4, four channels 8 (e / 4) + 4 (l / 32) ..
  const bool vec = SPLIT ? p.m.N % 4 == 0 : vectors<T>(p.m);
#pragma unroll
  for (int i = 0; i < FI; ++i) {
    const i64 m = i0 + wi + i * 32 + (lane & 31);
    if (m >= p.m.M) continue;
    const float sx = SPLIT ? 0.f : p.m.sx[m];
#pragma unroll
    for (int j = 0; j < FJ; ++j)
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        const int n = j0 + wj + j * 32 + 8 * (e >> 2) + 4 * kb;
        if (n >= p.m.N) continue;
        const int v[4] = {acc[i][j][e], acc[i][j][e + 1], acc[i][j][e + 2], acc[i][j][e + 3]};
        if constexpr (SPLIT) {
          int* o = p.part + (split * p.m.M + m) * p.m.N + n;
          if (vec) {
            *reinterpret_cast<int4*>(o) = make_int4(v[0], v[1], v[2], v[3]);
          } else {
#pragma unroll
            for (int x = 0; x < 4; ++x)
              if (n + x < p.m.N) o[x] = v[x];
          }
        } else {
          finish4<T>(p.m, m, n, v, sx, vec);
        }
      }
  }
}

template <typename T> __global__ __launch_bounds__(256) void qmul_join_kernel(MulParams p) {
  const int quads = (p.m.N + 3) >> 2;
  const i64 total = p.m.M * quads;
  const bool vec = vectors<T>(p.m), pvec = p.m.N % 4 == 0;
  for (i64 x = (i64)blockIdx.x * 256 + threadIdx.x; x < total; x += (i64)gridDim.x * 256) {
    const i64 m = x / quads;
    const int n = (int)(x - m * quads) * 4;
    int v[4] = {0, 0, 0, 0};
    for (int s = 0; s < p.splits; ++s) {
      const int* o = p.part + (s * p.m.M + m) * p.m.N + n;
      if (pvec) {
        const int4 w = *reinterpret_cast<const int4*>(o);
        v[0] += w.x; v[1] += w.y; v[2] += w.z; v[3] += w.w;
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (n + i < p.m.N) v[i] += o[i];
      }
    }
    finish4<T>(p.m, m, n, v, p.m.sx[m], vec);
  }
}

constexpr int CUS = 256;

struct Plan { int tile, splits, per; };   // tile: 256, 128 or 64 rows and channels
Plan plan_of(i64 M, int N, int K) {
  Plan pl = {64, 1, 1};
  auto tiles = [&](i64 t) { return ((M + t - 1) / t) * ((N + t - 1) / t); };
  const int nch = ceil_div(qrow(K), KC);
  pl.per = nch;
  if (M == 0) return pl;
  pl.tile = tiles(256) >= CUS ? 256 : M > 64 && tiles(128) >= CUS / 4 ? 128 : 64;
  const i64 t = tiles(pl.tile);
  const i64 want = pl.tile == 64 ? 2 * CUS : CUS;
  i64 s = t < want ? want / t : 1;
  if (s > nch / 2) s = nch / 2;
  if (s < 1) s = 1;
  pl.per = (int)((nch + s - 1) / s);
  pl.splits = ceil_div(nch, pl.per);
  return pl;
}

template <typename T, int TI, int TJ, int WI, int WJ, bool SPLIT> hipError_t launch_tiles(const MulParams& p, hipStream_t st) {
  using Cfg = MulCfg<TI, TJ, WI, WJ>;
  static LdsLimitOnce once;
  auto* k = &qmul_kernel<T, TI, TJ, WI, WJ, SPLIT>;
  const hipError_t e = set_lds_limit_once(once, (const void*)k, Cfg::LDS);
  if (e != hipSuccess) return e;
  k<<<(p.nti * p.ntj * p.splits + 7) / 8 * 8, Cfg::NT, Cfg::LDS, st>>>(p);
  return hipGetLastError();
}
template <typename T, bool SPLIT> hipError_t by_tile(int tile, const MulParams& p, hipStream_t st) {
  if (tile == 256) return launch_tiles<T, 256, 256, 64, 128, SPLIT>(p, st);
  if (tile == 128) return launch_tiles<T, 128, 128, 64, 64, SPLIT>(p, st);
  return launch_tiles<T, 64, 64, 32, 32, SPLIT>(p, st);
}
template <typename T> hipError_t mul_t(const MulParams& p, int tile, hipStream_t st) {
  if (p.splits == 1) return by_tile<T, false>(tile, p, st);
  const hipError_t e = by_tile<int, true>(tile, p, st);
  if (e != hipSuccess) return e;
  const i64 blocks = (p.m.M * ((p.m.N + 3) >> 2) + 255) / 256;
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
