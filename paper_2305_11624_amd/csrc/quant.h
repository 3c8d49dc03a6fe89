// 8-bit rows: what the kernels of quant_rows.hip, quant_mm.hip, quant_few.hip and quant_grad.hip share, and their launchers.
#pragma once
#include "common.h"

namespace convbn {

typedef long long i64;

// Bytes from one row of codes to the next: whole 16-byte pieces, zero past the last channel.
inline __host__ __device__ int qrow(int channels) { return (channels + 15) & ~15; }

typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr unsigned OOB = 0x80000000u;   // an offset beyond any buffer: the load returns zeros
// `bytes` (at most 2^31 - 16 of them) from p on, for loads into registers
__device__ __forceinline__ __amdgpu_buffer_rsrc_t make_rsrc(const void* p, i64 bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (int)(bytes > 0x7ffffff0LL ? 0x7ffffff0LL : bytes), 0x00020000);
}

// ---- copies from memory into LDS.  Inline asm: what the compiler knows to be such a copy it waits for before every LDS read.  Nothing is
// returned in registers.  Five wait states in front: a vector memory instruction must not follow sooner where a vector instruction wrote one
// of its scalar registers, and inside asm nobody else counts them (0.3 - 1 % of a pass).
// `bytes` from p on as a buffer; loads past it return zeros
__device__ __forceinline__ i32x4 make_desc(const void* p, int bytes) {
  const uint64_t a = (uint64_t)p;
  return (i32x4){__builtin_amdgcn_readfirstlane((int)(uint32_t)a), __builtin_amdgcn_readfirstlane((int)(uint32_t)(a >> 32) & 0xffff),
                 __builtin_amdgcn_readfirstlane(bytes), 0x00020000};
}
__device__ __forceinline__ unsigned lds_off(const void* p) { return (unsigned)(size_t)(__attribute__((address_space(3))) const void*)p; }
// 16 bytes a lane, lane l's to lds + 16 l (lds: the same for the whole wave)
__device__ __forceinline__ void dma16(i32x4 desc, unsigned voff, unsigned lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               ::"s"(__builtin_amdgcn_readfirstlane(lds)), "v"(voff), "s"(desc));   // (m0 holds nothing between instructions that need it)
}
// ... 4 bytes a lane
__device__ __forceinline__ void dma4(i32x4 desc, unsigned voff, unsigned lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dword %1, %2, 0 offen lds"
               ::"s"(__builtin_amdgcn_readfirstlane(lds)), "v"(voff), "s"(desc));
}
// Until at most N of this wave's copies and loads are in flight; then the workgroup's barrier
template <int N> __device__ __forceinline__ void landed() {
  static_assert(N >= 0 && N < 64, "vmcnt is a 6-bit field");
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// Tile (i, j) of nti x ntj and split of workgroup wg; false: none.  Workgroups go to the eight XCDs in turn, so each gets a contiguous run
// of the order, and the order walks bands of 8 rows of tiles: the 32 workgroups that an XCD runs at a time are about 8 x 4 tiles, which
// share what they read in its cache.
struct TileAt { int i, j, split; };
__device__ __forceinline__ bool tile_at(int wg, int nti, int ntj, int splits, TileAt* at) {
  const int total = nti * ntj * splits, run = (total + 7) >> 3, slot = wg >> 3;
  const int id = (wg & 7) * run + slot;
  if (slot >= run || id >= total) return false;
  at->split = id / (nti * ntj);
  const int tile = id - at->split * (nti * ntj), band = tile / (8 * ntj), in = tile - band * 8 * ntj;
  const int h = min(8, nti - band * 8);
  at->j = in / h;
  at->i = band * 8 + in - at->j * h;
  return true;
}

// ---- rows (quant_rows.hip): ld* in elements ----
hipError_t launch_qpack(int dtype, i64 rows, int K, i64 ld, const void* x, void* codes, float* scales, hipStream_t st);
hipError_t launch_qunpack(int dtype, i64 rows, int K, i64 ld, const void* codes, const float* scales, void* x, hipStream_t st);
// h_codes / h_scales, y, y_codes / y_scales: null = not wanted
hipError_t launch_qgate_fwd(int dtype, int kind, i64 rows, int K, i64 ldh, i64 ldy, const void* h, void* h_codes, float* h_scales,
                            void* y, void* y_codes, float* y_scales, hipStream_t st);
hipError_t launch_qgate_bwd(int dtype, int kind, i64 rows, int K, i64 ldh, i64 ldy, const void* h_codes, const float* h_scales,
                            const void* dy, void* dh, hipStream_t st);

// ---- products ----
// z [M][N] (ldz apart) = sx sw (qx . qw) + b + add
struct QMul {
  i64 M, ldz;
  int K, N, dtype;
  const void* qx; const float* sx; const void* qw; const float* sw; const float* b; const void* add;
  void* z;
};
size_t qmul_scratch(i64 M, int N, int K);
hipError_t launch_qmul(const QMul& p, void* ws, hipStream_t st);

// The same for few rows (quant_few.hip), which it can pack itself where qfew_packs(): x != null, codes and scales null = not kept
bool qfew_taken(i64 M, int N, int K);
bool qfew_packs(i64 M, int N, int K);
hipError_t launch_qfew(const QMul& p, const void* x, i64 ldx, void* codes, float* scales, hipStream_t st);

// dx [M][K] = dz . (sw qw) + add, dW [N][K] = dz^T . (sx qx), db = column sums of dz; dx, dW, db nullable
struct QGrad {
  i64 M, ldx, ldz;
  int K, N, dtype;
  const void* qx; const float* sx; const void* qw; const float* sw; const void* dz; const void* add;
  void* dx; void* dW; float* db;
};
bool qgrad_reads_in_place(int dtype, int N, i64 ldz);   // dz on 16 bytes then
size_t qgrad_scratch(const QGrad& p);
hipError_t launch_qgrad(const QGrad& p, void* ws, hipStream_t st);

// api.hip: keeps the message for convbn_last_error and returns the code
convbn_status set_error(convbn_status code, const char* fmt, ...);

}  // namespace convbn
