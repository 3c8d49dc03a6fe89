// Rows in 8-bit floating point: packing and reading back.  A block of 128 channels is 16 lanes of eight, held in registers from the one read to
// the store of its codes; nothing is shared beyond these lanes, so rows of any length are packed alike.  Bound by memory: 8192 x 4096 bf16, 67 MB in and 34 out, 17 - 20 us,
// read back 17; fp32 25 and 26.
#include "f8_code.h"

namespace convbn {

namespace {

constexpr int NT = 256;

struct RowArgs { i64 rows, ld; int K; const void* x; void* out; uint8_t* codes; uint8_t* scales; };

template <typename T> __global__ __launch_bounds__(NT) void f8_pack_kernel(RowArgs p, unsigned quads) {
  const int K = p.K, Kp = qrow(K);
  const i64 total = p.rows * quads;   // four blocks, a wave each
  const int lane = threadIdx.x & 63;
  for (i64 q = (i64)blockIdx.x * (NT / 64) + (threadIdx.x >> 6); q < total; q += (i64)gridDim.x * (NT / 64)) {
    const i64 row = q / quads;
    const int at = (int)(q - row * quads), k = at * 4 * BLK + lane * 8;
    const F8 f = load8<T>(static_cast<const T*>(p.x) + row * p.ld, k, K);
    const unsigned bits = block_max(amax8(f));
    if (k < Kp) *reinterpret_cast<uint2*>(p.codes + row * Kp + k) = f8_clip(f8_codes8(f, bits), k, K);
    if ((lane & 15) == 0) p.scales[row * (4 * quads) + at * 4 + (lane >> 4)] = k < K ? (uint8_t)(f8_exp(bits) + 127) : (uint8_t)127;
  }
}

template <typename T> __global__ __launch_bounds__(NT) void f8_unpack_kernel(RowArgs p, unsigned pieces) {
  const int K = p.K, Kp = qrow(K), Sp = f8srow(K);
  const i64 total = p.rows * pieces;
  for (i64 i = (i64)blockIdx.x * NT + threadIdx.x; i < total; i += (i64)gridDim.x * NT) {
    const i64 row = i >> 32 ? i / pieces : (i64)((unsigned)i / pieces);
    const int k = (int)(i - row * pieces) * 8;
    const uint2 c = *reinterpret_cast<const uint2*>(p.codes + row * Kp + k);
    store8<T>(static_cast<T*>(p.out) + row * p.ld, k, K, f8_decode8(c, scale_of_byte(p.scales[row * Sp + k / BLK])));
  }
}

int blocks_of(i64 work) { return (int)(work < 1 << 20 ? work : 1 << 20); }

}  // namespace

hipError_t launch_f8_pack(int dtype, i64 rows, int K, i64 ld, const void* x, void* codes, void* scales, hipStream_t st) {
  if (!rows) return hipSuccess;
  const RowArgs a = {rows, ld, K, x, nullptr, (uint8_t*)codes, (uint8_t*)scales};
  const unsigned quads = f8srow(K) / 4;
  const int grid = blocks_of((rows * quads + NT / 64 - 1) / (NT / 64));
  if (dtype == CONVBN_BF16) f8_pack_kernel<bf16_t><<<grid, NT, 0, st>>>(a, quads);
  else f8_pack_kernel<float><<<grid, NT, 0, st>>>(a, quads);
  return hipGetLastError();
}

hipError_t launch_f8_unpack(int dtype, i64 rows, int K, i64 ld, const void* codes, const void* scales, void* x, hipStream_t st) {
  if (!rows) return hipSuccess;
  const RowArgs a = {rows, ld, K, nullptr, x, (uint8_t*)codes, (uint8_t*)scales};
  const unsigned pieces = ceil_div(K, 8);
  const int grid = blocks_of((rows * pieces + NT - 1) / NT);
  if (dtype == CONVBN_BF16) f8_unpack_kernel<bf16_t><<<grid, NT, 0, st>>>(a, pieces);
  else f8_unpack_kernel<float><<<grid, NT, 0, st>>>(a, pieces);
  return hipGetLastError();
}

}  // namespace convbn
