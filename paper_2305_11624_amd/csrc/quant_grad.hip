// Gradients of the 8-bit product from the kept codes: dx = dz . (sw qw) + add, dW = dz^T . (sx qx), db = column sums of dz.
//
// Both products are C[i][j] = sum_r A(i, r) s[r] q[r][j] with codes that run along j: the input gradient reduces over the output
// channels (A = dz), the weight gradient over the rows (A = dz^T).  Codes become bf16 numbers s q on their way into LDS, once for
// all waves of a workgroup; q alone is exact there, s q is rounded to bf16.  That is the number that a checkpoint reads back as in bf16, so that a
// block's gradients are the same from the codes and from the rows; it takes the result from 0.0017 of its norm (its own rounding) to 0.0024
// against unrounded operands.  A product without it takes two or three bf16 parts in place of one: fp32 rows, in three, take 723 us for dx of
// 8192 x 4096 x 4096 and bf16 rows 231, dW 709 and 228.
//
// F32: A s is split into three bf16 parts that add up to all 24 bits, the codes stay whole numbers, and the three products are
// summed in fp32: nothing is rounded below that.
//
// 8192 x 4096 x 4096: dx and dW 227 - 236 us each (1165 - 1210 TFLOP/s, a bf16 product of the library at 8192^3 1325 - 1392).  The matrix pipe is busy for
// 58 - 59 % of the time; the rest goes to turning codes into bf16 numbers between the multiplies (4.9 vector instructions
// for each matrix instruction, itself among them; the int8 product has 3.0) and to the waits at a chunk's barrier.  1568 x 2048 x 512: both in one launch of 21.7 us,
// bound by the chunks' way from memory, one workgroup a compute unit.
#include "quant_code.h"

namespace convbn {

namespace {

typedef int i32x2 __attribute__((ext_vector_type(2)));

constexpr int RC = 64;                  // of the reduced index at a time

struct GradParams {
  const bf16_t* A;      // [planes][rows][lda]; aligned, zeros between the last channel and a multiple of 8
  i64 plane;            // elements of a plane
  i64 lda;
  const uint8_t* q;     // [R][Jp]
  const float* s;       // [R]; null with parts, which hold them
  void* C;              // [I][ldc], bf16 or fp32; several splits: [splits][I][J rounded up to 8] fp32
  const void* add;      // laid out like C, of its type
  int c_bf16;
  i64 ldc;
  i64 I, R;             // (I: rows of C)
  int J, Jp, Aw;        // Aw: channels of A's rows, a multiple of 8
  int planes, nch;      // chunks of RC of a plane
  int splits, per;      // chunks of a split
  int nti, ntj;
  float* db;            // TRANS: column sums of A, [splits][I]; null: not wanted
};

// NST stages of A; two of the codes as bf16 numbers.  The codes come through registers, a chunk ahead, or (DEEP) have a ring of their own,
// as they are in memory, and a copy of the scales for each wave.
// G groups of waves divide the workgroup's part of the sum, each with rings of its own (one wave on a SIMD waits for its own reads and
// copies most of the time); their sums meet on the way out.
template <int TI_, int TJ_, int WI_, int WJ_, int NST_, bool DEEP_, int G_> struct GradCfg {
  static constexpr int TI = TI_, TJ = TJ_, WI = WI_, WJ = WJ_, NST = NST_, G = G_, WAVES = (TI / WI) * (TJ / WJ), NT = 64 * WAVES;   // of a group
  static constexpr bool DEEP = DEEP_;
  static constexpr int A_BYTES = TI * RC * 2, B_BYTES = TJ * RC * 2, Q_BYTES = TJ * RC;
  static constexpr int B_AT = NST * A_BYTES, Q_AT = B_AT + 2 * B_BYTES, S_AT = Q_AT + (DEEP ? NST * Q_BYTES : 0);
  static constexpr int RING = S_AT + (DEEP ? NST * WAVES * 256 : 0);
  static constexpr int CPW = A_BYTES / 1024 / WAVES, QPW = Q_BYTES / 1024 / WAVES;   // copies a wave
  static constexpr int group(bool parts) { return CPW + QPW + (parts ? 0 : 1); }   // DEEP: copies of a chunk of A, the next one's codes and scales
  static constexpr int PITCH = WJ * 4 + 16, OUT_BYTES = G * WAVES * 32 * PITCH;   // sums of 32 rows a wave on their way out
  static constexpr int LDS = G * RING > OUT_BYTES ? G * RING : OUT_BYTES;
  static_assert(A_BYTES % (2048 * WAVES) == 0 && Q_BYTES % (1024 * WAVES) == 0 && LDS <= 160 * 1024, "whole pairs of copies");
};

// Two codes to bf16 numbers s q
__device__ __forceinline__ uint32_t code2(uint32_t w, int at, float s) {
  return pack_bf16x2((float)(int8_t)(w >> (8 * at)) * s, (float)(int8_t)(w >> (8 * at + 8)) * s);
}

// Workgroup wg of a product.  TRANS: A(i, r) = A[r][i].  PARTS: A comes in p.planes parts with the scales in it (fp32); else in one.
template <bool TRANS, bool PARTS, class Cfg> __device__ __forceinline__ void grad_body(const GradParams& p, const int wg, unsigned char* const shared) {
  constexpr int TI = Cfg::TI, TJ = Cfg::TJ, WI = Cfg::WI, WJ = Cfg::WJ, NST = Cfg::NST, G = Cfg::G;
  constexpr int NT = Cfg::NT, FI = WI / 32, FJ = WJ / 32;
  const int lane = threadIdx.x & 63, all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int group = all / Cfg::WAVES, wave = all % Cfg::WAVES, tid = wave * 64 + lane;
  unsigned char* const smem = shared + group * Cfg::RING;
  TileAt t;
  if (!tile_at(wg, p.nti, p.ntj, p.splits, &t)) return;
  const int split = t.split, j0 = t.j * TJ;
  const i64 i0 = (i64)t.i * TI;
  const int w_beg = split * p.per, w_end = min(p.planes * p.nch, w_beg + p.per), turns = (w_end - w_beg + G - 1) / G;
  const int c_beg = w_beg + group * turns, c_end = min(w_end, c_beg + turns);   // (all groups take as many turns)

  // ---- copies of A: 8 rows of 64 channels (direct) or 1 KB of rows of TI channels
  constexpr int CPW = Cfg::CPW, RPC = TRANS ? 512 / TI : 8;   // rows a copy
  unsigned a_off[CPW];
  const int dg = ((lane & 7) ^ (lane >> 4)) * 8;   // direct: this lane's channels in a chunk (a wave's odd copies: ^ 32)
#pragma unroll
  for (int i = 0; i < CPW; ++i) {
    const int r = (wave * CPW + i) * RPC + lane / (64 / RPC);
    if constexpr (TRANS) {
      const int l = lane % (TI / 8), g = (((l >> 2) ^ turn<TI>(r)) * 4 + (l & 3)) * 8;
      a_off[i] = i0 + g < p.Aw ? (unsigned)(r * (int)p.lda + g) * 2u : OOB;
    } else {
      a_off[i] = (unsigned)(r * (int)p.lda + (dg ^ (i & 1) * 32)) * 2u;
    }
  }
  const unsigned lds0 = lds_off(smem) + wave * CPW * 1024;
  // Where the next chunk of A starts, and how many there are: past the last one nothing is in bounds and zeros are copied, so the loop has
  // no branch.  In one part every chunk is a step further and only the slice's last can be short; parts start over at the first row.
  const int R = (int)p.R, left_last = R - (p.nch - 1) * RC, c_in = PARTS ? c_beg % max(p.nch, 1) : c_beg;
  const bool ends = c_end == p.nch;   // (one part: this slice holds the last chunk)
  int a_r0 = c_in * RC, a_left = c_end - c_beg;
  const int a_rows = (int)(p.I - i0 < TI ? p.I - i0 : TI);
  const int a_full = TRANS ? (int)((RC - 1) * p.lda + p.Aw - i0) * 2 : (int)((a_rows - 1) * p.lda + p.Aw) * 2;
  const int a_last = TRANS ? (int)((left_last - 1) * p.lda + p.Aw - i0) * 2 : 0;
  const i64 a_step = TRANS ? RC * p.lda : RC;
  const bf16_t* a_plane = p.A + (PARTS ? (c_beg / max(p.nch, 1)) * p.plane : 0) + (TRANS ? i0 : i0 * p.lda);
  const bf16_t* a_ptr = a_plane + c_in * a_step;
  i32x4 a_desc;
  bool a_in[2];
  auto next_a = [&]() {
    int bytes = a_full;
    if constexpr (!TRANS) bytes -= a_r0 * 2;
    else if (PARTS ? a_r0 + RC >= R : ends && a_left == 1) bytes = a_last;
    a_desc = make_desc(a_ptr, a_left > 0 ? bytes : 0);
    a_in[0] = TRANS || a_r0 + dg < p.Aw;
    a_in[1] = TRANS || a_r0 + (dg ^ 32) < p.Aw;
    --a_left;
    if constexpr (PARTS) {
      const bool wrap = a_r0 + RC >= R;
      a_r0 = wrap ? 0 : a_r0 + RC;
      a_plane = wrap ? a_plane + p.plane : a_plane;
      a_ptr = wrap ? a_plane : a_ptr + a_step;
    } else {
      a_r0 += RC;
      a_ptr += a_step;
    }
  };
  auto issue = [&](int slot, int from, int to) {
#pragma unroll
    for (int i = 0; i < CPW; ++i)
      if (i >= from && i < to) dma16(a_desc, a_in[i & 1] ? a_off[i] : OOB, lds0 + slot * Cfg::A_BYTES + i * 1024);
  };

  // ---- codes: 8 a piece
  constexpr int PB = TJ * 8 / NT;
  unsigned b_off[PB], b_lds[PB], s_off[PB];   // where they come from (DEEP: in the ring) and go
#pragma unroll
  for (int t = 0; t < PB; ++t) {
    const int w = t * NT + tid;
    const int r = w / (TJ / 8), g = w % (TJ / 8);
    b_off[t] = Cfg::DEEP ? r * TJ + g * 8 : j0 + g * 8 < p.Jp ? (unsigned)(r * p.Jp + g * 8) : OOB;
    b_lds[t] = r * (TJ * 2) + ((g >> 2) ^ turn<TJ>(r)) * 64 + (g & 3) * 16;
    s_off[t] = r * 4;
  }
  constexpr int QPW = Cfg::QPW, LPQ = TJ / 16;   // DEEP: copies a wave, lanes a row
  unsigned q_off[QPW];
#pragma unroll
  for (int i = 0; i < QPW; ++i) {
    const int r = (wave * QPW + i) * (64 / LPQ) + lane / LPQ, c = (lane % LPQ) * 16;
    q_off[i] = j0 + c < p.Jp ? (unsigned)(r * p.Jp + c) : OOB;
  }
  struct Codes { i32x2 q[PB]; float s[PB]; };
  // ... of the codes and (one part) the scales
  int q_r0 = c_in * RC, q_left = c_end - c_beg;
  const uint8_t* q_ptr = p.q + j0 + (i64)q_r0 * p.Jp;
  const float* s_ptr = p.s + (PARTS ? 0 : q_r0);
  const int q_step = RC * p.Jp;
  auto rows_left = [&]() {
    const bool last = PARTS ? q_r0 + RC >= R : ends && q_left == 1;
    return q_left > 0 ? last ? left_last : RC : 0;
  };
  auto next_q = [&]() {
    --q_left;
    if constexpr (PARTS) {
      const bool wrap = q_r0 + RC >= R;
      q_r0 = wrap ? 0 : q_r0 + RC;
      q_ptr = wrap ? p.q + j0 : q_ptr + q_step;
    } else {
      q_ptr += q_step;
      s_ptr += RC;
    }
  };
  auto fetch = [&]() {
    Codes b;
    const int left = rows_left();
    const __amdgpu_buffer_rsrc_t rq = make_rsrc(q_ptr, left ? left * p.Jp - j0 : 0);
#pragma unroll
    for (int t = 0; t < PB; ++t) b.q[t] = __builtin_amdgcn_raw_buffer_load_b64(rq, (int)b_off[t], 0, 0);
    if constexpr (!PARTS) {
      const __amdgpu_buffer_rsrc_t rs = make_rsrc(s_ptr, left * 4);
#pragma unroll
      for (int t = 0; t < PB; ++t) b.s[t] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rs, (int)s_off[t], 0, 0));
    }
    next_q();
    return b;
  };
  auto issue_q = [&](int slot) {   // DEEP: the next chunk's codes and scales
    const int left = rows_left();
    const i32x4 dq = make_desc(q_ptr, left ? left * p.Jp - j0 : 0);
#pragma unroll
    for (int i = 0; i < QPW; ++i) dma16(dq, q_off[i], lds_off(smem) + Cfg::Q_AT + slot * Cfg::Q_BYTES + (wave * QPW + i) * 1024);
    if constexpr (!PARTS) dma4(make_desc(s_ptr, left * 4), lane * 4, lds_off(smem) + Cfg::S_AT + (slot * Cfg::WAVES + wave) * 256);
    next_q();
  };
  auto from_ring = [&](int slot) {
    Codes b;
#pragma unroll
    for (int t = 0; t < PB; ++t) {
      b.q[t] = *reinterpret_cast<const i32x2*>(smem + Cfg::Q_AT + slot * Cfg::Q_BYTES + b_off[t]);
      if constexpr (!PARTS) b.s[t] = *reinterpret_cast<const float*>(smem + Cfg::S_AT + (slot * Cfg::WAVES + wave) * 256 + s_off[t]);
    }
    return b;
  };
  auto put = [&](const Codes& b, int slot, int from, int to) {
#pragma unroll
    for (int t = 0; t < PB; ++t) {
      if (t < from || t >= to) continue;
      const uint32_t lo = b.q[t][0], hi = b.q[t][1];
      const float s = PARTS ? 1.f : b.s[t];
      *reinterpret_cast<uint4*>(smem + Cfg::B_AT + slot * Cfg::B_BYTES + b_lds[t]) =
          make_uint4(code2(lo, 0, s), code2(lo, 2, s), code2(hi, 0, s), code2(hi, 2, s));
    }
  };

  // ---- operands of this wave
  const int wi = (wave % (TI / WI)) * WI, wj = (wave / (TI / WI)) * WJ;
  const int kb = lane >> 5, ep = (lane & 15) >> 2;
  // transposing reads: this lane addresses row kb * 8 + ep (+ 4) of a 16-row step, channels (l / 16 % 2) * 16 + (l % 4) * 4 of 32
  const int tr_row = kb * 8 + ep, tr_col = ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
  auto b_at = [&](int step, int f) {
    return (step * 16 + tr_row) * (TJ * 2) + (((wj >> 5) + f) ^ turn<TJ>(ep)) * 64 + tr_col;
  };
  auto a_at = [&](int step, int f) {
    if constexpr (TRANS) return (step * 16 + tr_row) * (TI * 2) + (((wi >> 5) + f) ^ turn<TI>(ep)) * 64 + tr_col;
    const int row = wi + f * 32 + (lane & 31);
    return row * 128 + (((step * 2 + kb) ^ ((row >> 1) & 7)) << 4);
  };

  f32x16 acc[FI][FJ];
#pragma unroll
  for (int i = 0; i < FI; ++i)
#pragma unroll
    for (int j = 0; j < FJ; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

  // Column sums of A on the side, by the workgroups of the first tile column: two columns and a share of the rows a thread
  const bool sums = TRANS && p.db && t.j == 0;
  constexpr int SHARE = NT / (TI / 2), ROWS = RC / SHARE;   // threads a pair of columns, rows each
  const int pair = tid % (TI / 2), share = tid / (TI / 2);
  float sum0 = 0.f, sum1 = 0.f;

  if (turns > 0) {
    Codes next;
    if constexpr (Cfg::DEEP) {
      issue_q(0);
#pragma unroll
      for (int s = 0; s < NST - 1; ++s) {
        next_a();
        issue(s, 0, CPW);
        issue_q(s + 1);
      }
      landed<Cfg::group(PARTS) * (NST - 1)>();
      put(from_ring(0), 0, 0, PB);
    } else {
#pragma unroll
      for (int s = 0; s < NST - 1; ++s) {
        next_a();
        issue(s, 0, CPW);
      }
      put(fetch(), 0, 0, PB);
      next = fetch();
    }
    next_a();
    int slot = 0;   // of A (and, of the ring of codes, this chunk's, which is free again)
    for (int c = c_beg; c < c_beg + turns; ++c) {
      landed<(Cfg::DEEP ? Cfg::group(PARTS) : CPW) * (NST - 2)>();   // this chunk is in place for all waves, and all have read the one before
      const unsigned char* cur = smem + slot * Cfg::A_BYTES;
      const unsigned char* curb = smem + Cfg::B_AT + ((c - c_beg) & 1) * Cfg::B_BYTES;
      const int fill = slot ? slot - 1 : NST - 1;
      const int putb = (c - c_beg + 1) & 1;
      bf16x8 af[2][FI], bf[2][FJ];
      auto read = [&](int step) {
#pragma unroll
        for (int f = 0; f < FI; ++f) {
          if constexpr (TRANS) af[step & 1][f] = read_tr8(cur + a_at(step, f), 4 * TI * 2);
          else af[step & 1][f] = *reinterpret_cast<const bf16x8*>(cur + a_at(step, f));
        }
#pragma unroll
        for (int f = 0; f < FJ; ++f) bf[step & 1][f] = read_tr8(curb + b_at(step, f), 4 * TJ * 2);
      };
      read(0);
      Codes b;
      const int after = slot + 1 == NST ? 0 : slot + 1;
      if constexpr (Cfg::DEEP) {
        b = from_ring(after);
      } else {
        b = next;
        next = fetch();
      }
#pragma unroll
      for (int step = 0; step < RC / 16; ++step) {
        if (step + 1 < RC / 16) read(step + 1);
        // (8192 x 4096 x 4096, dx: over half of the chunk's multiplies 241 us, over all of them 232; 1568 x 2048 x 512: 10.8 and 11.1)
        constexpr int OVER = TI == 256 ? 4 : 2;
        issue(fill, step * CPW / OVER, (step + 1) * CPW / OVER);
        if constexpr (Cfg::DEEP)
          if (step == 1) issue_q(slot);
        put(b, putb, step * PB / 4, (step + 1) * PB / 4);
#pragma unroll
        for (int i = 0; i < FI; ++i)
#pragma unroll
          for (int j = 0; j < FJ; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bf[step & 1][j], af[step & 1][i], acc[i][j], 0, 0, 0);
      }
      if (sums) {
#pragma unroll
        for (int x = 0; x < ROWS; ++x) {
          const int r = share * ROWS + x;
          const uint32_t w = *reinterpret_cast<const uint32_t*>(cur + r * (TI * 2) + ((pair >> 4) ^ turn<TI>(r)) * 64 + (pair & 15) * 4);
          sum0 += bf16_lo(w);
          sum1 += bf16_hi(w);
        }
      }
      next_a();
      slot = after;
    }
    landed<0>();
  }
  if (sums) {
    float* part = reinterpret_cast<float*>(shared);
    part[(group * SHARE + share) * TI + 2 * pair] = sum0;
    part[(group * SHARE + share) * TI + 2 * pair + 1] = sum1;
    __syncthreads();
    if (group == 0 && tid < TI && i0 + tid < p.I) {
      float v = 0.f;
#pragma unroll
      for (int x = 0; x < G * SHARE; ++x) v += part[x * TI + tid];
      p.db[split * p.I + i0 + tid] = v;
    }
    __syncthreads();
  }

  // ---- out, 32 rows of this wave at a time: a lane holds row l % 32 and, for each e / 4, four channels 8 (e / 4) + 4 (l / 32) ..;
  // through LDS they become whole rows
  constexpr int LPR = WJ / 8;   // lanes a row, 8 channels each
  unsigned char* mine = shared + all * 32 * Cfg::PITCH;
  auto meet = [] {
    if constexpr (G > 1) __syncthreads();
    else __builtin_amdgcn_wave_barrier();
  };
  const int col = (lane % LPR) * 8, n = j0 + wj + col;
  const i64 c0 = p.splits > 1 ? (i64)split * p.I * p.ldc : 0;
#pragma unroll
  for (int i = 0; i < FI; ++i) {
#pragma unroll
    for (int j = 0; j < FJ; ++j)
#pragma unroll
      for (int e = 0; e < 16; e += 4)
        *reinterpret_cast<float4*>(mine + (lane & 31) * Cfg::PITCH + (j * 32 + 8 * (e >> 2) + 4 * kb) * 4) =
            make_float4(acc[i][j][e], acc[i][j][e + 1], acc[i][j][e + 2], acc[i][j][e + 3]);
    meet();
    constexpr int RPI = 64 / LPR;   // rows at a time, a group after the other
#pragma unroll
    for (int r0 = 0; r0 < 32; r0 += RPI * G) {
      const int at = r0 + group * RPI + lane / LPR;
      const i64 row = i0 + wi + i * 32 + at;
      F8 v = {};
#pragma unroll
      for (int o = 0; o < G; ++o)
#pragma unroll
        for (int h = 0; h < 8; h += 4) {
          const float4 w = *reinterpret_cast<const float4*>(shared + ((o * Cfg::WAVES + wave) * 32 + at) * Cfg::PITCH + (col + h) * 4);
          v.v[h] += w.x; v.v[h + 1] += w.y; v.v[h + 2] += w.z; v.v[h + 3] += w.w;
        }
      if (row >= p.I || n >= p.J) continue;
      const i64 o = c0 + row * p.ldc;
      if (p.c_bf16) store8_plus<bf16_t>(static_cast<bf16_t*>(p.C) + o, p.add ? static_cast<const bf16_t*>(p.add) + o : nullptr, n, p.J, v);
      else store8_plus<float>(static_cast<float*>(p.C) + o, p.add ? static_cast<const float*>(p.add) + o : nullptr, n, p.J, v);
    }
    meet();
  }
}

using Big = GradCfg<256, 256, 128, 64, 3, false, 1>;        // (waves of 64 x 128: dW of 8192 x 4096 x 4096 240 us and not 235)
using Mid = GradCfg<128, 128, 64, 64, 2, false, 1>;
using MidAlone = GradCfg<128, 128, 64, 32, 4, true, 1>;     // one workgroup a compute unit: its copies are all that hides the way to memory
using Small = GradCfg<64, 64, 32, 32, 4, true, 2>;

template <bool TRANS, bool PARTS, class Cfg> __global__ __launch_bounds__(Cfg::NT * Cfg::G) void qgrad_kernel(GradParams p) {
  extern __shared__ __align__(16) unsigned char shared[];
  grad_body<TRANS, PARTS, Cfg>(p, (int)blockIdx.x, shared);
}
// Both gradients in one launch: where neither fills the chip for long, the second need not wait for the last workgroup of the first.
template <bool PARTS, class X, class W> __global__ __launch_bounds__(X::NT * X::G) void qgrad_pair_kernel(GradParams x, GradParams w, int first) {
  static_assert(X::NT * X::G == W::NT * W::G, "one launch");
  extern __shared__ __align__(16) unsigned char shared[];
  if ((int)blockIdx.x < first) grad_body<false, PARTS, X>(x, (int)blockIdx.x, shared);
  else grad_body<true, PARTS, W>(w, (int)blockIdx.x - first, shared);
}

// C = the sum of the splits + add; likewise the column sums.  Four threads share eight channels (or one column sum), each adds every fourth
// split, and the four sums meet in LDS: the order is the same in every run.
constexpr int JOIN = 4;
struct JoinParams {
  i64 I, ldc;
  int J, splits, db_splits, blocks;   // I x J of C (either 0: none); rows of the parts lie a multiple of 8 apart
  const float* part; void* C; const void* add;
  i64 N; const float* db_part; float* db;
};
template <typename OUT> __device__ __forceinline__ void join_body(const JoinParams& p, const int wg) {
  __shared__ float meet[JOIN][8][64];
  OUT* C = static_cast<OUT*>(p.C);
  const OUT* add = static_cast<const OUT*>(p.add);
  const int at = threadIdx.x & 63, q = threadIdx.x >> 6;
  const int pieces = (p.J + 7) >> 3;
  const i64 mine = p.I * pieces, total = mine + p.N;   // the column sums come last, one a thread
  for (i64 x0 = (i64)wg * 64; x0 < total; x0 += (i64)p.blocks * 64) {
    const i64 x = x0 + at;
    float v[8] = {};
    if (x < mine) {
#pragma unroll 4
      for (int s = q; s < p.splits; s += JOIN) {
        const float4* f = reinterpret_cast<const float4*>(p.part + (s * mine + x) * 8);
        const float4 a = f[0], b = f[1];
        v[0] += a.x; v[1] += a.y; v[2] += a.z; v[3] += a.w; v[4] += b.x; v[5] += b.y; v[6] += b.z; v[7] += b.w;
      }
    } else if (x < total) {
#pragma unroll 8
      for (int s = q; s < p.db_splits; s += JOIN) v[0] += p.db_part[s * p.N + (x - mine)];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) meet[q][e][at] = v[e];
    __syncthreads();
    if (q == 0 && x < total) {
      F8 f;
#pragma unroll
      for (int e = 0; e < 8; ++e) f.v[e] = (meet[0][e][at] + meet[1][e][at]) + (meet[2][e][at] + meet[3][e][at]);
      if (x >= mine) {
        p.db[x - mine] = f.v[0];
      } else {
        const i64 row = x / pieces, o = row * p.ldc;
        store8_plus<OUT>(C + o, add ? add + o : nullptr, (int)(x - row * pieces) * 8, p.J, f);
      }
    }
    __syncthreads();
  }
}
// (of both gradients, or of one: the other has no blocks)
template <typename OUT> __global__ __launch_bounds__(256) void qjoin_kernel(JoinParams x, JoinParams w) {
  if ((int)blockIdx.x < x.blocks) join_body<OUT>(x, (int)blockIdx.x);
  else join_body<OUT>(w, (int)blockIdx.x - x.blocks);
}

// One pass over dz for what the products do not take from it as it lies: its column sums, and dz as they want it, rows of a multiple of 8
// channels with zeros past the last (f32: dz s in three parts, s by column for dx, by row for dW).  A workgroup takes 256 columns, a thread
// eight of them and every 16th row of a slice; the sums of several slices are joined in order by a later launch.  A copy with its sums of
// 22144 x 3841 bf16 (340 MB in and out) takes 77 us, 4.4 TB/s, bound by memory; copy and sums in two launches took 108.
constexpr int PREP_ROWS = 16;
struct PrepParams {
  i64 M, ldz, per;
  int N;
  const void* dz; float* sums;          // [slices][N] or null
  bf16_t* copy; bf16_t* by_row;         // copy: of bf16 dz, or of f32 dz sw; by_row: of f32 dz sx; either null
  const float* sw; const float* sx;
};
template <typename T> __global__ __launch_bounds__(32 * PREP_ROWS) void qprep_kernel(PrepParams p) {
  __shared__ float meet[PREP_ROWS][256 + 8];
  const int c = (threadIdx.x & 31) * 8, r = threadIdx.x >> 5, n = blockIdx.x * 256 + c, N8 = (p.N + 7) & ~7;
  const i64 beg = (i64)blockIdx.y * p.per, end = beg + p.per < p.M ? beg + p.per : p.M, plane = p.M * N8;
  const T* dz = static_cast<const T*>(p.dz);
  F8 sum = {}, sw = {};
  if (n < p.N) {
    if (sizeof(T) == 4 && p.copy) sw = load8<float>(p.sw, n, p.N);
#pragma unroll 4
    for (i64 m = beg + r; m < end; m += PREP_ROWS) {
      const F8 v = load8<T>(dz + m * p.ldz, n, p.N);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum.v[e] += v.v[e];
      if constexpr (sizeof(T) == 2) {
        if (p.copy) store8<bf16_t>(p.copy + m * N8, n, N8, v);
      } else {
        F8 scaled, part[3];
        if (p.copy) {
#pragma unroll
          for (int e = 0; e < 8; ++e) scaled.v[e] = n + e < p.N ? v.v[e] * sw.v[e] : 0.f;
          split3(scaled, part);
#pragma unroll
          for (int x = 0; x < 3; ++x) store8<bf16_t>(p.copy + x * plane + m * N8, n, N8, part[x]);
        }
        if (p.by_row) {
          const float s = p.sx[m];
#pragma unroll
          for (int e = 0; e < 8; ++e) scaled.v[e] = n + e < p.N ? v.v[e] * s : 0.f;
          split3(scaled, part);
#pragma unroll
          for (int x = 0; x < 3; ++x) store8<bf16_t>(p.by_row + x * plane + m * N8, n, N8, part[x]);
        }
      }
    }
  }
  if (!p.sums) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) meet[r][c + e] = sum.v[e];
  __syncthreads();
  const int at = threadIdx.x, col = blockIdx.x * 256 + at;
  if (at < 256 && col < p.N) {
    float v = 0.f;
#pragma unroll
    for (int i = 0; i < PREP_ROWS; ++i) v += meet[i][at];
    p.sums[(i64)blockIdx.y * p.N + col] = v;
  }
}

int grid_of(i64 work) { const i64 b = (work + 255) / 256; return (int)(b < 1 ? 1 : b < 65536 ? b : 65536); }

constexpr int CUS = 256;

// The cheapest of tiles of 64 (as long as they are a round), 128 and 256, and of 1 to 256 parts of the sum, by what was measured in us: a
// launch 2.5, every round of workgroups 2.3, 3.2 or 7 and, for each chunk, 0.36, 0.76 or 1.85 with a workgroup alone on its compute unit,
// 1.4 with two (128); parts cost another launch and their sums' way through memory.  With one group of waves a tile, dW of 1568 x
// 2048 x 512: 64 whole 17.3 (with two 14.3), in two parts 28, 128 whole 24.2, in two 22.7, in four 22.5; dx of 64 x 2048 x 512: 64 8.0, 128 9.8; of 200 x 1024 x 4096: 64 whole 32.8, in four 16.7,
// 128 whole 47, in eight 17.8; of 1568 x 8192 x 2048: 128 82, 256 59.5; of 100352 x 256 x 64: 128 19.4, 256 20.3.
struct Plan { int tile, splits, per; };
Plan plan_of(i64 I, int J, i64 R, int planes) {
  const int nch = (int)((R + RC - 1) / RC) * planes;
  Plan pl = {128, 1, nch};
  auto tiles = [&](i64 t) { return ((I + t - 1) / t) * ((J + t - 1) / t); };
  if (!I || !nch) return pl;   // (no rows)
  double best = 1e30;
  for (int tile = 64; tile <= 256; tile *= 2)
    for (int s = 1; s <= 256 && s <= nch; s *= 2) {
      const int per = ceil_div(nch, s), parts = ceil_div(nch, per);
      const double w = (double)tiles(tile) * parts;
      if (tile == 64 && w > CUS) break;
      const bool alone = w <= CUS;
      const double rounds = (double)(i64)(tile == 256 ? (w + 255) / 256 : (w + 511) / 512);
      const double chunk = tile == 256 ? 1.85 : tile == 128 ? (alone ? 0.76 : 1.4) : 0.36;
      const double us = 2.5 + rounds * ((tile == 256 ? 7 : tile == 128 ? 3.2 : 2.3) + chunk * per) + (parts > 1 ? 4 + 2e-6 * parts * (double)I * J : 0);
      if (us < best) {
        best = us;
        pl = {tile, parts, per};
      }
    }
  return pl;
}

// Slices of dz's rows for its pass: some 2048 workgroups, of 32 rows or more (of 256 slices at most: their sums have to be joined)
int prep_slices(i64 M, int N) {
  i64 s = ceil_div(2048, ceil_div(N, 256));
  if (s > M / 32) s = M / 32;
  return (int)(s < 1 ? 1 : s < 256 ? s : 256);
}

// Whether the products read dz where it is (its first row on 16 bytes then: qgrad_reads_in_place); else a copy, or the three parts
bool direct(const QGrad& p) { return qgrad_reads_in_place(p.dtype, p.N, p.ldz); }

struct Scratch { size_t copy, part, cols, total; };
Scratch scratch_of(const QGrad& p) {   // (for all outputs)
  Scratch s;
  const int N8 = (p.N + 7) & ~7;
  const int planes = p.dtype == CONVBN_BF16 ? 1 : 3;
  if (p.dtype != CONVBN_BF16) s.copy = (size_t)6 * p.M * N8 * 2;   // three parts, for either product
  else s.copy = direct(p) ? 0 : (size_t)p.M * N8 * 2;
  const Plan dx = plan_of(p.M, p.K, p.N, planes), dw = plan_of(p.N, p.K, p.M, planes);
  const size_t K8 = (p.K + 7) & ~7;
  const size_t px = dx.splits > 1 ? (size_t)dx.splits * p.M * K8 * 4 : 0, pw = dw.splits > 1 ? (size_t)dw.splits * p.N * (K8 + 1) * 4 : 0;
  s.copy = align_up(s.copy, 256);
  s.part = align_up(px + pw, 256);
  s.cols = align_up((size_t)prep_slices(p.M, p.N) * p.N * 4, 256);
  s.total = s.copy + s.part + s.cols;
  return s;
}

int grid_of(const GradParams& g) { return (g.nti * g.ntj * g.splits + 7) / 8 * 8; }

template <bool TRANS, bool PARTS, class Cfg> hipError_t launch_one(const GradParams& g, hipStream_t st) {
  static LdsLimitOnce once;
  auto* k = &qgrad_kernel<TRANS, PARTS, Cfg>;
  const hipError_t e = set_lds_limit_once(once, (const void*)k, Cfg::LDS);
  if (e != hipSuccess) return e;
  k<<<grid_of(g), Cfg::NT * Cfg::G, Cfg::LDS, st>>>(g);
  return hipGetLastError();
}
template <bool PARTS, class X, class W> hipError_t launch_pair(const GradParams& x, const GradParams& w, hipStream_t st) {
  constexpr int LDS = X::LDS > W::LDS ? X::LDS : W::LDS;
  static LdsLimitOnce once;
  auto* k = &qgrad_pair_kernel<PARTS, X, W>;
  const hipError_t e = set_lds_limit_once(once, (const void*)k, LDS);
  if (e != hipSuccess) return e;
  k<<<grid_of(x) + grid_of(w), X::NT * X::G, LDS, st>>>(x, w, grid_of(x));
  return hipGetLastError();
}

// A product as it is launched, and what joins it
struct Product { bool on = false; int tile = 0; GradParams g = {}; JoinParams join = {}; };
bool alone(const Product& r) { return r.tile <= 128 && r.g.nti * r.g.ntj * r.g.splits <= CUS; }

template <bool TRANS, bool PARTS> hipError_t launch_product(const Product& r, hipStream_t st) {
  if (r.tile == 256) return launch_one<TRANS, PARTS, Big>(r.g, st);
  if (r.tile == 64) return launch_one<TRANS, PARTS, Small>(r.g, st);
  return alone(r) ? launch_one<TRANS, PARTS, MidAlone>(r.g, st) : launch_one<TRANS, PARTS, Mid>(r.g, st);
}

// sums: column sums of A as well (A = dz itself)
template <bool TRANS> Product product(const QGrad& p, const bf16_t* A, i64 lda, float* part, bool sums) {
  Product r;
  GradParams& g = r.g = {};
  const bool f32 = p.dtype != CONVBN_BF16;
  const int N8 = (p.N + 7) & ~7;
  r.on = true;
  g.planes = f32 ? 3 : 1;
  g.A = A; g.lda = lda; g.plane = p.M * (i64)N8; g.Aw = N8;
  g.q = static_cast<const uint8_t*>(TRANS ? p.qx : p.qw);
  g.s = f32 ? nullptr : TRANS ? p.sx : p.sw;
  g.J = p.K; g.Jp = qrow(p.K);
  g.I = TRANS ? p.N : p.M;
  g.R = TRANS ? p.M : p.N;
  g.nch = (int)((g.R + RC - 1) / RC);
  const Plan pl = plan_of(g.I, g.J, g.R, g.planes);
  r.tile = pl.tile;
  g.splits = pl.splits; g.per = pl.per;
  g.nti = (int)((g.I + pl.tile - 1) / pl.tile); g.ntj = ceil_div(g.J, pl.tile);
  void* C = TRANS ? p.dW : p.dx;
  const i64 ldc = TRANS ? p.K : p.ldx;
  const void* add = TRANS ? nullptr : p.add;
  if (pl.splits > 1) {
    g.C = part; g.ldc = (g.J + 7) & ~7;
    r.join = {g.I, ldc, g.J, pl.splits, 0, 0, part, C, add, 0, nullptr, nullptr};
    if (sums) {
      float* db_part = part + pl.splits * g.I * g.ldc;
      g.db = db_part;
      r.join.db_splits = pl.splits; r.join.N = p.N; r.join.db_part = db_part; r.join.db = p.db;
    }
  } else {
    g.C = C; g.ldc = ldc; g.add = add; g.c_bf16 = !f32; g.db = sums ? p.db : nullptr;
  }
  return r;
}

template <typename T> hipError_t grad_t(const QGrad& p, void* ws, hipStream_t st) {
  constexpr bool PARTS = sizeof(T) == 4;
  const Scratch sc = scratch_of(p);
  bf16_t* copy = static_cast<bf16_t*>(ws);
  float* part = reinterpret_cast<float*>(static_cast<char*>(ws) + sc.copy);
  float* cols = reinterpret_cast<float*>(static_cast<char*>(ws) + sc.copy + sc.part);
  const int N8 = (p.N + 7) & ~7;
  const bool in_place = direct(p), copies = p.M && (p.dx || p.dW) && !in_place;
  const bf16_t* A = copy;
  i64 lda = N8;
  if constexpr (!PARTS)
    if (in_place) { A = static_cast<const bf16_t*>(p.dz); lda = p.ldz; }
  bf16_t* by_row = copy + 3 * p.M * N8;
  // The column sums of dz that is read in place ride in the weight gradient, except with the largest tiles: the workgroups that add them up
  // would keep the others waiting (8192 x 4096 x 4096: 26 us more, a launch of their own 14; 1568 x 2048 x 512: 1 us more, a launch 6)
  const bool ride = p.db && p.dW && p.M && in_place && plan_of(p.N, p.K, p.M, 1).tile < 256;
  const int slices = prep_slices(p.M, p.N);
  if (copies || (p.db && !ride)) {
    const PrepParams q = {p.M, p.ldz, (p.M + slices - 1) / slices, p.N, p.dz, !p.db ? nullptr : slices > 1 ? cols : p.db,
                          copies && (!PARTS || p.dx) ? copy : nullptr, copies && PARTS && p.dW ? by_row : nullptr, p.sw, p.sx};
    qprep_kernel<T><<<dim3(ceil_div(p.N, 256), slices), 32 * PREP_ROWS, 0, st>>>(q);
  }
  Product x, w;
  if (p.dx && p.M) x = product<false>(p, A, lda, part, false);
  if (p.dW) w = product<true>(p, sizeof(T) == 4 ? by_row : A, lda, part + (x.on && x.g.splits > 1 ? x.g.splits * x.g.I * x.g.ldc : 0), ride);
  hipError_t e = hipSuccess;
  if (x.on && w.on && alone(x) && alone(w)) {
    if (x.tile == 64) e = w.tile == 64 ? launch_pair<PARTS, Small, Small>(x.g, w.g, st) : launch_pair<PARTS, Small, MidAlone>(x.g, w.g, st);
    else e = w.tile == 64 ? launch_pair<PARTS, MidAlone, Small>(x.g, w.g, st) : launch_pair<PARTS, MidAlone, MidAlone>(x.g, w.g, st);
  } else {
    if (x.on) e = launch_product<false, PARTS>(x, st);
    if (e == hipSuccess && w.on) e = launch_product<true, PARTS>(w, st);
  }
  if (e != hipSuccess) return e;
  if (p.db && !ride && slices > 1) { w.join.db_splits = slices; w.join.N = p.N; w.join.db_part = cols; w.join.db = p.db; }
  auto blocks = [](JoinParams& j) { j.blocks = j.I || j.N ? grid_of(JOIN * (j.I * ((j.J + 7) / 8) + j.N)) : 0; };
  blocks(x.join);
  blocks(w.join);
  if (x.join.blocks + w.join.blocks) qjoin_kernel<T><<<x.join.blocks + w.join.blocks, 256, 0, st>>>(x.join, w.join);
  return hipGetLastError();
}

}  // namespace

bool qgrad_reads_in_place(int dtype, int N, i64 ldz) { return dtype == CONVBN_BF16 && N % 8 == 0 && ldz % 8 == 0 && ldz <= 1 << 20; }
size_t qgrad_scratch(const QGrad& p) { return scratch_of(p).total; }
hipError_t launch_qgrad(const QGrad& p, void* ws, hipStream_t st) {
  return p.dtype == CONVBN_BF16 ? grad_t<bf16_t>(p, ws, st) : grad_t<float>(p, ws, st);
}

}  // namespace convbn
