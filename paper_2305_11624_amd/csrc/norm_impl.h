// Group norm with an activation, channels last, forward and backward.
//
// A team of lanes takes some neighbouring groups of an image.  A lane holds pieces of eight channels of one group: v counts the pieces of a
// group's pixel, then come the groups of the team, then the pixels, so that neighbouring lanes read neighbouring memory and a group's lanes meet by
// exchanging along the bits of v and of the pixel: within a wave by shuffles, between waves through LDS, one barrier an image.  Means are taken
// relative to the group's first value and variances merged from what each lane finds about its own mean, so neither loses bits to values that lie
// far from zero.
//
// Where a team's part of an image fits the registers (x forward, x and dy backward) it is read once: one launch that reads and writes
// each number once.  Larger parts, and images that are too few to fill the chip, go in two launches: the sums of segments of the
// pixels, and then the outputs, for which every workgroup merges its groups' segments for itself; the second reading is partly from the
// last-level cache.
//
// Backward walks several images with the same channels, so that dgamma and dbeta gather in registers; a launch joins what the workgroups found.
#pragma once
#include "f8_code.h"

namespace convbn {

namespace {

struct Team { int m, mlog, nblog, lprlog, ttlog; };   // pieces of a group's pixel; lanes of a group's pixel, groups, lanes of a pixel, of the team: powers of two

struct NormParams {
  Norm n;
  Team t;
  int cg, bundles;      // channels of a group, teams side by side
  int span, sections;   // a group of more channels than a workgroup has lanes for: sections of `span` channels, a team each
  int slices;           // workgroups along the images (each takes every slices'th team of images)
  int segs;             // segments of the pixels
  i64 seg;              // pixels of one
  float* part;          // sums of the segments, [M][groups][segs * sections][2]
  float* sums;          // [slices * segs][C][2]: dgamma, dbeta; null: not wanted
};

template <typename T, int F> __device__ __forceinline__ void act_of(float z, float* f, float* df) {
  if constexpr (F == CONVBN_NORM_NONE) { *f = z; *df = 1.f; }
  else if constexpr (F == CONVBN_NORM_RELU) { *f = z > 0.f ? z : 0.f * z; *df = z > 0.f ? 1.f : 0.f; }
  else gate_of<T, F == CONVBN_NORM_SILU ? CONVBN_GATE_SILU : CONVBN_GATE_GELU>(z, f, df);
}

// A piece of n channels (1 to 8; zeros past them).  FULL: all pieces are whole
template <bool FULL, typename T> __device__ __forceinline__ Raw8<T> load_piece(const T* p, int n) {
  if (FULL || n == 8) return *reinterpret_cast<const Raw8<T>*>(p);
  F8 f;
#pragma unroll
  for (int i = 0; i < 8; ++i) f.v[i] = i < n ? to_f32(p[i]) : 0.f;
  return narrow<T>(f);
}
template <bool FULL, typename T> __device__ __forceinline__ void store_piece(T* p, int n, const F8& f) {
  if (FULL || n == 8) {
    *reinterpret_cast<Raw8<T>*>(p) = narrow<T>(f);
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < n) p[i] = from_f32<T>(f.v[i]);
}

// From here on the pieces are what is in their registers: else the compiler keeps them as the eight fp32 numbers that an earlier pass made of
// each, which take twice the room (512 lanes of 32 pieces: 142 registers to memory)
template <typename T, int KP> __device__ __forceinline__ void as_held(Raw8<T> (&x)[KP]) {
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int k = 0; k < KP; ++k) {
      u32x4 a = x[k].a;
      asm volatile("" : "+v"(a));
      x[k].a = a;
    }
  }
}

// A lane's place
struct Lane {
  int wave, waves, r, RT, gl, c, n, lpr;   // waves: of the team; c: first channel, n: channels of the piece (0: none), gl: group in the team
  int g, section, team;
  bool first;                              // the group's (or its section's) first lane
  __device__ __forceinline__ Lane(const NormParams& p, int bundle) {
    const int tid = threadIdx.x, t = tid & ((1 << p.t.ttlog) - 1), v = t & ((1 << p.t.mlog) - 1);
    team = tid >> p.t.ttlog;
    wave = tid >> 6;
    waves = p.t.ttlog > 6 ? 1 << (p.t.ttlog - 6) : 1;
    lpr = p.t.lprlog;
    gl = t >> p.t.mlog & ((1 << p.t.nblog) - 1);
    r = t >> lpr;
    RT = 1 << (p.t.ttlog - lpr);
    section = bundle % p.sections;
    g = bundle / p.sections * (1 << p.t.nblog) + gl;
    const int at = section * p.span + v * 8;   // in the group
    c = g * p.cg + at;
    n = g < p.n.groups && v < p.t.m ? max(0, min(8, p.cg - at)) : 0;
    first = n && r == 0 && v == 0;
  }
  // this lane's entry of the segments' sums of image m
  __device__ __forceinline__ float* entry(const NormParams& p, i64 m, int i) const {
    return p.part + ((m * p.n.groups + g) * (p.segs * p.sections) + i) * 2;
  }
  // Sums over a group's lanes of this wave
  template <int N> __device__ __forceinline__ void wave_sums(const Team& t, float (&s)[N]) const {
    for (int o = 1; o < 64 && o < 1 << t.mlog; o <<= 1)
#pragma unroll
      for (int i = 0; i < N; ++i) s[i] += __shfl_xor(s[i], o, 64);
    for (int o = 1 << lpr; o < 64 && o < 1 << t.ttlog; o <<= 1)
#pragma unroll
      for (int i = 0; i < N; ++i) s[i] += __shfl_xor(s[i], o, 64);
  }
  // Where this wave's sums go and the team's begin; entries of N floats
  __device__ __forceinline__ int slot(int w) const { return w * 64 + gl; }
  __device__ __forceinline__ int first_wave() const { return wave & ~(waves - 1); }
};

struct Moments { float n, mean, m2; };
__device__ __forceinline__ void merge(Moments& a, const Moments& b) {
  if (b.n == 0.f) return;
  const float n = a.n + b.n, d = b.mean - a.mean, q = b.n / n;
  a.mean += d * q;
  a.m2 += b.m2 + d * d * a.n * q;
  a.n = n;
}
// A group's moments from its lanes'; every lane of the team returns them.  buf: [64 * waves of the workgroup][3]
__device__ __forceinline__ Moments team_moments(const Lane& l, const Team& t, Moments a, float (*buf)[3]) {
  float s[2] = {a.n, a.n * a.mean};
  l.wave_sums(t, s);
  const float wmean = s[0] > 0.f ? s[1] / s[0] : 0.f, d = a.mean - wmean;
  float q[1] = {a.n > 0.f ? a.m2 + a.n * d * d : 0.f};
  l.wave_sums(t, q);
  Moments w = {s[0], wmean, q[0]};
  if (t.ttlog <= 6) return w;
  if ((threadIdx.x & 63) == (l.gl << t.mlog & 63)) {
    float* o = buf[l.slot(l.wave)];
    o[0] = w.n; o[1] = w.mean; o[2] = w.m2;
  }
  __syncthreads();
  float n = 0.f, sum = 0.f, m2 = 0.f;
  for (int i = 0; i < l.waves; ++i) {
    const float* o = buf[l.slot(l.first_wave() + i)];
    n += o[0];
    sum += o[0] * o[1];
  }
  const float mean = sum / n;
  for (int i = 0; i < l.waves; ++i) {
    const float* o = buf[l.slot(l.first_wave() + i)];
    const float e = o[1] - mean;
    m2 += o[2] + o[0] * e * e;
  }
  return {n, mean, m2};
}
__device__ __forceinline__ void team_sums(const Lane& l, const Team& t, float (&s)[2], float (*buf)[3]) {
  l.wave_sums(t, s);
  if (t.ttlog <= 6) return;
  if ((threadIdx.x & 63) == (l.gl << t.mlog & 63)) {
    float* o = buf[l.slot(l.wave)];
    o[0] = s[0]; o[1] = s[1];
  }
  __syncthreads();
  s[0] = s[1] = 0.f;
  for (int i = 0; i < l.waves; ++i) {
    const float* o = buf[l.slot(l.first_wave() + i)];
    s[0] += o[0];
    s[1] += o[1];
  }
}

// Moments about `pivot` of KP pieces, rows of which are in
template <bool FULL, typename T, int KP> __device__ __forceinline__ Moments moments_of(Raw8<T> (&x)[KP], int rows, int n, float pivot) {
  float s = 0.f;
#pragma unroll
  for (int k = 0; k < KP; ++k)
    if (k < rows) {
      const F8 f = widen(x[k]);
#pragma unroll
      for (int i = 0; i < 8; ++i) s += FULL || i < n ? f.v[i] - pivot : 0.f;
    }
  Moments m = {(float)(rows * n), 0.f, 0.f};
  if (rows * n == 0) return m;
  m.mean = s / m.n;
  as_held(x);
#pragma unroll
  for (int k = 0; k < KP; ++k)
    if (k < rows) {
      const F8 f = widen(x[k]);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float d = FULL || i < n ? (f.v[i] - pivot) - m.mean : 0.f;
        m.m2 = fmaf(d, d, m.m2);
      }
    }
  return m;
}

struct Columns { F8 ga, be; };
__device__ __forceinline__ Columns columns_of(const Norm& p, const Lane& l) {
  Columns o;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    o.ga.v[i] = i < l.n ? p.gamma ? p.gamma[l.c + i] : 1.f : 0.f;
    o.be.v[i] = i < l.n && p.beta ? p.beta[l.c + i] : 0.f;
  }
  return o;
}

enum { WHOLE, SUMS, OUTPUTS };   // an image at a time, or the two launches of segments

// A workgroup's place: bundles of channels run fastest, and each XCD gets a run of them, so that neighbours share what they read in its cache
struct Place { int bundle, slice, seg; };
__device__ __forceinline__ bool place_of(const NormParams& p, Place* at) {
  const int total = p.bundles * p.slices * p.segs, run = (total + 7) >> 3, s = (int)blockIdx.x >> 3, id = ((int)blockIdx.x & 7) * run + s;
  if (s >= run || id >= total) return false;
  at->bundle = id % p.bundles;
  const int rest = id / p.bundles;
  at->slice = rest % p.slices;
  at->seg = rest / p.slices;
  return true;
}

template <typename T, int F, int NT, int KP, int PHASE, bool FULL> __global__ __launch_bounds__(NT) void norm_fwd_kernel(NormParams p) {
  __shared__ float buf[2][NT][3];
  Place at;
  if (!place_of(p, &at)) return;
  const Lane l(p, at.bundle);
  const int teams = NT >> p.t.ttlog;
  const i64 beg = at.seg * p.seg, end = beg + p.seg < p.n.P ? beg + p.seg : p.n.P;
  const Columns col = PHASE == SUMS ? Columns{} : columns_of(p.n, l);
  const float count = (float)p.n.P * (float)p.cg;
  int turn = 0;
  for (i64 m0 = (i64)at.slice * teams; m0 < p.n.M; m0 += (i64)p.slices * teams, turn ^= 1) {   // (every lane of the workgroup takes part in the barrier)
    const i64 m = m0 + l.team;
    const bool live = m < p.n.M && l.n;
    const T* x = static_cast<const T*>(p.n.x) + (m * p.n.P) * p.n.ldx + l.c;
    const float pivot = live ? to_f32(x[l.g * p.cg - l.c]) : 0.f;   // (the group's first value)
    T* y = static_cast<T*>(p.n.y) + (m * p.n.P) * p.n.ldy + l.c;
    Raw8<T> v[KP];
    auto load = [&](i64 px) {   // rows of this lane from px on
      const i64 left = end - px;
      const int rows = !live || left <= 0 ? 0 : (int)((left + l.RT - 1) / l.RT < KP ? (left + l.RT - 1) / l.RT : KP);
#pragma unroll
      for (int k = 0; k < KP; ++k)
        if (k < rows) v[k] = load_piece<FULL>(x + (px + (i64)k * l.RT) * p.n.ldx, l.n);
      return rows;
    };
    auto put = [&](i64 px, int rows, float mean, float r) {
      as_held(v);
#pragma unroll
      for (int k = 0; k < KP; ++k)
        if (k < rows) {
          F8 f = widen(v[k]);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            float z = fmaf((f.v[i] - mean) * r, col.ga.v[i], col.be.v[i]), df;
            act_of<T, F>(z, &f.v[i], &df);
          }
          store_piece<FULL>(y + (px + (i64)k * l.RT) * p.n.ldy, l.n, f);
        }
    };
    auto keep = [&](float mean, float r) {
      if (p.n.stats && live && l.first && l.section == 0 && at.seg == 0)
        *reinterpret_cast<float2*>(p.n.stats + (m * p.n.groups + l.g) * 2) = make_float2(mean, r);
    };
    if constexpr (PHASE == WHOLE) {
      const int rows = load(beg + l.r);
      const Moments a = team_moments(l, p.t, moments_of<FULL>(v, rows, l.n, pivot), buf[turn]);
      const float r = 1.f / sqrtf(a.m2 / count + p.n.eps), mean = pivot + a.mean;
      put(beg + l.r, rows, mean, r);
      keep(mean, r);
    } else if constexpr (PHASE == SUMS) {
      Moments a = {0.f, 0.f, 0.f};
      for (i64 px = beg + l.r; px < end; px += (i64)KP * l.RT) {
        const int rows = load(px);
        merge(a, moments_of<FULL>(v, rows, l.n, pivot));
      }
      a = team_moments(l, p.t, a, buf[turn]);
      if (live && l.first) *reinterpret_cast<float2*>(l.entry(p, m, at.seg * p.sections + l.section)) = make_float2(a.mean, a.m2);
    } else {
      Moments a = {0.f, 0.f, 0.f};
      if (live)
        for (int s = 0; s < p.segs; ++s)
          for (int e = 0; e < p.sections; ++e) {
            const float2 q = *reinterpret_cast<const float2*>(l.entry(p, m, s * p.sections + e));
            const i64 px = p.n.P - s * p.seg < p.seg ? p.n.P - s * p.seg : p.seg;
            merge(a, {(float)px * (float)min(p.span, p.cg - e * p.span), q.x, q.y});
          }
      const float r = 1.f / sqrtf(a.m2 / count + p.n.eps), mean = pivot + a.mean;
      for (i64 px = beg + l.r; px < end; px += (i64)KP * l.RT) put(px, load(px), mean, r);
      keep(mean, r);
    }
  }
}

// dxhat = gamma dz, dz = dy f'(z);  dx = r (dxhat - mean(dxhat) - xhat mean(dxhat xhat)),  dgamma = sum dz xhat,  dbeta = sum dz
template <typename T, int F, int NT, int KP, int PHASE, bool FULL> __global__ __launch_bounds__(NT) void norm_bwd_kernel(NormParams p) {
  __shared__ float buf[2][NT][3];
  extern __shared__ float cols[];   // [waves][64][16]
  Place at;
  if (!place_of(p, &at)) return;
  const Lane l(p, at.bundle);
  const int teams = NT >> p.t.ttlog;
  const i64 beg = at.seg * p.seg, end = beg + p.seg < p.n.P ? beg + p.seg : p.n.P;
  const Columns col = columns_of(p.n, l);
  const float count = (float)p.n.P * (float)p.cg;
  F8 dga = {}, dbe = {};
  int turn = 0;
  for (i64 m0 = (i64)at.slice * teams; m0 < p.n.M; m0 += (i64)p.slices * teams, turn ^= 1) {
    const i64 m = m0 + l.team;
    const bool live = m < p.n.M && l.n;
    const T* x = static_cast<const T*>(p.n.x) + (m * p.n.P) * p.n.ldx + l.c;
    const T* dy = static_cast<const T*>(p.n.dy) + (m * p.n.P) * p.n.ldy + l.c;
    const float2 st = live ? *reinterpret_cast<const float2*>(p.n.stats + (m * p.n.groups + l.g) * 2) : make_float2(0.f, 0.f);
    const float mean = st.x, r = st.y;
    Raw8<T> v[KP], d[KP];
    auto load = [&](i64 px) {
      const i64 left = end - px;
      const int rows = !live || left <= 0 ? 0 : (int)((left + l.RT - 1) / l.RT < KP ? (left + l.RT - 1) / l.RT : KP);
#pragma unroll
      for (int k = 0; k < KP; ++k)
        if (k < rows) {
          v[k] = load_piece<FULL>(x + (px + (i64)k * l.RT) * p.n.ldx, l.n);
          d[k] = load_piece<FULL>(dy + (px + (i64)k * l.RT) * p.n.ldy, l.n);
        }
      return rows;
    };
    auto dz_of = [&](float xv, float dyv, int i, float* xhat) {
      *xhat = (xv - mean) * r;
      if constexpr (F == CONVBN_NORM_NONE) return dyv;
      float f, df;
      act_of<T, F>(fmaf(*xhat, col.ga.v[i], col.be.v[i]), &f, &df);
      return dyv * df;
    };
    auto add_up = [&](int rows, float (&s)[2]) {
#pragma unroll
      for (int k = 0; k < KP; ++k)
        if (k < rows) {
          const F8 a = widen(v[k]), b = widen(d[k]);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            float xhat;
            const float dz = FULL || i < l.n ? dz_of(a.v[i], b.v[i], i, &xhat) : xhat = 0.f, q = dz * xhat;
            dbe.v[i] += dz;
            dga.v[i] += q;
            s[0] = fmaf(dz, col.ga.v[i], s[0]);
            s[1] = fmaf(q, col.ga.v[i], s[1]);
          }
        }
    };
    auto put = [&](i64 px, int rows, float s0, float s1) {
      as_held(v);
      as_held(d);
#pragma unroll
      for (int k = 0; k < KP; ++k)
        if (k < rows) {
          const F8 a = widen(v[k]), b = widen(d[k]);
          const i64 o = (m * p.n.P + px + (i64)k * l.RT) * p.n.ldx + l.c;
          F8 f;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            float xhat;
            const float dz = dz_of(a.v[i], b.v[i], i, &xhat);
            f.v[i] = r * (fmaf(dz, col.ga.v[i], -s0) - xhat * s1);
          }
          if (p.n.add) {
            const F8 e = widen(load_piece<FULL>(static_cast<const T*>(p.n.add) + o, l.n));
#pragma unroll
            for (int i = 0; i < 8; ++i) f.v[i] += e.v[i];
          }
          store_piece<FULL>(static_cast<T*>(p.n.dx) + o, l.n, f);
        }
    };
    if constexpr (PHASE == WHOLE) {
      float s[2] = {0.f, 0.f};
      const int rows = load(beg + l.r);
      add_up(rows, s);
      if (p.n.dx) {
        team_sums(l, p.t, s, buf[turn]);
        put(beg + l.r, rows, s[0] / count, s[1] / count);
      }
    } else if constexpr (PHASE == SUMS) {
      float s[2] = {0.f, 0.f};
      for (i64 px = beg + l.r; px < end; px += (i64)KP * l.RT) add_up(load(px), s);
      team_sums(l, p.t, s, buf[turn]);
      if (live && l.first) *reinterpret_cast<float2*>(l.entry(p, m, at.seg * p.sections + l.section)) = make_float2(s[0], s[1]);
    } else {
      float s0 = 0.f, s1 = 0.f;
      if (live)
        for (int s = 0; s < p.segs * p.sections; ++s) {
          const float2 q = *reinterpret_cast<const float2*>(l.entry(p, m, s));
          s0 += q.x;
          s1 += q.y;
        }
      for (i64 px = beg + l.r; px < end; px += (i64)KP * l.RT) put(px, load(px), s0 / count, s1 / count);
    }
  }
  if (PHASE == OUTPUTS || !p.sums) return;
  // lanes of the same channels: those of a wave by shuffles, then the waves
  for (int o = 1 << l.lpr; o < 64; o <<= 1)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      dga.v[i] += __shfl_xor(dga.v[i], o, 64);
      dbe.v[i] += __shfl_xor(dbe.v[i], o, 64);
    }
  const int lane = threadIdx.x & 63, hop = l.lpr > 6 ? 1 << (l.lpr - 6) : 1;   // waves with the same channels are `hop` apart
  if (NT / 64 > hop) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      cols[(l.wave * 16 + i) * 64 + lane] = dga.v[i];
      cols[(l.wave * 16 + 8 + i) * 64 + lane] = dbe.v[i];
    }
    __syncthreads();
    if (l.wave >= hop) return;
    for (int w = l.wave + hop; w < NT / 64; w += hop)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        dga.v[i] += cols[(w * 16 + i) * 64 + lane];
        dbe.v[i] += cols[(w * 16 + 8 + i) * 64 + lane];
      }
  }
  if ((int)threadIdx.x < 1 << l.lpr) {
    float* out = p.sums + ((i64)(at.seg * p.slices + at.slice) * p.n.C + l.c) * 2;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < l.n) *reinterpret_cast<float2*>(out + 2 * i) = make_float2(dga.v[i], dbe.v[i]);
  }
}

// dgamma and dbeta: what `rows` workgroups found, [rows][C][2], in a fixed order; 16 threads a channel
__global__ __launch_bounds__(1024) void norm_join_kernel(const float* sums, int rows, int C, float* dgamma, float* dbeta) {
  __shared__ float2 meet[16][64];
  const int at = threadIdx.x & 63, q = threadIdx.x >> 6, c = blockIdx.x * 64 + at;
  float2 v = make_float2(0.f, 0.f);
  if (c < C) {
#pragma unroll 4
    for (int r = q; r < rows; r += 16) {
      const float2 w = *reinterpret_cast<const float2*>(sums + ((i64)r * C + c) * 2);
      v.x += w.x;
      v.y += w.y;
    }
  }
  meet[q][at] = v;
  __syncthreads();
  if (q || c >= C) return;
#pragma unroll
  for (int i = 1; i < 16; ++i) {
    v.x += meet[i][at].x;
    v.y += meet[i][at].y;
  }
  if (dgamma) dgamma[c] = v.x;
  if (dbeta) dbeta[c] = v.y;
}

int log2_up(i64 v) {
  int l = 0;
  while ((1LL << l) < v) ++l;
  return l;
}

constexpr int CUS = 256, MAX_SPAN = 8192;   // channels of a workgroup's lanes

// How a call is run: workgroups of nt, the teams, one launch or two
struct Plan {
  int nt;
  bool few, whole, full;   // few: at most two pieces a lane; full: pieces are
  NormParams p;
  size_t part, sums, total;
};
// Pieces that a lane's registers hold, of workgroups of 256 and 512
constexpr int most_of(int size, bool bwd, int nt) { return (nt == 512 ? bwd ? 16 : 32 : bwd ? 4 : 8) * 2 / size; }
constexpr int FEW = 2, STREAM = 4;   // pieces a lane: of short parts, of a turn of the segments' launches

Plan plan_of(const Norm& n, bool bwd) {
  Plan s = {};
  NormParams& p = s.p;
  p.n = n;
  p.cg = n.C / n.groups;
  s.full = p.cg % 8 == 0;
  p.sections = ceil_div(p.cg, MAX_SPAN);
  p.span = p.sections > 1 ? MAX_SPAN : p.cg;
  const int size = n.dtype == CONVBN_BF16 ? 2 : 4;
  Team& t = p.t;
  t.m = ceil_div(p.span, 8);
  t.mlog = log2_up(t.m);
  const int glog = log2_up(n.groups);
  // groups side by side until a pixel's part is 64 bytes, or until a wave is full of pieces of few channels
  while (t.nblog < glog && t.mlog + t.nblog < 6 && (p.cg << t.nblog) * size < 64) ++t.nblog;
  auto lanes = [&](int log) { return (n.P + (1LL << (log - t.lprlog)) - 1) >> (log - t.lprlog); };   // pieces of a lane
  auto fits = [&] { return p.sections == 1 && (t.lprlog <= 9 ? lanes(9) <= most_of(size, bwd, 512) : n.P <= FEW); };
  t.lprlog = t.mlog + t.nblog;
  // (backward holds twice as much: pixels' parts of 32 bytes if that keeps it in one launch)
  while (!fits() && t.nblog > 0 && (p.cg << (t.nblog - 1)) * size >= 32) {
    --t.nblog;
    --t.lprlog;
  }
  p.bundles = (int)((n.groups + (1LL << t.nblog) - 1) >> t.nblog) * p.sections;
  // one launch where the parts fit and are enough to fill a quarter of the chip, or short
  s.whole = fits() && (n.M * p.bundles >= CUS / 4 || n.P << t.lprlog <= 4096);
  t.ttlog = t.lprlog;
  if (s.whole) {
    while (t.ttlog < 8 && lanes(t.ttlog) > FEW) ++t.ttlog;
    if (t.ttlog == 8 && lanes(8) > most_of(size, bwd, 256)) t.ttlog = 9;
    s.nt = t.ttlog <= 8 ? 256 : 1 << t.ttlog;
    s.few = lanes(t.ttlog) <= FEW;
    p.segs = 1;
  } else {
    s.nt = 1024;
    t.ttlog = 10;
    // two workgroups a compute unit, each with two turns of its lanes at least
    const i64 turn = (i64)STREAM << (10 - t.lprlog);
    i64 segs = n.M ? 2 * CUS / (n.M * p.bundles) : 1;
    if (segs > n.P / (2 * turn)) segs = n.P / (2 * turn);
    p.segs = (int)(segs < 1 ? 1 : segs < 64 ? segs : 64);
  }
  p.seg = (n.P + p.segs - 1) / p.segs;
  p.segs = (int)((n.P + p.seg - 1) / p.seg);
  const i64 teams = s.nt >> t.ttlog, each = (n.M + teams - 1) / teams;
  auto bounded = [&](i64 most) { return (int)(each < 1 ? 1 : each < most ? each : most < 1 ? 1 : most); };
  const i64 side = (i64)p.bundles * p.segs;
  p.slices = bwd ? bounded((s.nt == 256 ? 8 : s.nt == 512 ? 4 : 2) * CUS / side) : bounded((1LL << 22) / side);
  if (bwd) s.sums = align_up((size_t)p.slices * p.segs * n.C * 8, 256);
  if (!s.whole) s.part = align_up((size_t)n.M * n.groups * p.segs * p.sections * 8, 256);
  s.total = s.part + s.sums;
  return s;
}

// Calls f(T, activation)
template <class F> hipError_t by_type(const Norm& p, F&& f) {
  using std::integral_constant;
  auto with = [&](auto t) {
    switch (p.f) {
      case CONVBN_NORM_RELU: return f(t, integral_constant<int, CONVBN_NORM_RELU>{});
      case CONVBN_NORM_SILU: return f(t, integral_constant<int, CONVBN_NORM_SILU>{});
      case CONVBN_NORM_GELU: return f(t, integral_constant<int, CONVBN_NORM_GELU>{});
    }
    return f(t, integral_constant<int, CONVBN_NORM_NONE>{});
  };
  return p.dtype == CONVBN_BF16 ? with(bf16_t{}) : with(float{});
}
int grid_of(const NormParams& p) { return (p.bundles * p.slices * p.segs + 7) / 8 * 8; }

template <bool BWD, typename T, int F, int NT, int KP, int PHASE, bool FULL> hipError_t run(const NormParams& p, hipStream_t st) {
  if constexpr (BWD) {
    constexpr int LDS = NT * 64;
    static LdsLimitOnce once;
    auto* k = &norm_bwd_kernel<T, F, NT, KP, PHASE, FULL>;
    const hipError_t e = set_lds_limit_once(once, (const void*)k, LDS);
    if (e != hipSuccess) return e;
    k<<<grid_of(p), NT, p.sums && PHASE != OUTPUTS ? LDS : 0, st>>>(p);
  } else {
    norm_fwd_kernel<T, F, NT, KP, PHASE, FULL><<<grid_of(p), NT, 0, st>>>(p);
  }
  return hipGetLastError();
}
template <bool BWD, typename T, int F, bool FULL> hipError_t run_plan(const Plan& s, hipStream_t st) {
  constexpr int SIZE = sizeof(T), KP = BWD ? STREAM / 2 : STREAM;
  if (!s.whole) {
    const hipError_t e = run<BWD, T, BWD ? F : (int)CONVBN_NORM_NONE, 1024, KP, SUMS, FULL>(s.p, st);
    return e != hipSuccess || (BWD && !s.p.n.dx) ? e : run<BWD, T, F, 1024, KP, OUTPUTS, FULL>(s.p, st);
  }
  if (s.nt == 1024) return run<BWD, T, F, 1024, FEW, WHOLE, FULL>(s.p, st);
  if constexpr (FULL) {   // (others are few: they do with the larger kernels)
    if (s.few) return s.nt == 256 ? run<BWD, T, F, 256, FEW, WHOLE, FULL>(s.p, st) : run<BWD, T, F, 512, FEW, WHOLE, FULL>(s.p, st);
  }
  return s.nt == 256 ? run<BWD, T, F, 256, most_of(SIZE, BWD, 256), WHOLE, FULL>(s.p, st)
                     : run<BWD, T, F, 512, most_of(SIZE, BWD, 512), WHOLE, FULL>(s.p, st);
}
template <bool BWD> hipError_t run_norm(const Plan& s, hipStream_t st) {
  return by_type(s.p.n, [&](auto t, auto f) {
    return s.full ? run_plan<BWD, decltype(t), f.value, true>(s, st) : run_plan<BWD, decltype(t), f.value, false>(s, st);
  });
}

}  // namespace
}  // namespace convbn
