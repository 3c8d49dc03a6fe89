// Group norm with an activation, channels last, forward and backward.
//
// A team of lanes takes some neighbouring groups of an image.  A lane holds pieces of eight channels of one group: v counts the pieces of a
// group's pixel, then come the groups of the team, then the pixels, so that neighbouring lanes read neighbouring memory and a group's lanes meet by
// exchanging along the bits of v and of the pixel: within a wave by shuffles, between waves through LDS, one barrier an image.  A wave takes its values
// twice: for a number near their mean, and for the sums of the differences to that number and of their squares.  So neither the mean nor the variance loses
// bits to values that lie far from zero, nor to one that lies far from the others.
//
// Where a team's part of an image fits the registers (x forward, x and dy backward) it is read once: one launch that reads and writes
// each number once.  Larger parts, and images that are too few to fill the chip, go in two launches: the sums of segments of the
// pixels, and then the outputs, for which every workgroup merges its groups' segments for itself; the second reading is partly from the
// last-level cache.
//
// Backward walks several images with the same channels, so that dgamma and dbeta gather in registers; a launch joins what the workgroups found.
//
// Bound by memory where it is large: 8192 tokens of 4096 forward 41 us (134 MB, 3.3 TB/s) and backward 44 (201 MB, 4.6); 32 x 56 x 56 x 256, whose 51 MB the
// last-level cache holds, forward 27, backward 28 + 29 and the join 5.  Small calls are bound by their launches: 49 x 2048 in one of 4.2 us.
#pragma once
#include "f8_code.h"

namespace convbn {

namespace {

struct Team { int m, mlog, nblog, lprlog, ttlog; };   // pieces of a group's pixel; lanes of a group's pixel, groups, lanes of a pixel, of the team: powers of two

struct NormParams {
  Norm n;
  Team t;
  int cg, bundles;      // channels of a group, teams side by side
  unsigned per_bundle, per_slice;   // ceil(2^32 / bundles), ceil(2^32 / slices): exact for the small numbers here; 0: divide by one
  int linelog;          // neighbouring bundles on a cache line: a power of two
  int span, sections;   // a group of more channels than a workgroup has lanes for: sections of `span` channels, a team each
  int slices;           // workgroups along the images (each takes every slices'th team of images)
  int segs;             // segments of the pixels
  i64 seg;              // pixels of one
  double2* part;        // sums of the segments, [M][groups][segs * sections]
  float* sums;          // [slices * segs][C][2]: dgamma, dbeta; null: not wanted
};

template <typename T, int F> __device__ __forceinline__ void act_of(float z, float* f, float* df) {
  if constexpr (F == CONVBN_NORM_NONE) { *f = z; *df = 1.f; }
  else if constexpr (F == CONVBN_NORM_RELU) { *f = z < 0.f ? 0.f : z; *df = z > 0.f ? 1.f : 0.f; }   // (NaN stays)
  else gate_of<T, F == CONVBN_NORM_SILU ? CONVBN_GATE_SILU : CONVBN_GATE_GELU>(z, f, df);
}

// Pieces of a group's channels: whole ones of eight (EIGHTS), of eight with a shorter last one (TAIL: groups of other sizes, of some length), or single
// channels (ONES: short groups of other sizes).  n: channels of this one.
enum { EIGHTS, TAIL, ONES };
template <int V> constexpr int width_of = V == ONES ? 1 : 8;
template <typename T, int V> struct Held { Raw8<T> r; };
template <typename T> struct Held<T, ONES> { float r; };
template <int N> struct Vals { float v[N]; };

template <typename T, int V> __device__ __forceinline__ Held<T, V> load_piece(const T* p, int n) {
  Held<T, V> h;
  if constexpr (V == ONES) {
    h.r = to_f32(*p);
  } else if (V == EIGHTS || n == 8) {
    h.r = *reinterpret_cast<const Raw8<T>*>(p);
  } else {
    F8 f;
#pragma unroll
    for (int i = 0; i < 8; ++i) f.v[i] = i < n ? to_f32(p[i]) : 0.f;
    h.r = narrow<T>(f);
  }
  return h;
}
template <typename T, int V> __device__ __forceinline__ Vals<width_of<V>> vals(const Held<T, V>& h) {
  if constexpr (V == ONES) {
    return {{h.r}};
  } else {
    const F8 f = widen(h.r);
    return {{f.v[0], f.v[1], f.v[2], f.v[3], f.v[4], f.v[5], f.v[6], f.v[7]}};
  }
}
// Results go past the L2 caches, which leaves them to what is read again.  us, each call over and over, in brackets if they stay: 8192 tokens of 4096 forward 40 (41), backward
// 47 (46), fp32 51 (49) and 77 (83); 32 x 28 x 28 x 512 18 (20) and 24 (26); 32 x 56 x 56 x 256 27 (23) and 52 (52).
template <typename T, int V> __device__ __forceinline__ void store_piece(T* p, int n, const Vals<width_of<V>>& f) {
  if constexpr (V == ONES) {
    *p = from_f32<T>(f.v[0]);
  } else {
    if (V == EIGHTS || n == 8) {
      store8<T, true>(p, 0, 8, F8{{f.v[0], f.v[1], f.v[2], f.v[3], f.v[4], f.v[5], f.v[6], f.v[7]}});
      return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = from_f32<T>(f.v[i]);
  }
}
// From here on the pieces are what is in their registers: else the compiler keeps them as the eight fp32 numbers that an earlier pass made of
// each, which take twice the room (512 lanes of 32 pieces: 142 registers to memory)
template <typename T, int V, int KP> __device__ __forceinline__ void as_held(Held<T, V> (&x)[KP]) {
  if constexpr (sizeof(T) == 2 && V != ONES) {
#pragma unroll
    for (int k = 0; k < KP; ++k) {
      u32x4 a = x[k].r.a;
      asm volatile("" : "+v"(a));
      x[k].r.a = a;
    }
  }
}

template <int CTRL> __device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ float across16(float v) {   // + lane ^ 16
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float across32(float v) {   // + lane ^ 32
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// ... and for 64 bits, as two halves
template <int CTRL> __device__ __forceinline__ double dpp(double v) {
  const int2 q = __builtin_bit_cast(int2, v);
  return __builtin_bit_cast(double, make_int2(__builtin_amdgcn_update_dpp(0, q.x, CTRL, 0xf, 0xf, false), __builtin_amdgcn_update_dpp(0, q.y, CTRL, 0xf, 0xf, false)));
}
__device__ __forceinline__ double across16(double v) {
  const uint2 q = __builtin_bit_cast(uint2, v);
  const auto x = __builtin_amdgcn_permlane16_swap(q.x, q.x, false, false), y = __builtin_amdgcn_permlane16_swap(q.y, q.y, false, false);
  return __builtin_bit_cast(double, make_uint2(x[0], y[0])) + __builtin_bit_cast(double, make_uint2(x[1], y[1]));
}
__device__ __forceinline__ double across32(double v) {
  const uint2 q = __builtin_bit_cast(uint2, v);
  const auto x = __builtin_amdgcn_permlane32_swap(q.x, q.x, false, false), y = __builtin_amdgcn_permlane32_swap(q.y, q.y, false, false);
  return __builtin_bit_cast(double, make_uint2(x[0], y[0])) + __builtin_bit_cast(double, make_uint2(x[1], y[1]));
}
// Sums over 16 lanes
template <int N, typename A> __device__ __forceinline__ void row_sums(A (&s)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) s[i] += dpp<0x121>(s[i]);
#pragma unroll
  for (int i = 0; i < N; ++i) s[i] += dpp<0x122>(s[i]);
#pragma unroll
  for (int i = 0; i < N; ++i) s[i] += dpp<0x124>(s[i]);
#pragma unroll
  for (int i = 0; i < N; ++i) s[i] += dpp<0x128>(s[i]);
}

// A lane's place
struct Lane {
  int wave, waves, r, RT, gl, c, n, lpr;   // waves: of the team; c: first channel, n: channels of the piece (0: none), gl: group in the team
  int g, section, team;
  bool first;                              // the group's (or its section's) first lane
  template <int W> __device__ __forceinline__ void init(const NormParams& p, int bundle) {
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
    const int at = section * p.span + v * W;   // in the group
    c = g * p.cg + at;
    n = g < p.n.groups && v < p.t.m ? max(0, min(W, p.cg - at)) : 0;
    first = n && r == 0 && v == 0;
  }
  // this lane's entry of the segments' sums of image m
  __device__ __forceinline__ double2* entry(const NormParams& p, i64 m, int i) const {
    return p.part + (m * p.n.groups + g) * (p.segs * p.sections) + i;
  }
  // Sums over a group's lanes of this wave.  Its pieces are the low bits of a lane; its pixels the high ones, turned within rows of 16 (a team
  // that has several pixels side by side has 16 lanes at least) and exchanged between rows.
  template <int N, typename A> __device__ __forceinline__ void wave_sums(const Team& t, A (&s)[N]) const {
    auto each = [&](auto f) {
#pragma unroll
      for (int i = 0; i < N; ++i) s[i] = f(s[i]);
    };
    if (t.mlog > 0) each([](A v) { return v + dpp<0xb1>(v); });    // lane ^ 1
    if (t.mlog > 1) each([](A v) { return v + dpp<0x4e>(v); });    // lane ^ 2
    if (t.mlog > 2) each([](A v) { return v + dpp<0x141>(v); });   // 7 - lane: fours are equal by now
    if (t.mlog > 3) each([](A v) { return v + dpp<0x140>(v); });   // 15 - lane
    if (t.ttlog > t.lprlog) {
      if (t.lprlog < 1) each([](A v) { return v + dpp<0x121>(v); });
      if (t.lprlog < 2) each([](A v) { return v + dpp<0x122>(v); });
      if (t.lprlog < 3) each([](A v) { return v + dpp<0x124>(v); });
      if (t.lprlog < 4) each([](A v) { return v + dpp<0x128>(v); });
    }
    if (t.mlog > 4 || (t.lprlog < 5 && t.ttlog > 4)) each([](A v) { return across16(v); });
    if (t.mlog > 5 || (t.lprlog < 6 && t.ttlog > 5)) each([](A v) { return across32(v); });
  }
  // One number for all of a group's lanes of this wave from what wave_sums left in them: turned within rows they add in different orders
  __device__ __forceinline__ float same(const Team& t, float v) const {
    return t.ttlog > t.lprlog && t.lprlog < 4 ? __shfl(v, (threadIdx.x & 63 & ~((1u << t.ttlog) - 1)) + (gl << t.mlog), 64) : v;
  }
  // Where this wave's sums go and the team's begin
  __device__ __forceinline__ int slot(const Team& t, int w) const { return (w << t.nblog) + gl; }
  __device__ __forceinline__ int first_wave() const { return wave & ~(waves - 1); }
  __device__ __forceinline__ bool writes(const Team& t) const { return (int)(threadIdx.x & 63) == (gl << t.mlog & 63); }
};

// What lanes' sums are added up in: fp32, or, in front of a ReLU, 64 bits (what is left to err is then a lane's own sums, some 6e-9 of a deviation)
template <int F> using Sum = std::conditional_t<F == CONVBN_NORM_RELU, double, float>;
// Moments about a number that is kept beside them
template <typename A> struct Moments { A n, mean, m2; };
// Moments of IM images' groups: in, of the wave's lanes, about c; out, of the team, about the first wave's c.  That one's distance to the others' is at most
// some deviations of the values, so that fp32 keeps what counts (about one value of the group it would not: that may lie as many deviations away as the root of the
// group's size).  buf: [IM][waves << nblog] entries of four
template <int IM, typename A> __device__ __forceinline__ void join_waves(const Lane& l, const Team& t, Moments<A> (&a)[IM], float (&c)[IM], A* buf, int entries) {
  if (t.ttlog <= 6) return;
  if (l.writes(t)) {
#pragma unroll
    for (int i = 0; i < IM; ++i) {
      A* o = buf + (i * entries + l.slot(t, l.wave)) * 4;
      o[0] = a[i].n; o[1] = a[i].mean; o[2] = a[i].m2; o[3] = (A)c[i];
    }
  }
  __syncthreads();
  // wave w's, about the first one's c
  auto of = [&](int i, int w) {
    const A* o = buf + (i * entries + l.slot(t, l.first_wave() + w)) * 4;
    return Moments<A>{o[0], o[3] - (A)c[i] + o[1], o[2]};
  };
#pragma unroll
  for (int i = 0; i < IM; ++i) c[i] = (float)buf[(i * entries + l.slot(t, l.first_wave())) * 4 + 3];
  if (t.nblog == 0) {   // one group: 16 lanes read a wave's each
    const int w = threadIdx.x & 15;
    A mean[IM], s[2 * IM], q[IM];
#pragma unroll
    for (int i = 0; i < IM; ++i) {
      a[i] = w < l.waves ? of(i, w) : Moments<A>{A(0), A(0), A(0)};
      s[2 * i] = a[i].n;
      s[2 * i + 1] = a[i].n * a[i].mean;
    }
    row_sums(s);
#pragma unroll
    for (int i = 0; i < IM; ++i) {
      mean[i] = s[2 * i] > A(0) ? s[2 * i + 1] / s[2 * i] : A(0);
      const A e = a[i].mean - mean[i];
      q[i] = a[i].m2 + a[i].n * e * e;
    }
    row_sums(q);
#pragma unroll
    for (int i = 0; i < IM; ++i) a[i] = {s[2 * i], mean[i], q[i]};
    return;
  }
#pragma unroll
  for (int i = 0; i < IM; ++i) {
    A n = A(0), sum = A(0), m2 = A(0);
    for (int w = 0; w < l.waves; ++w) {
      const Moments<A> o = of(i, w);
      n += o.n;
      sum += o.n * o.mean;
    }
    const A mean = n > A(0) ? sum / n : A(0);
    for (int w = 0; w < l.waves; ++w) {
      const Moments<A> o = of(i, w);
      const A e = o.mean - mean;
      m2 += o.m2 + o.n * e * e;
    }
    a[i] = {n, mean, m2};
  }
}
// ... of lanes' that have each their own, about c
__device__ __forceinline__ void team_moments(const Lane& l, const Team& t, Moments<double> (&a)[1], float c, double* buf, int entries) {
  double s[2] = {a[0].n, a[0].n * a[0].mean};
  l.wave_sums(t, s);
  const double mean = s[0] > 0. ? s[1] / s[0] : 0., d = a[0].mean - mean;
  double q[1] = {a[0].n > 0. ? a[0].m2 + a[0].n * d * d : 0.};
  l.wave_sums(t, q);
  a[0] = {s[0], mean, q[0]};
  float about[1] = {c};
  join_waves(l, t, a, about, buf, entries);
}
// A group's statistics from its moments about c
struct Stats { double mean, r; };
template <typename A> __device__ __forceinline__ Stats stats_of(const Moments<A>& a, float c, A count, float eps) {
  if constexpr (sizeof(A) == 8) return {c + a.mean, 1. / sqrt(a.m2 / count + eps)};
  else return {(double)c + a.mean, 1.f / sqrtf(a.m2 / count + eps)};
}
// The team's sums of IM pairs.  buf: [waves << nblog] entries of 2 IM
template <int IM> __device__ __forceinline__ void team_sums(const Lane& l, const Team& t, float (&s)[2 * IM], float* buf) {
  l.wave_sums(t, s);
  if (t.ttlog <= 6) return;
  if (l.writes(t)) {
#pragma unroll
    for (int i = 0; i < 2 * IM; ++i) buf[l.slot(t, l.wave) * 2 * IM + i] = s[i];
  }
  __syncthreads();
  if (t.nblog == 0) {
    const int w = threadIdx.x & 15;
#pragma unroll
    for (int i = 0; i < 2 * IM; ++i) s[i] = w < l.waves ? buf[(l.first_wave() + w) * 2 * IM + i] : 0.f;
    row_sums(s);
    return;
  }
#pragma unroll
  for (int i = 0; i < 2 * IM; ++i) s[i] = 0.f;
  for (int w = 0; w < l.waves; ++w)
#pragma unroll
    for (int i = 0; i < 2 * IM; ++i) s[i] += buf[l.slot(t, l.first_wave() + w) * 2 * IM + i];
}

// Of KP pieces, rows of which are in: the sum of the differences to `pivot`
template <typename T, int V, int KP> __device__ __forceinline__ float sum_about(const Held<T, V> (&x)[KP], int rows, int n, float pivot) {
  float s = 0.f;
#pragma unroll
  for (int k = 0; k < KP; ++k)
    if (k < rows) {
      const auto f = vals(x[k]);
#pragma unroll
      for (int i = 0; i < width_of<V>; ++i) s += V != TAIL || i < n ? f.v[i] - pivot : 0.f;
    }
  return s;
}
// ... and of their squares
struct Sums { float m1, m2; };
template <typename T, int V, int KP> __device__ __forceinline__ Sums sums_about(Held<T, V> (&x)[KP], int rows, int n, float c) {
  as_held(x);
  Sums s = {0.f, 0.f};
#pragma unroll
  for (int k = 0; k < KP; ++k)
    if (k < rows) {
      const auto f = vals(x[k]);
#pragma unroll
      for (int i = 0; i < width_of<V>; ++i) {
        const float d = V != TAIL || i < n ? f.v[i] - c : 0.f;
        s.m1 += d;
        s.m2 = fmaf(d, d, s.m2);
      }
    }
  return s;
}
// A lane's sums, turn by turn: each turn's about a number near its own mean, in fp32, and these about the first turn's in 64 bits.  What such a number is off by
// (2^-24 of the distance to `pivot` for each addition) is in the sum of the differences to it.
struct Turns {
  float c = 0.f;
  int n = 0;
  double m1 = 0., m2 = 0.;
  template <typename T, int V, int KP> __device__ __forceinline__ void add(Held<T, V> (&x)[KP], int rows, int channels, float pivot) {
    const int many = rows * channels;
    const float s = sum_about(x, rows, channels, pivot);
    if (many == 0) return;
    const float near = pivot + s / (float)many;
    const Sums q = sums_about(x, rows, channels, near);
    if (n == 0) c = near;
    const double e = (double)near - c;
    m1 += many * e + q.m1;
    m2 += q.m2 + e * (2. * q.m1 + many * e);
    n += many;
  }
  __device__ __forceinline__ Moments<double> about(float pivot) const {
    if (n == 0) return {0., 0., 0.};
    const double mean = m1 / n;
    return {(double)n, (double)c - pivot + mean, m2 - mean * m1};
  }
};
// The team's moments of IM images' pieces; c: in, a value of each group, out, what they are about
template <typename A, int IM, typename T, int V, int KP>
__device__ __forceinline__ void whole_moments(const Lane& l, const Team& t, Held<T, V> (&x)[IM][KP], const int (&rows)[IM], Moments<A> (&a)[IM], float (&c)[IM], A* buf, int entries) {
  float s[2 * IM];
#pragma unroll
  for (int i = 0; i < IM; ++i) {
    s[2 * i] = (float)(rows[i] * l.n);
    s[2 * i + 1] = sum_about(x[i], rows[i], l.n, c[i]);
  }
  l.wave_sums(t, s);
  A q[2 * IM];
#pragma unroll
  for (int i = 0; i < IM; ++i) {
    c[i] = l.same(t, s[2 * i] > 0.f ? c[i] + s[2 * i + 1] / s[2 * i] : c[i]);
    const Sums w = sums_about(x[i], rows[i], l.n, c[i]);
    q[2 * i] = w.m1;
    q[2 * i + 1] = w.m2;
  }
  l.wave_sums(t, q);
#pragma unroll
  for (int i = 0; i < IM; ++i) {
    const A n = s[2 * i], mean = n > A(0) ? q[2 * i] / n : A(0);
    a[i] = {n, mean, q[2 * i + 1] - mean * q[2 * i]};
  }
  join_waves(l, t, a, c, buf, entries);
}

template <int V> struct Columns { Vals<width_of<V>> ga, be; };
template <int V> __device__ __forceinline__ Columns<V> columns_of(const Norm& p, const Lane& l) {
  Columns<V> o;
  if (V == EIGHTS && l.n) {
    const F8 ga = p.gamma ? load8<float>(p.gamma, l.c, l.c + 8) : F8{{1, 1, 1, 1, 1, 1, 1, 1}}, be = p.beta ? load8<float>(p.beta, l.c, l.c + 8) : F8{};
#pragma unroll
    for (int i = 0; i < width_of<V>; ++i) {
      o.ga.v[i] = ga.v[i];
      o.be.v[i] = be.v[i];
    }
    return o;
  }
#pragma unroll
  for (int i = 0; i < width_of<V>; ++i) {
    o.ga.v[i] = i < l.n ? p.gamma ? p.gamma[l.c + i] : 1.f : 0.f;
    o.be.v[i] = i < l.n && p.beta ? p.beta[l.c + i] : 0.f;
  }
  return o;
}

enum { WHOLE, SUMS, OUTPUTS };   // an image at a time, or the two launches of segments

// Waves a SIMD that kernels shall have registers for which need about as many as that leaves: one more halves what is in flight (8192 tokens of 4096 backward
// 44 us with 128 registers, 63 with 129; sums of single channels, 64 registers, 8 x 3136 x 256 in groups of one)
constexpr int least_waves(bool bwd, int f, int size, int kp, int im, int phase, int v) {
  const bool relu = f == CONVBN_NORM_RELU;
  if (phase == SUMS && v == ONES) return bwd ? 1 : 8;
  if (phase != WHOLE || v != EIGHTS || kp > 2) return 1;
  if (!bwd) return !relu ? 1 : im == 1 ? 4 : 3;
  return f == CONVBN_NORM_NONE || (im == 1 && kp * size <= 4) ? 4 : relu && im == 1 ? 3 : 1;
}

// A lane's rows, one after the other.  WHOLE: 32-bit offsets from what is the same for the workgroup (plan_of sees to it), which take one register
// for all of them.
template <typename T, int PHASE> struct Rows {
  char* base;      // WHOLE: of the workgroup's image; else of this lane's channels in it
  unsigned off;
  i64 row, hop;    // bytes from a pixel, from a row of this lane to the next
  __device__ __forceinline__ Rows(const void* p, const Lane& l, i64 P, i64 ld, i64 m0) {
    row = ld * sizeof(T);
    hop = row * l.RT;
    base = static_cast<char*>(const_cast<void*>(p)) + m0 * P * row;
    off = (unsigned)(((l.team * P + l.r) * ld + l.c) * (int)sizeof(T));
    if constexpr (PHASE != WHOLE) base += l.team * P * row + l.c * (i64)sizeof(T);
  }
  __device__ __forceinline__ void from(i64 px) {   // (WHOLE: from its first)
    if constexpr (PHASE != WHOLE) base += px * row;
  }
  __device__ __forceinline__ T* next() {
    T* at = reinterpret_cast<T*>(PHASE == WHOLE ? base + off : base);
    base += hop;
    return at;
  }
};

// A workgroup's place: bundles of channels run fastest.  Neighbours whose parts of a pixel lie on the same cache line are on the same XCD; apart from
// that neighbours are on different ones, so that few images keep them all busy.
struct Place { int bundle, slice, seg; };
__device__ __forceinline__ bool place_of(const NormParams& p, Place* at) {
  const int total = p.bundles * p.slices * p.segs, s = (int)blockIdx.x >> 3, in = s & ((1 << p.linelog) - 1);
  const int id = ((s - in) << 3) + (((int)blockIdx.x & 7) << p.linelog) + in;
  if (id >= total) return false;
  const int rest = p.per_bundle ? (int)__umulhi((unsigned)id, p.per_bundle) : id;
  at->bundle = id - rest * p.bundles;
  at->seg = p.per_slice ? (int)__umulhi((unsigned)rest, p.per_slice) : rest;
  at->slice = rest - at->seg * p.slices;
  return true;
}
// Rows of a lane from px on
template <int KP> __device__ __forceinline__ int rows_from(const Lane& l, bool live, i64 px, i64 end) {
  const i64 n = (end - px + l.RT - 1) >> (31 - __clz(l.RT));
  return !live || n <= 0 ? 0 : n < KP ? (int)n : KP;
}

// Calls f for each of a group's segments, a lane of each wave for a part of them, and sums what they add to s (1 x 2289 x 1472, one group: the
// outputs' launch 13 us; every lane all of them, one after the other, 34).
template <int N, typename A, class F> __device__ __forceinline__ void over_entries(const NormParams& p, const Lane& l, A (&s)[N], F&& f) {
  const int lane = threadIdx.x & 63, of = p.t.nblog ? (lane >> l.lpr << p.t.mlog) | (lane & ((1 << p.t.mlog) - 1)) : lane;   // (groups side by side fit a wave)
  if (l.g < p.n.groups)
    for (int i = of; i < p.segs * p.sections; i += 64 >> p.t.nblog) f(i);
  l.wave_sums(p.t, s);
}

// IM: images at a time (WHOLE)
template <typename T, int F, int NT, int KP, int IM, int PHASE, int V>
__global__ __launch_bounds__(NT, least_waves(false, F, sizeof(T), KP, IM, PHASE, V)) void norm_fwd_kernel(NormParams p) {
  using A = std::conditional_t<PHASE == WHOLE, Sum<F>, double>;
  extern __shared__ __align__(16) unsigned char lds[];   // two turns' moments
  Place at;
  if (!place_of(p, &at)) return;
  Lane l;
  l.init<width_of<V>>(p, at.bundle);
  const int teams = NT >> p.t.ttlog, entries = NT / 64 << p.t.nblog;
  const i64 beg = at.seg * p.seg, end = beg + p.seg < p.n.P ? beg + p.seg : p.n.P;
  const A count = (A)p.n.P * (A)p.cg;
  auto live_at = [&](i64 m0) { return m0 + l.team < p.n.M && l.n; };
  auto pivot_at = [&](i64 m0) {   // the group's first value
    return live_at(m0) ? to_f32(static_cast<const T*>(p.n.x)[(m0 + l.team) * p.n.P * p.n.ldx + l.g * p.cg]) : 0.f;
  };
  auto load = [&](Held<T, V> (&v)[KP], i64 m0, i64 px) {
    Rows<T, PHASE> x(p.n.x, l, p.n.P, p.n.ldx, m0);
    const int rows = rows_from<KP>(l, live_at(m0), px, end);
    x.from(px);
#pragma unroll
    for (int k = 0; k < KP; ++k) {
      const T* q = x.next();
      if (k < rows) v[k] = load_piece<T, V>(q, l.n);
    }
    return rows;
  };
  Columns<V> col;
  if constexpr (PHASE != SUMS && IM > 1) col = columns_of<V>(p.n, l);
  auto put = [&](Held<T, V> (&v)[KP], i64 m0, i64 px, int rows, const Stats& z) {
    Rows<T, PHASE> y(p.n.y, l, p.n.P, p.n.ldy, m0);
    y.from(px);
    as_held(v);
    // (x - c) r + shift, c the mean and shift what rounding c leaves of it: x r - mean r would keep 2^-24 of mean r
    const float r = (float)z.r, c = (float)z.mean, shift = (float)((c - z.mean) * z.r);
#pragma unroll
    for (int k = 0; k < KP; ++k) {
      T* q = y.next();
      if (k >= rows) continue;
      auto f = vals(v[k]);
#pragma unroll
      for (int i = 0; i < width_of<V>; ++i) {
        float df;
        act_of<T, F>(fmaf(fmaf(f.v[i] - c, r, shift), col.ga.v[i], col.be.v[i]), &f.v[i], &df);
      }
      store_piece<T, V>(q, l.n, f);
    }
  };
  auto keep = [&](i64 m0, const Stats& z) {
    if (p.n.stats && live_at(m0) && l.first && l.section == 0 && at.seg == 0) {
      const float mean = (float)z.mean, r = (float)z.r;
      *reinterpret_cast<float4*>(p.n.stats + ((m0 + l.team) * p.n.groups + l.g) * 4) = make_float4(mean, (float)(z.mean - mean), r, (float)(z.r - r));
    }
  };
  const i64 stride = (i64)p.slices * teams * IM;
  int turn = 0;   // (every lane of the workgroup takes part in the barrier of every turn)
  for (i64 m0 = (i64)at.slice * teams * IM; m0 < p.n.M; m0 += stride, turn ^= 1) {
    A* const buf = reinterpret_cast<A*>(lds) + turn * IM * entries * 4;
    Held<T, V> v[IM][KP];
    Moments<A> a[IM];
    if constexpr (PHASE == WHOLE) {
      float c[IM];
      int rows[IM];
#pragma unroll
      for (int i = 0; i < IM; ++i) {
        c[i] = pivot_at(m0 + i * teams);
        rows[i] = load(v[i], m0 + i * teams, l.r);
      }
      if constexpr (IM == 1) col = columns_of<V>(p.n, l);
      whole_moments(l, p.t, v, rows, a, c, buf, entries);
#pragma unroll
      for (int i = 0; i < IM; ++i) {
        const Stats z = stats_of(a[i], c[i], count, p.n.eps);
        put(v[i], m0 + i * teams, l.r, rows[i], z);
        keep(m0 + i * teams, z);
      }
    } else {
      const i64 m = m0 + l.team;
      const float pivot = pivot_at(m0);
      if constexpr (PHASE == SUMS) {
        Turns sums;
        for (i64 px = beg + l.r; px < end; px += (i64)KP * l.RT) {
          const int rows = load(v[0], m0, px);
          sums.add(v[0], rows, l.n, pivot);
        }
        a[0] = sums.about(pivot);
        team_moments(l, p.t, a, pivot, buf, entries);
        if (live_at(m0) && l.first) *l.entry(p, m, at.seg * p.sections + l.section) = make_double2(a[0].mean, a[0].m2);
      } else {
        col = columns_of<V>(p.n, l);
        auto part = [&](int i) {
          const int s = i / p.sections, e = i - s * p.sections;
          const i64 px = p.n.P - s * p.seg < p.seg ? p.n.P - s * p.seg : p.seg;
          const double2 q = *l.entry(p, m, i);
          return Moments<A>{(A)px * (A)min(p.span, p.cg - e * p.span), (A)q.x, (A)q.y};
        };
        A sum[1] = {A(0)}, m2[1] = {A(0)};
        over_entries(p, l, sum, [&](int i) {
          const Moments<A> b = part(i);
          sum[0] += b.n * b.mean;
        });
        const A mean = sum[0] / count;
        over_entries(p, l, m2, [&](int i) {
          const Moments<A> b = part(i);
          const A d = b.mean - mean;
          m2[0] += b.m2 + b.n * d * d;
        });
        a[0] = {count, mean, m2[0]};
        const Stats z = stats_of(a[0], pivot, count, p.n.eps);
        for (i64 px = beg + l.r; px < end; px += (i64)KP * l.RT) {
          const int rows = load(v[0], m0, px);
          put(v[0], m0, px, rows, z);
        }
        keep(m0, z);
      }
    }
  }
}

// dxhat = gamma dz, dz = dy f'(z);  dx = r (dxhat - mean(dxhat) - xhat mean(dxhat xhat)),  dgamma = sum dz xhat,  dbeta = sum dz
template <typename T, int F, int NT, int KP, int IM, int PHASE, int V>
__global__ __launch_bounds__(NT, least_waves(true, F, sizeof(T), KP, IM, PHASE, V)) void norm_bwd_kernel(NormParams p) {
  constexpr int W = width_of<V>;
  extern __shared__ float cols[];   // two turns' sums; at the end the columns', [waves][2 W][64]
  Place at;
  if (!place_of(p, &at)) return;
  Lane l;
  l.init<W>(p, at.bundle);
  const int teams = NT >> p.t.ttlog, entries = NT / 64 << p.t.nblog;
  const i64 beg = at.seg * p.seg, end = beg + p.seg < p.n.P ? beg + p.seg : p.n.P;
  const Columns<V> col = columns_of<V>(p.n, l);
  const float count = (float)p.n.P * (float)p.cg;
  Vals<W> dga = {}, dbe = {};
  struct Image { Held<T, V> v[KP], d[KP]; float r, shift, mean, mean_l, r_l; int rows; };   // xhat = (x - mean) r + shift; RELU: the rest of the statistics
  auto live_at = [&](i64 m0) { return m0 + l.team < p.n.M && l.n; };
  auto stats_of = [&](Image& q, i64 m0) {
    const float4 st = live_at(m0) ? *reinterpret_cast<const float4*>(p.n.stats + ((m0 + l.team) * p.n.groups + l.g) * 4) : make_float4(0.f, 0.f, 0.f, 0.f);
    q.r = st.z;
    q.shift = -st.y * st.z;
    q.mean = st.x;
    q.mean_l = st.y;
    q.r_l = st.w;
  };
  auto load = [&](Image& q, i64 m0, i64 px) {
    Rows<T, PHASE> x(p.n.x, l, p.n.P, p.n.ldx, m0), dy(p.n.dy, l, p.n.P, p.n.ldy, m0);
    q.rows = rows_from<KP>(l, live_at(m0), px, end);
    x.from(px);
    dy.from(px);
#pragma unroll
    for (int k = 0; k < KP; ++k) {
      const T *a = x.next(), *b = dy.next();
      if (k >= q.rows) continue;
      q.v[k] = load_piece<T, V>(a, l.n);
      q.d[k] = load_piece<T, V>(b, l.n);
    }
  };
  // RELU: which of a piece's values passed, a bit each.  Values next to the border are looked at again with all bits: each that falls on the wrong side is off
  // by a whole gradient (2e-4 of dbeta's norm at 32 x 56 x 56 x 256).
  // (next to zero z is off by less than 2^-22 of beta, with which gamma xhat cancels, and 2^-21 of gamma times what rounding the mean left of xhat)
  float edge = 1.f, steep = 0.f;
#pragma unroll
  for (int i = 0; i < W; ++i) {
    edge = fmaxf(edge, fabsf(col.be.v[i]));
    steep = fmaxf(steep, fabsf(col.ga.v[i]));
  }
  edge *= 1e-6f;
  steep *= 1e-6f;
  auto passed = [&](const Image& q, const Vals<W>& x) {
    unsigned open = 0;
    if constexpr (F == CONVBN_NORM_RELU) {
      float near = INFINITY;
#pragma unroll
      for (int i = 0; i < W; ++i) {
        const float z = fmaf(fmaf(x.v[i] - q.mean, q.r, q.shift), col.ga.v[i], col.be.v[i]);
        open |= z > 0.f ? 1u << i : 0u;
        near = fminf(near, fabsf(z));
      }
      if (near < fmaf(steep, fabsf(q.shift), edge)) {
        // (x - mean) r with what each rounding leaves, in `dl` and `el`; the last product and its sum are rounded once, relative to a result next to 0
        open = 0;
#pragma unroll
        for (int i = 0; i < W; ++i) {
          const float d = x.v[i] - q.mean, back = d - x.v[i], dl = (x.v[i] - (d - back)) - (q.mean + back) - q.mean_l;
          const float e = d * q.r, el = fmaf(d, q.r, -e) + fmaf(d, q.r_l, dl * q.r);
          open |= fmaf(el, col.ga.v[i], fmaf(e, col.ga.v[i], col.be.v[i])) > 0.f ? 1u << i : 0u;
        }
      }
    }
    return open;
  };
  auto dz_of = [&](unsigned open, float xhat, float dyv, int i) {
    if constexpr (F == CONVBN_NORM_NONE) return dyv;
    if constexpr (F == CONVBN_NORM_RELU) return open >> i & 1 ? dyv : 0.f;   // (an infinite gradient behind a closed ReLU is none)
    float f, df;
    act_of<T, F>(fmaf(xhat, col.ga.v[i], col.be.v[i]), &f, &df);
    return dyv * df;
  };
  // what an image adds to a lane's columns, and s: the sums of dxhat and dxhat xhat
  auto add_up = [&](Image& q, float* s) {
    Vals<W> sz = {}, sx = {};
#pragma unroll
    for (int k = 0; k < KP; ++k)
      if (k < q.rows) {
        const auto a = vals(q.v[k]), b = vals(q.d[k]);
        const unsigned open = passed(q, a);
#pragma unroll
        for (int i = 0; i < W; ++i) {
          const float d = a.v[i] - q.mean, xhat = fmaf(d, q.r, q.shift), dz = V != TAIL || i < l.n ? dz_of(open, xhat, b.v[i], i) : 0.f;
          sz.v[i] += dz;
          sx.v[i] = fmaf(dz, PHASE == SUMS ? d : xhat, sx.v[i]);
        }
      }
#pragma unroll
    for (int i = 0; i < W; ++i) {
      if constexpr (PHASE == SUMS) sx.v[i] = fmaf(sx.v[i], q.r, sz.v[i] * q.shift);   // (of dz (x - mean) until here: 28.7 us for 30.5 at 32 x 56 x 56 x 256)
      dbe.v[i] += sz.v[i];
      dga.v[i] += sx.v[i];
      s[0] = fmaf(sz.v[i], col.ga.v[i], s[0]);
      s[1] = fmaf(sx.v[i], col.ga.v[i], s[1]);
    }
  };
  auto put = [&](Image& q, i64 m0, i64 px, float s0, float s1) {
    Rows<T, PHASE> dx(p.n.dx, l, p.n.P, p.n.ldx, m0), add(p.n.add, l, p.n.P, p.n.ldx, m0);
    dx.from(px);
    add.from(px);
    as_held(q.v);
    as_held(q.d);
    const float r0 = -q.r * s0, r1 = -q.r * s1;
    Vals<W> rg;
#pragma unroll
    for (int i = 0; i < W; ++i) rg.v[i] = q.r * col.ga.v[i];
#pragma unroll
    for (int k = 0; k < KP; ++k) {
      T* o = dx.next();
      const T* e = add.next();
      if (k >= q.rows) continue;
      const auto a = vals(q.v[k]), b = vals(q.d[k]);
      const unsigned open = passed(q, a);
      Vals<W> f;
#pragma unroll
      for (int i = 0; i < W; ++i) {
        const float xhat = fmaf(a.v[i] - q.mean, q.r, q.shift), dz = dz_of(open, xhat, b.v[i], i);
        f.v[i] = fmaf(dz, rg.v[i], fmaf(xhat, r1, r0));
      }
      if (p.n.add) {
        const auto w = vals(load_piece<T, V>(e, l.n));
#pragma unroll
        for (int i = 0; i < W; ++i) f.v[i] += w.v[i];
      }
      store_piece<T, V>(o, l.n, f);
    }
  };
  const i64 stride = (i64)p.slices * teams * IM;
  int turn = 0;
  for (i64 m0 = (i64)at.slice * teams * IM; m0 < p.n.M; m0 += stride, turn ^= 1) {
    float* const buf = cols + turn * IM * entries * 2;
    Image q[IM];
    float s[2 * IM] = {};
#pragma unroll
    for (int i = 0; i < IM; ++i) stats_of(q[i], m0 + i * teams);
    if constexpr (PHASE == WHOLE) {
#pragma unroll
      for (int i = 0; i < IM; ++i) load(q[i], m0 + i * teams, l.r);
#pragma unroll
      for (int i = 0; i < IM; ++i) add_up(q[i], s + 2 * i);
      if (p.n.dx) {
        team_sums<IM>(l, p.t, s, buf);
#pragma unroll
        for (int i = 0; i < IM; ++i) put(q[i], m0 + i * teams, l.r, s[2 * i] / count, s[2 * i + 1] / count);
      }
    } else {
      const i64 m = m0 + l.team;
      if constexpr (PHASE == SUMS) {
        for (i64 px = beg + l.r; px < end; px += (i64)KP * l.RT) {
          load(q[0], m0, px);
          add_up(q[0], s);
        }
        team_sums<IM>(l, p.t, s, buf);
        if (live_at(m0) && l.first) *l.entry(p, m, at.seg * p.sections + l.section) = make_double2(s[0], s[1]);
      } else {
        over_entries(p, l, s, [&](int i) {
          const double2 e = *l.entry(p, m, i);
          s[0] += (float)e.x;
          s[1] += (float)e.y;
        });
        for (i64 px = beg + l.r; px < end; px += (i64)KP * l.RT) {
          load(q[0], m0, px);
          put(q[0], m0, px, s[0] / count, s[1] / count);
        }
      }
    }
  }
  if (PHASE == OUTPUTS || !p.sums) return;
  // lanes of the same channels: those of a wave by shuffles, then the waves
  for (int o = 1 << l.lpr; o < 64; o <<= 1)
#pragma unroll
    for (int i = 0; i < W; ++i) {
      dga.v[i] += __shfl_xor(dga.v[i], o, 64);
      dbe.v[i] += __shfl_xor(dbe.v[i], o, 64);
    }
  const int lane = threadIdx.x & 63, hop = l.lpr > 6 ? 1 << (l.lpr - 6) : 1;   // waves with the same channels are `hop` apart
  if (NT / 64 > hop) {
    __syncthreads();   // (the sums' place)
#pragma unroll
    for (int i = 0; i < W; ++i) {
      cols[(l.wave * 2 * W + i) * 64 + lane] = dga.v[i];
      cols[(l.wave * 2 * W + W + i) * 64 + lane] = dbe.v[i];
    }
    __syncthreads();
    if (l.wave >= hop) return;
    for (int w = l.wave + hop; w < NT / 64; w += hop)
#pragma unroll
      for (int i = 0; i < W; ++i) {
        dga.v[i] += cols[(w * 2 * W + i) * 64 + lane];
        dbe.v[i] += cols[(w * 2 * W + W + i) * 64 + lane];
      }
  }
  if ((int)threadIdx.x < 1 << l.lpr) {
    float* out = p.sums + ((i64)(at.seg * p.slices + at.slice) * p.n.C + l.c) * 2;
#pragma unroll
    for (int i = 0; i < W; ++i)
      if (i < l.n) *reinterpret_cast<float2*>(out + 2 * i) = make_float2(dga.v[i], dbe.v[i]);
  }
}

// dgamma and dbeta: what `rows` workgroups found, [rows][C][2], in a fixed order; 64 threads a channel
__global__ __launch_bounds__(1024) void norm_join_kernel(const float* sums, int rows, int C, float* dgamma, float* dbeta) {
  __shared__ float2 meet[16][16];
  const int at = threadIdx.x & 15, q = threadIdx.x >> 4, c = blockIdx.x * 16 + at;
  float2 v = make_float2(0.f, 0.f);
  if (c < C) {
#pragma unroll 8
    for (int r = q; r < rows; r += 64) {
      const float2 w = *reinterpret_cast<const float2*>(sums + ((i64)r * C + c) * 2);
      v.x += w.x;
      v.y += w.y;
    }
  }
  v = make_float2(across32(across16(v.x)), across32(across16(v.y)));
  if ((threadIdx.x & 63) < 16) meet[threadIdx.x >> 6][at] = v;
  __syncthreads();
  if (q || c >= C) return;
  v = make_float2(0.f, 0.f);
#pragma unroll
  for (int i = 0; i < 16; ++i) {
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

constexpr int CUS = 256, MAX_LANES = 1024;   // of a group's pixel
constexpr int SEGS = 256;   // of an image, at most: the join and every workgroup of the outputs read one number of each

// How a call is run: workgroups of nt, the teams, one launch or two
struct Plan {
  int nt, pieces;
  bool few, single, whole;   // at most two pieces a lane; one; one launch
  NormParams p;
  size_t part, sums, total;
};
// Pieces that a lane's registers hold, of workgroups of 256 and 512
constexpr int most_of(int size, bool bwd, int nt, int v) {
  return v == ONES ? nt == 512 ? 32 : 16 : (nt == 512 ? bwd ? 16 : 32 : bwd ? 4 : 8) * 2 / size;
}
constexpr int FEW = 2, STREAM = 4;   // pieces a lane: of short parts, of a turn of the segments' launches
constexpr int images_at_once(int size, bool bwd) { return (bwd ? 4 : 8) / size; }   // that have one piece a lane

Plan plan_of(const Norm& n, bool bwd) {
  Plan s = {};
  NormParams& p = s.p;
  p.n = n;
  p.cg = n.C / n.groups;
  s.pieces = p.cg % 8 == 0 ? EIGHTS : p.cg < 64 ? ONES : TAIL;
  const int width = s.pieces == ONES ? 1 : 8;
  p.sections = ceil_div(p.cg, MAX_LANES * width);
  p.span = p.sections > 1 ? MAX_LANES * width : p.cg;
  const int size = n.dtype == CONVBN_BF16 ? 2 : 4;
  Team& t = p.t;
  t.m = ceil_div(p.span, width);
  t.mlog = log2_up(t.m);
  const int glog = log2_up(n.groups);
  // groups side by side until a pixel's part is 64 bytes, or until a wave is full of pieces of few channels (32 x 56 x 56 x 256, parts of 32 bytes: forward
  // 48.6 us instead of 24; backward in one launch 53 us, in two with parts of 64 bytes 50).  Single 16-bit channels of rows that begin inside such a part: 128
  // bytes (groups of one channel, forward and backward, 3 x 1884 x 3123 174 us, with 64 bytes 235; 8 x 3136 x 256 89 and 76; 52 x 132 x 472 fp32 50 and 34)
  const int part = s.pieces == ONES && size == 2 && n.ldx % 32 ? 128 : 64;
  while (t.nblog < glog && t.mlog + t.nblog < 6 && (p.cg << t.nblog) * size < part) ++t.nblog;
  auto lanes = [&](int log) { return (n.P + (1LL << (log - t.lprlog)) - 1) >> (log - t.lprlog); };   // pieces of a lane
  auto fits = [&] { return p.sections == 1 && (t.lprlog <= 9 ? lanes(9) <= most_of(size, bwd, 512, s.pieces) : n.P <= FEW); };
  t.lprlog = t.mlog + t.nblog;
  // (few numbers, which the caches hold: one launch counts more than whole parts)
  while (!fits() && t.nblog > 0 && n.M * n.P * n.C <= 1 << 20) {
    --t.nblog;
    --t.lprlog;
  }
  p.bundles = (int)((n.groups + (1LL << t.nblog) - 1) >> t.nblog) * p.sections;
  // one launch where the parts fit and are enough to fill an eighth of the chip, or short
  s.whole = fits() && (n.M * p.bundles >= CUS / 8 || n.P << t.lprlog <= 4096);
  t.ttlog = t.lprlog;
  if (s.whole) {
    while (t.ttlog < 8 && lanes(t.ttlog) > FEW) ++t.ttlog;
    if (t.ttlog == 8 && lanes(8) > most_of(size, bwd, 256, s.pieces)) t.ttlog = 9;
    s.nt = t.ttlog <= 8 ? 256 : 1 << t.ttlog;
    if (t.ttlog > t.lprlog && t.ttlog < 4) t.ttlog = 4;   // (see Lane::wave_sums)
    s.few = lanes(t.ttlog) <= FEW;
    s.single = s.pieces == EIGHTS && s.nt <= 512 && lanes(t.ttlog) == 1 && n.M >= 4 * CUS;
    p.segs = 1;
    // (32-bit offsets of the rows of a workgroup's images)
    const i64 teams = s.nt >> t.ttlog, ld = n.ldx > n.ldy ? n.ldx : n.ldy;
    if ((teams * n.P * ld + n.C) * size > 0x7fffffffLL) s.whole = s.few = s.single = false;
  }
  if (!s.whole) {
    t.ttlog = t.lprlog;
    s.nt = 1024;
    t.ttlog = 10;
    // two workgroups a compute unit, each with a turn of its lanes at least, or with two where there is one for each of them anyway (32 x 56 x 56 x 256 88
    // us; with one turn 98)
    const i64 turn = (i64)STREAM << (10 - t.lprlog);
    i64 segs = n.M ? 2 * CUS / (n.M * p.bundles) : 1;
    const i64 most = n.P / (n.M * p.bundles < CUS ? turn : 2 * turn);
    if (segs > most) segs = most;
    p.segs = (int)(segs < 1 ? 1 : segs < SEGS ? segs : SEGS);
  }
  p.seg = (n.P + p.segs - 1) / p.segs;
  p.segs = (int)((n.P + p.seg - 1) / p.seg);
  const i64 teams = (i64)(s.nt >> t.ttlog) * (s.single ? images_at_once(size, bwd) : 1), each = (n.M + teams - 1) / teams;
  auto bounded = [&](i64 most) { return (int)(each < 1 ? 1 : each < most ? each : most < 1 ? 1 : most); };
  const i64 side = (i64)p.bundles * p.segs;
  auto over = [](int d) { return d > 1 ? (unsigned)(((1ULL << 32) + d - 1) / d) : 0u; };
  p.slices = bounded((s.nt == 256 ? 8 : 2) * CUS / side);
  while (p.bundles > 1 && p.linelog < 3 && (p.span << t.nblog << p.linelog) * size < 128) ++p.linelog;
  p.per_bundle = over(p.bundles);
  p.per_slice = over(p.slices);
  if (bwd) s.sums = align_up((size_t)p.slices * p.segs * n.C * 8, 256);
  if (!s.whole) s.part = align_up((size_t)n.M * n.groups * p.segs * p.sections * 16, 256);
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
int grid_of(const NormParams& p) {
  const int unit = 8 << p.linelog;
  return (p.bundles * p.slices * p.segs + unit - 1) / unit * unit;
}

template <bool BWD, typename T, int F, int NT, int KP, int IM, int PHASE, int V> hipError_t run(const NormParams& p, hipStream_t st) {
  const int turns = p.t.ttlog > 6 ? 2 * IM * (BWD ? 2 * 4 : 4 * (int)(PHASE == WHOLE ? sizeof(Sum<F>) : 8)) * (NT / 64 << p.t.nblog) : 0;
  if constexpr (BWD) {
    constexpr int COLS = NT * 8 * width_of<V>;
    static LdsLimitOnce once;
    auto* k = &norm_bwd_kernel<T, F, NT, KP, IM, PHASE, V>;
    const hipError_t e = set_lds_limit_once(once, (const void*)k, COLS > 16384 ? COLS : 16384);   // (a turn of 16 waves of 64 groups: 16384)
    if (e != hipSuccess) return e;
    const int cols = p.sums && PHASE != OUTPUTS ? COLS : 0;
    k<<<grid_of(p), NT, cols > turns ? cols : turns, st>>>(p);
  } else {
    static LdsLimitOnce once;
    auto* k = &norm_fwd_kernel<T, F, NT, KP, IM, PHASE, V>;
    const hipError_t e = set_lds_limit_once(once, (const void*)k, 2 * IM * 4 * 8 * NT);   // (64 groups a wave)
    if (e != hipSuccess) return e;
    k<<<grid_of(p), NT, turns, st>>>(p);
  }
  return hipGetLastError();
}
template <bool BWD, typename T, int F, int V> hipError_t run_plan(const Plan& s, hipStream_t st) {
  constexpr int SIZE = sizeof(T), KP = BWD ? STREAM / 2 : STREAM;
  if (!s.whole) {
    const hipError_t e = run<BWD, T, BWD ? F : (int)CONVBN_NORM_NONE, 1024, KP, 1, SUMS, V>(s.p, st);
    return e != hipSuccess || (BWD && !s.p.n.dx) ? e : run<BWD, T, F, 1024, KP, 1, OUTPUTS, V>(s.p, st);
  }
  if (s.nt == 1024) return run<BWD, T, F, 1024, FEW, 1, WHOLE, V>(s.p, st);
  if constexpr (V == EIGHTS) {   // (others are rare: they do with the larger kernels)
    constexpr int IM = images_at_once(SIZE, BWD);
    if (s.single) return s.nt == 256 ? run<BWD, T, F, 256, 1, IM, WHOLE, V>(s.p, st) : run<BWD, T, F, 512, 1, IM, WHOLE, V>(s.p, st);
    if (s.few) return s.nt == 256 ? run<BWD, T, F, 256, FEW, 1, WHOLE, V>(s.p, st) : run<BWD, T, F, 512, FEW, 1, WHOLE, V>(s.p, st);
  }
  return s.nt == 256 ? run<BWD, T, F, 256, most_of(SIZE, BWD, 256, V), 1, WHOLE, V>(s.p, st)
                     : run<BWD, T, F, 512, most_of(SIZE, BWD, 512, V), 1, WHOLE, V>(s.p, st);
}
template <bool BWD> hipError_t run_norm(const Plan& s, hipStream_t st) {
  return by_type(s.p.n, [&](auto t, auto f) {
    using T = decltype(t);
    return s.pieces == EIGHTS ? run_plan<BWD, T, f.value, EIGHTS>(s, st) : s.pieces == TAIL ? run_plan<BWD, T, f.value, TAIL>(s, st)
                                                                                            : run_plan<BWD, T, f.value, ONES>(s, st);
  });
}

}  // namespace
}  // namespace convbn
