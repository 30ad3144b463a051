// Rotation of rows by their positions.
#pragma once

#include "lvspec_dev.h"
#include "lvspec_kernels.h"

namespace lvspec {

namespace {

// Cosine and sine in 64 bits: the angle less a multiple of pi/2, taken off in two parts of pi/2 with one rounding
// each, and Taylor's series on what is left, |x| <= pi/4, whose next terms are 2e-14 (9e-14 at angles of 2^48).  In 64
// bits because the angles of far positions need them (position 10^6 in 32 bits is 0.06 off), and because rows that go into
// a cache of few bits stand on the borders between two codes: one in 60 bf16 numbers does, and a last bit that depends on
// how the sine was taken would choose the code.  That costs nothing where memory bounds a call (16384 rows of keys into a
// cache 27.0 us, 25.6 with angles as they are in place of their sines) and one to two microseconds where latency does
// (16 x 5 rows 7.0 and 5.6, 2048 rows 17.4 and 15.6).
LVS_DEV void cos_sin(double a, double& c, double& s) {
  const double n = __builtin_rint(a * 0.63661977236758134308);                     // 2 / pi
  double x = __builtin_fma(-n, 1.57079632679489661923, a);                         // pi / 2, rounded
  x = __builtin_fma(-n, 6.12323399573676603587e-17, x);                            // and the rest of it
  const int quarter = (int)(n - 4.0 * __builtin_floor(n * 0.25));
  const double z = x * x;
  double p = 1.0 / 6227020800.0;
  p = __builtin_fma(p, z, -1.0 / 39916800.0);
  p = __builtin_fma(p, z, 1.0 / 362880.0);
  p = __builtin_fma(p, z, -1.0 / 5040.0);
  p = __builtin_fma(p, z, 1.0 / 120.0);
  p = __builtin_fma(p, z, -1.0 / 6.0);
  p = __builtin_fma(p * z, x, x);
  double q = -1.0 / 87178291200.0;
  q = __builtin_fma(q, z, 1.0 / 479001600.0);
  q = __builtin_fma(q, z, -1.0 / 3628800.0);
  q = __builtin_fma(q, z, 1.0 / 40320.0);
  q = __builtin_fma(q, z, -1.0 / 720.0);
  q = __builtin_fma(q, z, 1.0 / 24.0);
  q = __builtin_fma(q, z, -0.5);
  q = __builtin_fma(q, z, 1.0);
  c = quarter & 1 ? p : q;
  s = quarter & 1 ? q : p;
  if (quarter == 1 || quarter == 2) c = -c;
  if (quarter >= 2) s = -s;
}

// Cosines and sines of a piece's W frequencies (Piece), for packed row t.
template <int W>
struct Turn {
  double c[W], s[W];
  LVS_DEV void at(const RotaryKernelArgs& r, int64_t t, int f0) {
    const int first = r.axis != nullptr ? 0 : r.pos[t];
    const int jump = W > 1 && r.interleaved != 0 ? (r.half - W) / 2 : 0;
#pragma unroll
    for (int j = 0; j < W; ++j) {
      const int f = f0 + j + (j >= W / 2 ? jump : 0);
      const int pos = r.axis != nullptr ? r.pos[(int64_t)min((int)r.axis[f], r.n_axes - 1) * r.pos_sa + t] : first;
      cos_sin((double)pos * (double)r.inv_freq[f], c[j], s[j]);      // (the product is exact up to 2^29)
      c[j] *= r.factor;
      s[j] *= r.sine;
    }
  }
  // Pair j: a[j] and b[j], or (`pairs`) neighbours of the 2 W channels a, b.  The sums are in 64 bits, rounded to
  // binary32 and then to the rows' type, in every channel and every call alike, since a key's codes go by it.  (Left to
  // itself the compiler takes the two roundings as one where both stand in one basic block, one channel in 8 of rows and
  // one in 16 of appends, and about one number in 2^17 is another there.  Rounded once, that one would be nearer by up to
  // 2^-17 of a step of bf16; but no instruction rounds 64 bits to bf16, and every number would take several.)
  LVS_DEV void apply(float (&a)[W], float (&b)[W], bool pairs) const {
    auto one = [&](float& x, float& y, int j) {
#pragma clang fp contract(off)
      const double u = x, v = y;
      x = (float)__builtin_fma(u, c[j], -(v * s[j]));
      y = (float)__builtin_fma(v, c[j], u * s[j]);
    };
    if (!pairs || W == 1) {
#pragma unroll
      for (int j = 0; j < W; ++j) one(a[j], b[j], j);
    } else if constexpr (W > 1) {
#pragma unroll
      for (int j = 0; j < W / 2; ++j) {
        one(a[2 * j], a[2 * j + 1], j);
        one(b[2 * j], b[2 * j + 1], W / 2 + j);
      }
    }
  }
};

// W values of a type in memory as floats, and back (to nearest even).
template <class T, int W>
struct Packed {
  typedef T vec __attribute__((ext_vector_type(W)));
  vec x;
  LVS_DEV void load(const T* p) { x = *reinterpret_cast<const vec*>(p); }
  LVS_DEV void store(T* p) const { *reinterpret_cast<vec*>(p) = x; }
  LVS_DEV void get(float (&f)[W]) const {
#pragma unroll
    for (int i = 0; i < W; ++i) f[i] = (float)x[i];
  }
  LVS_DEV void put(const float (&f)[W]) {
#pragma unroll
    for (int i = 0; i < W; ++i) x[i] = (T)f[i];
  }
};
template <class T>
struct Packed<T, 1> {
  T x;
  LVS_DEV void load(const T* p) { x = *p; }
  LVS_DEV void store(T* p) const { *p = x; }
  LVS_DEV void get(float (&f)[1]) const { f[0] = (float)x; }
  LVS_DEV void put(const float (&f)[1]) { x = (T)f[0]; }
};

// What a thread has of a head's channels: W at a and W at b, far enough apart that the threads of a row read in one
// piece.  Turned are pieces p < half / W: channels p W and half + p W, which are pairs, or whose neighbours are (W = 1: the
// two neighbours).  Pieces behind them stay as they are (the last one W channels, where their number is odd).
struct Piece {
  int a, b;                // channels; b < 0: none
  int f;                   // first frequency (of the second W / 2 neighbours half / 2 further on)
  bool turned;
};
LVS_DEV Piece piece_of(int p, int W, int half, int D, bool pairs) {
  if (W == 1 && pairs && p < half) return Piece{2 * p, 2 * p + 1, p, true};
  if (p * W < half) return Piece{p * W, half + p * W, pairs ? p * W / 2 : p * W, true};
  const int rest = (D - 2 * half) / W, at = p - half / W, b = at + (rest + 1) / 2;
  return Piece{2 * half + at * W, b < rest ? 2 * half + b * W : -1, 0, false};
}
inline int pieces(int W, int half, int D) { return half / W + ((D - 2 * half) / W + 1) / 2; }

// A thread's piece of row t in the heads first .. last-1 of a tensor: loads of kAhead heads at a time, the first of them
// ahead of the angles, where those are not `ready`.  Two, four and eight heads: 16384 rows of 40 + 8 heads in bf16 85.3, 83.7
// and 83.4 us, 1500 rows 9.7, 10.2 and 11.0, 5001 rows of 32 heads in fp32 31.1, 29.6 and 27.5.
constexpr int kAhead = 4;
template <class T, int W>
LVS_DEV void rotate_heads(const RotaryRows& x, const RotaryKernelArgs& r, Turn<W>& turn, bool& ready, const Piece& e,
                          int64_t t, int first, int last) {
  const bool pairs = r.interleaved != 0;
  const T* from = static_cast<const T*>(x.x) + t * x.x_sr;
  T* to = static_cast<T*>(x.y) + t * x.y_sr;
  for (int h0 = first; h0 < last; h0 += kAhead) {
    Packed<T, W> u[kAhead], v[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (h0 + i < last) {
        u[i].load(from + (h0 + i) * x.x_sh + e.a);
        if (e.b >= 0) v[i].load(from + (h0 + i) * x.x_sh + e.b);
      }
    if (e.turned && !ready) turn.at(r, t, e.f);
    ready = true;
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (h0 + i < last) {
        if (e.turned) {
          float a[W], b[W];
          u[i].get(a);
          v[i].get(b);
          turn.apply(a, b, pairs);
          u[i].put(a);
          v[i].put(b);
        }
        u[i].store(to + (h0 + i) * x.y_sh + e.a);
        if (e.b >= 0) v[i].store(to + (h0 + i) * x.y_sh + e.b);
      }
  }
}

}  // namespace

}  // namespace lvspec
