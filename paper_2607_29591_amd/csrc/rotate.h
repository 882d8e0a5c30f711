// Rotation of row pairs by their positions, shared by the kernels that rotate:
// one order of operations, so that every call writes the same bits.
#pragma once

#include "common.h"

#include "../../include/reskv.h"

namespace reskv {

// A cos a, A sin a of a = pos * f. The angle reaches 1e5 radians and more at far
// positions, where 32 bits hold it to 0.01: it is formed in 64 bits and reduced by
// quarter turns with pi / 2 in two parts, so that the remainder keeps the 2^-53 of
// the product. On [-pi/4, pi/4] the Taylor sums to r^17 and r^16 are within 2^-58
// (r^19 / 19! < 9e-20, r^18 / 18! < 3e-18). About 30 instructions, a fifth of the
// library's sine and cosine, which reduce any argument once more.
__device__ __forceinline__ double2 turn(double f, int pos, double scale) {
  constexpr double kQuarter = 1.5707963267948966, kQuarterLo = 6.123233995736766e-17, kPerTurn = 0.6366197723675814;
  const double a = (double)pos * f;
  const double n = rint(a * kPerTurn);
  const double r = fma(-n, kQuarterLo, fma(-n, kQuarter, a)), z = r * r;
  double s = 1.0 / 355687428096000.0, c = 1.0 / 20922789888000.0;
  s = fma(s, z, -1.0 / 1307674368000.0);
  c = fma(c, z, -1.0 / 87178291200.0);
  s = fma(s, z, 1.0 / 6227020800.0);
  c = fma(c, z, 1.0 / 479001600.0);
  s = fma(s, z, -1.0 / 39916800.0);
  c = fma(c, z, -1.0 / 3628800.0);
  s = fma(s, z, 1.0 / 362880.0);
  c = fma(c, z, 1.0 / 40320.0);
  s = fma(s, z, -1.0 / 5040.0);
  c = fma(c, z, -1.0 / 720.0);
  s = fma(s, z, 1.0 / 120.0);
  c = fma(c, z, 1.0 / 24.0);
  s = fma(s, z, -1.0 / 6.0);
  c = fma(c, z, -0.5);
  s = fma(s * z, r, r);
  c = fma(c, z, 1.0);
  const int q = (int)(n - 4.0 * floor(n * 0.25));  // quarter turns, 0..3
  const double cq = q & 1 ? s : c, sq = q & 1 ? c : s;
  return make_double2(scale * (q == 1 || q == 2 ? -cq : cq), scale * (q >= 2 ? -sq : sq));
}

// One element of a pair turned by cs = (A cos a, A sin a): x takes -y's part, y
// takes x's.
__device__ __forceinline__ double rotate_one(float own, float other, double2 cs, bool first) {
  const double part = (double)other * cs.y;
  return fma((double)own, cs.x, first ? -part : part);
}
__device__ __forceinline__ void rotate_pair(float x, float y, double2 cs, double& xr, double& yr) {
  xr = rotate_one(x, y, cs, true);
  yr = rotate_one(y, x, cs, false);
}

// 64-bit results rounded once to the row's type. For bf16 by way of 32 bits, which
// rounds twice only where the 32-bit number is the middle between two bf16 ones
// (one in 2^16): there the last bit tells the side the result was on.
__device__ __forceinline__ bool is_middle(float f) { return (__float_as_uint(f) & 0xffffu) == 0x8000u; }
__device__ __forceinline__ float off_middle(float f, double v) {
  const double back = (double)f;
  if (back == v) return f;
  return __uint_as_float(__float_as_uint(f) + (fabs(back) < fabs(v) ? 1u : ~0u));  // one step towards v
}
__device__ __forceinline__ float round_to(double v, const float*) { return (float)v; }
__device__ __forceinline__ float round_to(double v, const uint16_t*) {
  float f = (float)v;
  if (is_middle(f)) f = off_middle(f, v);
  return __uint_as_float((uint32_t)f32_to_bf16_rne(f) << 16);
}

__device__ __forceinline__ float elem(const uint16_t* row, int i) { return __uint_as_float((uint32_t)row[i] << 16); }
__device__ __forceinline__ float elem(const float* row, int i) { return row[i]; }

// Where element i of a row has the other one of its pair: index arithmetic that
// holds for both layouts, without branches.
struct PairIndex {
  int rot, half, odd, lim;  // half: rot / 2 in the half layout, else 0; odd: 1 in the interleaved one
  __device__ __forceinline__ PairIndex(int rot_dim, int layout) {
    const bool h = layout == RESKV_ROPE_HALF;
    rot = rot_dim;
    half = h ? rot_dim / 2 : 0;
    odd = h ? 0 : 1;
    lim = h ? rot_dim / 2 : rot_dim;
  }
  __device__ __forceinline__ bool turned(int i) const { return i < rot; }
  __device__ __forceinline__ bool first(int i) const { return !(i & odd) && i < lim; }  // the pair's x
  __device__ __forceinline__ int pair(int i) const { return (i >> odd) - (i < lim ? 0 : half); }
  // (some element of the row for i >= rot)
  __device__ __forceinline__ int other(int i) const { return (i ^ odd) + (i < lim ? half : -half); }
};
// Element i of a row as stored, with its pair's other element; rotated once the
// turns cs[pair] of the row's position are known, and rounded to T.
template <typename T>
struct PairElem {
  T own, other;
  __device__ __forceinline__ void load(const T* row, int i, const PairIndex& at) {
    own = row[i];
    other = row[at.other(i)];
  }
  __device__ __forceinline__ float rotated(int i, const PairIndex& at, const double2* cs) const {
    const float x = elem(&own, 0), y = elem(&other, 0);
    if (!at.turned(i)) return x;
    return round_to(rotate_one(x, y, cs[at.pair(i)], at.first(i)), &own);
  }
};

}  // namespace reskv
