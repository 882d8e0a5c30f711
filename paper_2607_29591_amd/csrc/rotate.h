// Rotation of row pairs by their positions, shared by the kernels that rotate:
// one order of operations, so that every call writes the same bits.
#pragma once

#include "common.h"

#include "../../include/reskv.h"

namespace reskv {

// A cos a, A sin a of a = pos * f. The angle reaches 1e5 radians and more at far
// positions, where 32 bits hold it to 0.01: it is formed in 64 bits and reduced
// by whole turns with 2 pi in two parts, so that the remainder keeps the 2^-53
// of the product.
__device__ __forceinline__ double2 turn(double f, int pos, double scale) {
  constexpr double kTwoPi = 6.283185307179586, kTwoPiLo = 2.4492935982947064e-16, kPerTurn = 0.15915494309189535;
  const double a = (double)pos * f;
  const double n = rint(a * kPerTurn);
  double s, c;
  sincos(fma(-n, kTwoPiLo, fma(-n, kTwoPi, a)), &s, &c);
  return make_double2(scale * c, scale * s);
}

// (x, y) turned by cs = (A cos a, A sin a).
__device__ __forceinline__ void rotate_pair(float x, float y, double2 cs, double& xr, double& yr) {
  xr = fma((double)x, cs.x, -((double)y * cs.y));
  yr = fma((double)x, cs.y, (double)y * cs.x);
}

// A 64-bit result rounded once to the row's type. For bf16 through 32 bits
// truncated with the last bit set where something was cut off: a plain rounding
// to 32 bits could land on the middle between two bf16 numbers and lose the side.
__device__ __forceinline__ float round_to(double v, const float*) { return (float)v; }
__device__ __forceinline__ uint32_t bf16_bits(double v) {
  const float f = __double2float_rz(v);
  const uint32_t odd = __float_as_uint(f) | ((double)f != v ? 1u : 0u);
  return (uint32_t)f32_to_bf16_rne(__uint_as_float(odd));
}
__device__ __forceinline__ float round_to(double v, const uint16_t*) {
  return __uint_as_float(bf16_bits(v) << 16);
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
    const bool first = at.first(i);
    double xr, yr;
    rotate_pair(first ? x : y, first ? y : x, cs[at.pair(i)], xr, yr);
    return round_to(first ? xr : yr, &own);
  }
};

}  // namespace reskv
