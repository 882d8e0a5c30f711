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

// Element i of a row, rotated with the turns cs[pair] of its position.
template <typename T>
__device__ __forceinline__ float rotated_elem(const T* row, int i, int rot, int layout, const double2* cs) {
  if (i >= rot) return elem(row, i);
  double xr, yr;
  if (layout == RESKV_ROPE_HALF) {
    const int p = i < rot / 2 ? i : i - rot / 2;
    rotate_pair(elem(row, p), elem(row, p + rot / 2), cs[p], xr, yr);
    return round_to(i < rot / 2 ? xr : yr, row);
  }
  const int p = i >> 1;
  rotate_pair(elem(row, 2 * p), elem(row, 2 * p + 1), cs[p], xr, yr);
  return round_to(i & 1 ? yr : xr, row);
}

}  // namespace reskv
