// The 4-bit cache format (include/reskv.h): where a slot's codes and scales
// are, and a group's scale and codes.
#pragma once

#include "common.h"

namespace reskv {

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;

// Lengths of a (b, kv head) cache clamped to its capacities, so that corrupt
// lengths cannot make a kernel touch anything outside it.
__device__ __forceinline__ void clamp_lengths(int r_raw, int n_raw, int C, int Rcap, int& r, int& n) {
  r = clampi(r_raw, 0, min(Rcap, C));
  n = clampi(n_raw, 0, C - r);
}
__device__ __forceinline__ void cache_lengths(const int32_t* res_len, const int32_t* main_len, int bh, int C, int Rcap,
                                              int& r, int& n) {
  clamp_lengths(res_len[bh], main_len[bh], C, Rcap, r, n);
}

// 16-byte store; kStream: past the caches, for results that are larger than them.
template <bool kStream>
__device__ __forceinline__ void store16(void* p, u32x4_t v) {
  if constexpr (kStream) __builtin_nontemporal_store(v, static_cast<u32x4_t*>(p));
  else *static_cast<u32x4_t*>(p) = v;
}

// Offsets in a block of 64 slots.
template <int D>
struct QuantBlock {
  static constexpr int kSlots = 64;
  static constexpr int kGroups = D / 32;  // scales of a row
  static constexpr int kPiece = D / 16;   // value elements of one matrix lane
  static constexpr int kV = 32 * D, kKS = 64 * D, kVS = 66 * D, kBytes = 68 * D;
  static __device__ __forceinline__ int k_code(int s) { return s * (D / 2); }
  static __device__ __forceinline__ int v_code(int s, int piece) {
    return kV + ((s >> 2) * 16 + piece) * 2 * kPiece + (s & 3) * (kPiece / 2);
  }
  static __device__ __forceinline__ int k_scale(int s, int c) { return kKS + ((s & 15) * kGroups + c) * 4 + (s >> 4); }
  static __device__ __forceinline__ int v_scale(int s, int c) {
    return kVS + ((((s >> 2) & 3) * kGroups + c) * 4 + (s >> 4)) * 4 + (s & 3);
  }
};

// Scale byte of a group whose largest magnitude has these bits: with the
// largest in [2^E, 2^(E+1)), the scale 2^(E-2) maps it to [4, 8), and to at most
// 7 unless it is above 1.75 * 2^E, where the next scale is taken. Inside
// [2, 252] every value that a code stands for is a normal bf16 number.
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax_bits) {
  const int e = (int)(amax_bits >> 23);
  if (e == 255) return 255;
  return (uint32_t)clampi(e - 2 + ((amax_bits & 0x7fffffu) > 0x600000u ? 1 : 0), 2, 252);
}
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// Codes of two numbers in the low byte: the conversion divides by the scale,
// rounds to nearest even and clips.
__device__ __forceinline__ uint32_t code_pair(float a, float b, float scale) {
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, a, b, scale, 0) & 0xffu;
}
// Values of the code pair in byte kByte, times the scale, as two bf16 (exact).
template <int kByte>
__device__ __forceinline__ uint32_t value_pair(uint32_t codes, float scale) {
  const bf16x2_t v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, kByte);
  return __builtin_bit_cast(uint32_t, v);
}

// Largest of the 16 lanes of a DPP row, as unsigned numbers (magnitude bits
// order like magnitudes, infinities and NaN above all of them).
template <int Ctrl>
__device__ __forceinline__ uint32_t dpp_umax(uint32_t v) {
  const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, Ctrl, 0xF, 0xF, false);
  return v > o ? v : o;
}
__device__ __forceinline__ uint32_t row16_umax(uint32_t v) {
  v = dpp_umax<0xB1>(v);    // quad_perm [1,0,3,2]
  v = dpp_umax<0x4E>(v);    // quad_perm [2,3,0,1]
  v = dpp_umax<0x141>(v);   // row_half_mirror
  return dpp_umax<0x140>(v);  // row_mirror
}

// One row into a block, by a wave: lane l < D / 2 holds elements 2l and 2l + 1
// (16 lanes a group of 32). Every lane of the wave must be active.
template <int D>
__device__ __forceinline__ void store_row_quant(uint8_t* block, int slot, bool value, float a, float b, int lane) {
  using Q = QuantBlock<D>;
  const uint32_t ma = __float_as_uint(a) & 0x7fffffffu, mb = __float_as_uint(b) & 0x7fffffffu;
  const uint32_t byte = scale_byte(row16_umax(ma > mb ? ma : mb));
  const uint8_t code = (uint8_t)code_pair(a, b, scale_of(byte));
  if (lane >= D / 2) return;
  const int i = 2 * lane;
  if (value) block[Q::v_code(slot, i / Q::kPiece) + (i % Q::kPiece) / 2] = code;
  else block[Q::k_code(slot) + lane] = code;
  if (lane % 16 == 0) block[value ? Q::v_scale(slot, lane / 16) : Q::k_scale(slot, lane / 16)] = (uint8_t)byte;
}

}  // namespace reskv
