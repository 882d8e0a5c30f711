// Rotary positions: rotate rows of queries and keys, from any order of rows
// into any other.
#include <math.h>

#include "internal.h"
#include "rotate.h"

namespace reskv {

namespace {

constexpr int kThreads = 256;

struct RopeArgs {
  reskv_rope_t rope;
  const int32_t* positions;
  const int32_t* n_tok;
  const void* src[2];  // queries, keys
  void* dst[2];
  reskv_rows_t from[2], to[2];
  long long tokens;    // B * n
  int n, heads[2];     // 0 heads: absent
};

// 8 elements of a row as fp32 and back, rounded from 64 bits.
__device__ __forceinline__ void store8(uint16_t* p, const double (&v)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = bf16_bits(v[2 * i]) | (bf16_bits(v[2 * i + 1]) << 16);
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store8(float* p, const double (&v)[8]) {
  *reinterpret_cast<float4*>(p) = make_float4((float)v[0], (float)v[1], (float)v[2], (float)v[3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4((float)v[4], (float)v[5], (float)v[6], (float)v[7]);
}
__device__ __forceinline__ void copy8(const uint16_t* from, uint16_t* to) {
  *reinterpret_cast<uint4*>(to) = *reinterpret_cast<const uint4*>(from);
}
__device__ __forceinline__ void copy8(const float* from, float* to) {
  const float4 a = reinterpret_cast<const float4*>(from)[0], b = reinterpret_cast<const float4*>(from)[1];
  reinterpret_cast<float4*>(to)[0] = a;
  reinterpret_cast<float4*>(to)[1] = b;
}

// A lane holds 16 elements of a row: 8 pairs (two runs of 8 in the half layout,
// one run of 16 in the interleaved one), or 16 elements past rot_dim. The
// D / 16 lanes of a row and the rows of neighbouring tokens adjoin.
template <typename T, int D, bool kHalf>
__global__ __launch_bounds__(kThreads) void rope_kernel(RopeArgs a) {
  constexpr int kL = D / 16;
  const long long i = blockIdx.x * (long long)kThreads + threadIdx.x;
  const long long token = i / kL;
  if (token >= a.tokens) return;
  const int j = (int)(i % kL), b = (int)(token / a.n), t = (int)(token % a.n);
  if (a.n_tok && t >= a.n_tok[b]) return;
  const int head = blockIdx.y, kind = head >= a.heads[0], h = kind ? head - a.heads[0] : head;
  const T* src = static_cast<const T*>(a.src[kind]) + b * a.from[kind].batch + h * a.from[kind].head + t * a.from[kind].row;
  T* dst = static_cast<T*>(a.dst[kind]) + b * a.to[kind].batch + h * a.to[kind].head + t * a.to[kind].row;
  const int rot = a.rope.rot_dim;
  if (16 * j >= rot) {  // past the rotated part
    if (src != dst) {
      copy8(src + 16 * j, dst + 16 * j);
      copy8(src + 16 * j + 8, dst + 16 * j + 8);
    }
    return;
  }
  const int e0 = kHalf ? 8 * j : 16 * j, e1 = kHalf ? rot / 2 + 8 * j : 16 * j + 8;
  const int pos = a.positions[token];
  float x[8], y[8];
  load8_f32(src + e0, x);
  load8_f32(src + e1, y);
  double u[8], v[8];
#pragma unroll
  for (int p = 0; p < 8; ++p) {
    const double2 cs = turn(a.rope.freq[8 * j + p], pos, a.rope.attn_scale);
    if constexpr (kHalf) {
      rotate_pair(x[p], y[p], cs, u[p], v[p]);
    } else if (p < 4) {
      rotate_pair(x[2 * p], x[2 * p + 1], cs, u[2 * p], u[2 * p + 1]);
    } else {
      rotate_pair(y[2 * p - 8], y[2 * p - 7], cs, v[2 * p - 8], v[2 * p - 7]);
    }
  }
  store8(dst + e0, u);
  store8(dst + e1, v);
}

template <typename T, int D>
void launch(const RopeArgs& ra, hipStream_t stream) {
  const dim3 grid((unsigned)((ra.tokens * (D / 16) + kThreads - 1) / kThreads), ra.heads[0] + ra.heads[1]);
  if (ra.rope.layout == RESKV_ROPE_HALF)
    hipLaunchKernelGGL((rope_kernel<T, D, true>), grid, dim3(kThreads), 0, stream, ra);
  else
    hipLaunchKernelGGL((rope_kernel<T, D, false>), grid, dim3(kThreads), 0, stream, ra);
}

}  // namespace

void make_rope(const reskv_rope_params_t& p, reskv_rope_t* rope, double* freq) {
  const double kTwoPi = 6.283185307179586;
  const int rot = p.rot_dim;
  rope->rot_dim = rot;
  rope->layout = p.layout;
  rope->freq = nullptr;
  rope->attn_scale = p.attn_scale;
  if (p.attn_scale == 0.0) rope->attn_scale = p.scaling == RESKV_ROPE_YARN ? 0.1 * log(p.factor) + 1.0 : 1.0;
  const double base = p.scaling == RESKV_ROPE_NTK ? p.theta * pow(p.factor, rot / (rot - 2.0)) : p.theta;
  double lo = 0.0, hi = 0.0;
  if (p.scaling == RESKV_ROPE_YARN) {
    auto dim = [&](double n) { return rot * log(p.original_len / (kTwoPi * n)) / (2.0 * log(p.theta)); };
    lo = fmax(floor(dim(p.beta_fast)), 0.0);
    hi = fmin(ceil(dim(p.beta_slow)), rot - 1.0);
  }
  for (int i = 0; i < rot / 2; ++i) {
    double f = pow(base, -2.0 * i / rot);
    if (p.scaling == RESKV_ROPE_LINEAR) f /= p.factor;
    if (p.scaling == RESKV_ROPE_LLAMA3) {
      const double turns = p.original_len * f / kTwoPi;
      const double t = (turns - p.low_freq_factor) / (p.high_freq_factor - p.low_freq_factor);
      if (t < 0.0) f /= p.factor;
      else if (t <= 1.0) f *= (1.0 - t) / p.factor + t;
    }
    if (p.scaling == RESKV_ROPE_YARN) {
      const double t = fmin(fmax((i - lo) / fmax(hi - lo, 0.001), 0.0), 1.0);
      f = f / p.factor * t + f * (1.0 - t);
    }
    freq[i] = f;
  }
}

hipError_t launch_rope(const reskv_shape_t& s, const reskv_rope_t& rope, int n_rows, const int32_t* positions,
                       const int32_t* n_tok, const void* q, const reskv_rows_t* q_at, void* q_out,
                       const reskv_rows_t* q_out_at, const void* k, const reskv_rows_t* k_at, void* k_out,
                       const reskv_rows_t* k_out_at, hipStream_t stream) {
  RopeArgs ra{};
  ra.rope = rope;
  ra.positions = positions;
  ra.n_tok = n_tok;
  ra.n = n_rows;
  ra.tokens = (long long)s.batch * n_rows;
  if (q) {
    ra.heads[0] = s.num_q_heads;
    ra.src[0] = q; ra.from[0] = *q_at; ra.dst[0] = q_out; ra.to[0] = *q_out_at;
  }
  if (k) {
    ra.heads[1] = s.num_kv_heads;
    ra.src[1] = k; ra.from[1] = *k_at; ra.dst[1] = k_out; ra.to[1] = *k_out_at;
  }
  const bool bf = s.dtype == RESKV_BF16;
  if (s.head_dim == 128) bf ? launch<uint16_t, 128>(ra, stream) : launch<float, 128>(ra, stream);
  else bf ? launch<uint16_t, 64>(ra, stream) : launch<float, 64>(ra, stream);
  return hipGetLastError();
}

}  // namespace reskv
