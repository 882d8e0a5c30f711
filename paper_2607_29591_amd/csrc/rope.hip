// Rotary positions: rotate rows of queries and keys, from any order of rows
// into any other.
#include <math.h>

#include "internal.h"
#include "rotate.h"

namespace reskv {

namespace {

constexpr int kThreads = 256;
// Waves that the heads are dealt to where tokens are few (32768 tokens 144, 144, 144,
// 143 us at 1024, 2048, 4096, 8192; 8144 fp32 tokens of 28 + 4 heads of 64: 21.1,
// 20.1, 19.7, 19.5): more of them hide more latency, each pays its sines once more.
constexpr int kWaves = 8192;

struct RopeArgs {
  reskv_rope_t rope;
  const int32_t* positions;
  const int32_t* n_tok;
  const void* src[2];  // queries, keys
  void* dst[2];
  reskv_rows_t from[2], to[2];
  int tokens, n;       // B * n
  int heads[2];        // 0: absent
  int log_tw, hp;      // log2 of a wave's tokens; heads of a wave
};

// Two 16-byte pieces of a row: kE elements each.
template <typename T>
struct Chunk {
  static constexpr int kE = 16 / (int)sizeof(T);
  uint4 w[2];
  __device__ __forceinline__ void load(const T* row, int e0, int e1) {
    w[0] = *reinterpret_cast<const uint4*>(row + e0);
    w[1] = *reinterpret_cast<const uint4*>(row + e1);
  }
  __device__ __forceinline__ void store(T* row, int e0, int e1) const {
    *reinterpret_cast<uint4*>(row + e0) = w[0];
    *reinterpret_cast<uint4*>(row + e1) = w[1];
  }
};
__device__ __forceinline__ void unpack(uint4 w, float (&x)[8]) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = bf16_lo(u[i]);
    x[2 * i + 1] = bf16_hi(u[i]);
  }
}
__device__ __forceinline__ void unpack(uint4 w, float (&x)[4]) {
  x[0] = __uint_as_float(w.x); x[1] = __uint_as_float(w.y); x[2] = __uint_as_float(w.z); x[3] = __uint_as_float(w.w);
}
__device__ __forceinline__ uint4 pack(const double (&v)[8]) {  // round_to, eight at once
  typedef __attribute__((ext_vector_type(2))) float f32x2_t;
  typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
  float f[8];
  bool middle = false;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    f[i] = (float)v[i];
    middle |= is_middle(f[i]);
  }
  if (middle) {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = is_middle(f[i]) ? off_middle(f[i], v[i]) : f[i];
  }
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2_t{f[2 * i], f[2 * i + 1]}, bf16x2_t));
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ uint4 pack(const double (&v)[4]) {
  return make_uint4(__float_as_uint((float)v[0]), __float_as_uint((float)v[1]), __float_as_uint((float)v[2]),
                    __float_as_uint((float)v[3]));
}

// A lane holds two pieces of a row, half of the rotated part apart (so that the
// lanes of a row read adjoining pieces in both layouts): the x and the y of kE
// pairs in the half layout, kE / 2 whole pairs each in the interleaved one; the
// lanes past rot_dim two pieces of the rest. Its position and so its kE turns stay
// the same over the heads it goes through: sines and cosines in 64 bits are paid
// once for all heads of a wave. The rows of a wave are 2^log_tw neighbouring tokens
// of one head and, where tokens are few, several heads. Bound by memory: a batch of
// heads is requested while the one before is turned. 32768 tokens of 32 + 8 heads
// of 128 (671 MB): 353 us with a thread's own sines for every row, 148 us with a
// wave's over its heads, 137-140 us with the Taylor sums (4.9 TB/s; a copy of that
// size reaches 5.0); one token: 7.0, 4.7 and 3.5 us.
template <typename T, int D, bool kHalf>
__global__ __launch_bounds__(kThreads, sizeof(T) == 4 && !kHalf ? 4 : 2) void rope_kernel(RopeArgs a) {
  constexpr int kE = Chunk<T>::kE, kL = D / (2 * kE), kRows = 64 / kL;
  constexpr int kB = 4;  // heads requested together
  const int lane = threadIdx.x & 63, row = lane / kL, j = lane % kL;
  const int token = ((blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6)) << a.log_tw) + (row & ((1 << a.log_tw) - 1));
  if (token >= a.tokens) return;
  const int b = token / a.n, t = token % a.n;
  if (a.n_tok && t >= a.n_tok[b]) return;
  const int step = kRows >> a.log_tw, heads = a.heads[0] + a.heads[1];
  const int end = min((int)(blockIdx.y + 1) * a.hp, heads);
  int head = blockIdx.y * a.hp + (row >> a.log_tw);
  if (head >= end) return;
  const int rot = a.rope.rot_dim, lanes = rot / (2 * kE);  // lanes of the rotated part
  const bool turned = j < lanes;
  const int e0 = turned ? kE * j : rot + kE * (j - lanes), e1 = e0 + (turned ? rot : D - rot) / 2;
  const T* src[2];
  T* dst[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    src[k] = static_cast<const T*>(a.src[k]) + b * a.from[k].batch + t * a.from[k].row;
    dst[k] = static_cast<T*>(a.dst[k]) + b * a.to[k].batch + t * a.to[k].row;
  }
  auto request = [&](Chunk<T> (&c)[kB], int h0) {
#pragma unroll
    for (int k = 0; k < kB; ++k) {
      const int h = min(h0 + k * step, end - 1), kind = h >= a.heads[0];
      c[k].load(src[kind] + (kind ? h - a.heads[0] : h) * a.from[kind].head, e0, e1);
    }
  };
  Chunk<T> now[kB], next[kB];
  request(now, head);
  double2 cs[kE];
  if (turned) {
    const int pos = a.positions[token];
#pragma unroll
    for (int p = 0; p < kE; ++p) {
      const int pair = kHalf ? e0 + p : p < kE / 2 ? e0 / 2 + p : e1 / 2 + p - kE / 2;
      cs[p] = turn(a.rope.freq[pair], pos, a.rope.attn_scale);
    }
  }
  for (;;) {
    const int more = head + kB * step;
    if (more < end) request(next, more);
#pragma unroll
    for (int k = 0; k < kB; ++k) {
      const int h = head + k * step, kind = h >= a.heads[0];
      if (h < end && turned) {
        float x[kE], y[kE];
        double u[kE], v[kE];
        unpack(now[k].w[0], x);
        unpack(now[k].w[1], y);
#pragma unroll
        for (int p = 0; p < kE; ++p) {
          if constexpr (kHalf) rotate_pair(x[p], y[p], cs[p], u[p], v[p]);
          else if (p < kE / 2) rotate_pair(x[2 * p], x[2 * p + 1], cs[p], u[2 * p], u[2 * p + 1]);
          else rotate_pair(y[2 * p - kE], y[2 * p - kE + 1], cs[p], v[2 * p - kE], v[2 * p - kE + 1]);
        }
        now[k].w[0] = pack(u);
        now[k].w[1] = pack(v);
      }
      if (h < end) now[k].store(dst[kind] + (kind ? h - a.heads[0] : h) * a.to[kind].head, e0, e1);
    }
    if (more >= end) break;
    head = more;
    for (int k = 0; k < kB; ++k) now[k] = next[k];
  }
}

template <typename T, int D>
void launch(RopeArgs& ra, hipStream_t stream) {
  // as many tokens as a wave has rows, fewer where there are fewer; heads over
  // enough waves to fill the GPU
  constexpr int kRows = 128 * Chunk<T>::kE / D;
  while (ra.log_tw < 31 && (1 << ra.log_tw) < kRows && (1 << ra.log_tw) < ra.tokens) ++ra.log_tw;
  const int waves = ((ra.tokens - 1) >> ra.log_tw) + 1, step = kRows >> ra.log_tw, heads = ra.heads[0] + ra.heads[1];
  const int slices = waves >= kWaves ? 1 : (kWaves + waves - 1) / waves;
  ra.hp = (heads + slices - 1) / slices;
  ra.hp = (ra.hp + step - 1) / step * step;
  const dim3 grid((waves + kThreads / 64 - 1) / (kThreads / 64), (heads + ra.hp - 1) / ra.hp);
  auto kernel = ra.rope.layout == RESKV_ROPE_HALF ? rope_kernel<T, D, true> : rope_kernel<T, D, false>;
  hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, stream, ra);
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
  ra.tokens = s.batch * n_rows;  // at most 2^26
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
