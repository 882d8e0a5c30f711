// Shared-softmax residual decode (Sec. 5.4; Sec. 5.5.2 gate; App. D, Algorithm 2)
// over a cache held in 4 bits.
//
// One block of 8 waves per (b, kv head), or several where few heads have long
// caches; a wave takes blocks of 64 slots (the cache's own blocks) and keeps a
// running maximum, sum and output per query head for the residual slots, then for
// the main slots; the waves' states are merged in LDS, where the gate joins the
// two kinds, or in a second launch over the blocks' records. With hd = lane % 16,
// g = lane / 16:
//   * logits S^T = K Q^T per 16-slot tile t: lane (hd, g) loads D / 4 elements
//     of key row 16t + hd (16 bytes at D = 128), all of one scale, which the
//     conversion applies: every code times its scale is a bf16 number, so the
//     matrix instruction gets exact operands. The contraction index of step i,
//     lane group g stands for elements g D/4 + 8i .. + 7 on both sides. The lane
//     ends with the logits of slots 16t + 4g + i' of head hd, in base 2 with
//     log2(e) / sqrt(d) in the scale.
//   * O^T += V^T P^T: lane (m, g) loads the m-th piece (D / 16 elements) of value
//     rows 16T + 4g + u, u = 0..3, in one load per T; contraction index 8g + i'
//     of step h stands for slot 16(2h + i'/4) + 4g + i'%4, so the B operand is
//     the lane's own probabilities, as bf16 hi + lo parts, each rounded to
//     nearest: for p in [1, 2) the first is off by at most 2^-8, and what is below
//     2^-8 by at most 2^-17 once it is rounded (2^-17 of the probability).
// fp32 queries enter as three bf16 parts, which hold all of their 24 bits. (The
// scaled products of 4-bit with 8-bit numbers would need no conversion of keys, but
// their sums over differently scaled groups were off by up to 2^-11 of the largest
// product; logits need 2^-20.)
//
// Bound by reading the units, with about 3 us before the first one (arguments,
// lengths, queries, rotation) and 1.5 us after the last (merge, gate), by clocks in the
// kernel. d = 128, bf16, a launch in a replayed graph: 256 heads of 2048 slots, 4 query
// heads each (72 MB), 16.8 us where the last-level cache holds them, 18.9 us from memory
// (3.8 TB/s); 8 heads of 65000 slots 20.5 and 22.1 us, 4 of them the join; 8 heads of
// 512 with rotation and append 8.4 us.
#include "internal.h"
#include "quant.h"
#include "rotate.h"

namespace reskv {

namespace {

// A CU holds one block at d = 128 (151 to 174 registers a wave: two waves a SIMD, or
// three, where a second block would need four) and two at d = 64 (at most 125
// registers; one with 16 fp32 heads, whose LDS two would pass). 16 waves of half the
// registers and units ran 23.6 us where 8 ran 17.3 (d = 128, 256 heads of 2048 slots):
// what a wave does once weighs as much as two units. Requesting a unit ahead changed
// nothing (17.4).
constexpr int kWaves = 8;
constexpr int kThreads = 64 * kWaves;
constexpr int kUnit = 64;  // slots of a cache block
constexpr int kTiles = kUnit / 16;
// 16 bytes a row, so that the rows of the heads start in different LDS banks (788
// thousand conflict clocks a launch of 256 heads without, 1.5 thousand with; uneven
// caches of 7 query heads 12.4 -> 11.8 us)
constexpr int kPadQ = 8, kPadAcc = 4;
constexpr int kMaxParts = 64;  // blocks a head is split over

struct QuantDecodeArgs {
  reskv_rope_t rope;
  const int32_t* positions;  // NULL: no rotation
  const void* q;
  uint8_t* cache;
  const float* logc;
  const int32_t* res_len;
  int32_t* main_len;
  const void* k_new;  // appended first, or NULL
  const void* v_new;
  const float* tau;
  float* out;
  float* dbg_lse_main;
  float* dbg_lse_res;
  float* dbg_gate;
  float* rec_ml;   // split: [BH][P][2 kinds][GP][2] (maximum in base 2, sum)
  float* rec_acc;  // split: [BH][P][2 kinds][GP][D], written for kinds with slots
  int G, C, Rcap, NB;
  int P, W;        // blocks of a head and cache blocks of each (unsplit: 1, NB)
  float qk_scale;   // log2(e) / sqrt(d)
  float beta_log2;  // beta * log2(e)
  float tau_scalar, alpha, g_min;
};

template <int kBytes>
struct Words;
template <>
struct Words<16> {
  uint32_t w[4];
  __device__ __forceinline__ void load(const uint8_t* p) {
    const uint4 x = *reinterpret_cast<const uint4*>(p);
    w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
  }
};
template <>
struct Words<8> {
  uint32_t w[2];
  __device__ __forceinline__ void load(const uint8_t* p) {
    const uint2 x = *reinterpret_cast<const uint2*>(p);
    w[0] = x.x; w[1] = x.y;
  }
};

// One block of 64 slots in registers.
template <int D>
struct Unit {
  Words<D / 8> k[kTiles];  // key codes of row 16t + hd, elements g D/4 ..
  uint32_t ks;             // their scales, byte t
  Words<D / 8> v[kTiles];  // value codes of piece hd, rows 16T + 4g + u
  Words<16> vs;            // their scales, word T, byte u
  float lc;                // log-count of slot `lane` (of an entry; else unused)
  __device__ __forceinline__ void load(const uint8_t* cache, int blk, const float* logc, int Rcap, int lane) {
    const uint8_t* block = cache + (size_t)blk * QuantBlock<D>::kBytes;
    const int hd = lane & 15, g = lane >> 4;
    using Q = QuantBlock<D>;
    constexpr int kLanes = 4 / Q::kGroups;  // lane groups of one key scale
#pragma unroll
    for (int t = 0; t < kTiles; ++t) k[t].load(block + Q::k_code(16 * t + hd) + g * (D / 8));
    ks = *reinterpret_cast<const uint32_t*>(block + Q::k_scale(hd, g / kLanes));
#pragma unroll
    for (int t = 0; t < kTiles; ++t) v[t].load(block + Q::v_code(16 * t + 4 * g, hd));
    vs.load(block + Q::v_scale(4 * g, hd * Q::kPiece / 32));
    lc = logc[min(blk * kUnit + lane, Rcap - 1)];
  }
};

template <int kByte>
__device__ __forceinline__ float byte_scale(uint32_t w) {
  return scale_of((w >> (8 * kByte)) & 0xffu);
}

// 8 codes of a word as 8 bf16 numbers.
__device__ __forceinline__ uint4 eight(uint32_t codes, float scale) {
  return make_uint4(value_pair<0>(codes, scale), value_pair<1>(codes, scale), value_pair<2>(codes, scale),
                    value_pair<3>(codes, scale));
}

// Products of the unit's keys and the queries, whose fragments are read from LDS
// here (kept in registers over the unit they would not fit beside the rest).
template <int D, int GP, int NP>
__device__ __forceinline__ void unit_logits(const Unit<D>& u, const uint16_t (*s_q)[GP][D + kPadQ], int hq, int g,
                                            float (&s)[kTiles][4]) {
  uint4 q[NP][D / 32];
#pragma unroll
  for (int p = 0; p < NP; ++p)
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
      q[p][i] = *reinterpret_cast<const uint4*>(&s_q[p][min(hq, GP - 1)][g * (D / 4) + 8 * i]);
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    const float scale = t == 0 ? byte_scale<0>(u.ks) : t == 1 ? byte_scale<1>(u.ks)
                      : t == 2 ? byte_scale<2>(u.ks) : byte_scale<3>(u.ks);
    f32x4_t c = zero4();
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      const bf16x8_t k = as_bf16x8(eight(u.k[t].w[i], scale));
#pragma unroll
      for (int p = NP - 1; p >= 0; --p)  // the smallest part first
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, as_bf16x8(q[p][i]), c, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) s[t][i] = c[i];
  }
}

// Running state of one kind of slots: head hd's maximum and sum (the same in
// the four lane groups), and O[hd][(D/16)(4g + i) + e] in acc[e][i].
template <int D>
struct State {
  static constexpr int kE = D / 16;
  float m, l;
  f32x4_t acc[kE];
  __device__ void reset() {
    m = kNegInf;
    l = 0.f;
#pragma unroll
    for (int e = 0; e < kE; ++e) acc[e] = zero4();
  }
};

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  typedef __attribute__((ext_vector_type(2))) float f32x2_t;
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2_t{a, b}, bf16x2_t));
}

// Up to 8 query heads take half of the 16 columns of a matrix instruction: the
// other half holds the same heads, with the low parts of their probabilities
// (one product where more heads need two).
template <int GP>
constexpr bool kPaired = GP <= 8;

// O^T += V^T P^T for the unit; rows without weight must hold finite numbers.
template <int D, int GP>
__device__ __forceinline__ void pv_unit(State<D>& st, const Unit<D>& u, const float (&p)[kTiles][4], int hd) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t bh[4], bl[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float pa = p[2 * h + w / 2][2 * (w % 2)], pb = p[2 * h + w / 2][2 * (w % 2) + 1];
      bh[w] = pack_bf16(pa, pb);
      bl[w] = pack_bf16(pa - bf16_lo(bh[w]), pb - bf16_hi(bh[w]));
      if (kPaired<GP> && hd >= 8) bh[w] = bl[w];
    }
    const bf16x8_t Bh = as_bf16x8(make_uint4(bh[0], bh[1], bh[2], bh[3]));
    const bf16x8_t Bl = as_bf16x8(make_uint4(bl[0], bl[1], bl[2], bl[3]));
    // element pair e, e + 1 of the 8 rows of this step
    auto step = [&](int e, const uint32_t (&x)[8]) {
#pragma unroll
      for (int o = 0; o < 2; ++o) {
        const uint32_t sel = o ? 0x07060302u : 0x05040100u;
        uint32_t a[4];
#pragma unroll
        for (int w = 0; w < 4; ++w) a[w] = __builtin_amdgcn_perm(x[2 * w + 1], x[2 * w], sel);
        const bf16x8_t A = as_bf16x8(make_uint4(a[0], a[1], a[2], a[3]));
        st.acc[e + o] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(A, Bh, st.acc[e + o], 0, 0, 0);
        if (!kPaired<GP>) st.acc[e + o] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(A, Bl, st.acc[e + o], 0, 0, 0);
      }
    };
    float vs[8];  // scales of the rows
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      vs[4 * t] = byte_scale<0>(u.vs.w[2 * h + t]);
      vs[4 * t + 1] = byte_scale<1>(u.vs.w[2 * h + t]);
      vs[4 * t + 2] = byte_scale<2>(u.vs.w[2 * h + t]);
      vs[4 * t + 3] = byte_scale<3>(u.vs.w[2 * h + t]);
    }
    uint32_t x[8];
    if constexpr (D == 128) {  // a word per row
#define RESKV_PAIRS(B)                                                                       \
  {                                                                                          \
    _Pragma("unroll") for (int k = 0; k < 8; ++k) x[k] =                                     \
        value_pair<B>(u.v[2 * h + k / 4].w[k % 4], vs[k]);                                   \
    step(2 * B, x);                                                                          \
  }
      RESKV_PAIRS(0) RESKV_PAIRS(1) RESKV_PAIRS(2) RESKV_PAIRS(3)
#undef RESKV_PAIRS
    } else {  // half a word per row
#define RESKV_PAIRS(B)                                                                       \
  {                                                                                          \
    _Pragma("unroll") for (int k = 0; k < 8; k += 2) {                                       \
      x[k] = value_pair<B>(u.v[2 * h + k / 4].w[k % 4 / 2], vs[k]);                          \
      x[k + 1] = value_pair<B + 2>(u.v[2 * h + k / 4].w[k % 4 / 2], vs[k + 1]);              \
    }                                                                                        \
    step(2 * B, x);                                                                          \
  }
      RESKV_PAIRS(0) RESKV_PAIRS(1)
#undef RESKV_PAIRS
    }
  }
}

// A logit in 32 bits. Rounded here and never within a later sum: the maximum and the
// exponents are of the same numbers, so that the largest weight is exactly 1. (With the
// product fused into the exponent's difference it was off by half of a step of the
// logit: by 2^64 at 2^31, and a p_max of 0.8 to 1.2 where it is 1 from 2^22 on.)
__device__ __forceinline__ float scaled(float product, float qk_scale) {
#pragma clang fp contract(off)
  return product * qk_scale;
}

// Online softmax over the unit's slots [lo, hi) of one kind, from the logits'
// products p, which become the probabilities. Residual slots add beta * log2 count;
// slots of no weight (outside, empty entries) get zero probability and the least
// scale, so whatever their codes say does not enter. A unit full of main slots
// needs none of that.
template <int D, int GP>
__device__ __forceinline__ void softmax_pv(State<D>& st, Unit<D>& u, float (&p)[kTiles][4], int lo, int hi,
                                           bool is_res, float qk_scale, float beta_log2, float* s_bias, int lane) {
  const int hd = lane & 15, g = lane >> 4;
  float top = kNegInf;
  const bool full = !is_res && lo <= 0 && hi >= kUnit;  // wave-uniform
  if (full) {
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[t][i] = scaled(p[t][i], qk_scale);
        top = fmaxf(top, p[t][i]);
      }
  } else {
    // what a slot's logits are moved by (-inf: no weight), from the lane of the
    // slot to the lanes of its logits
    const bool weighs = lane >= lo && lane < hi && !(is_res && u.lc == kNegInf);
    s_bias[lane] = !weighs ? kNegInf : is_res ? beta_log2 * u.lc : 0.f;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      const f32x4_t bias = *reinterpret_cast<const f32x4_t*>(&s_bias[16 * t + 4 * g]);
      uint32_t mask = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool live = bias[i] != kNegInf;
        p[t][i] = live ? fmaf(p[t][i], qk_scale, bias[i]) : kNegInf;
        mask |= live ? 0xffu << (8 * i) : 0u;
        top = fmaxf(top, p[t][i]);
      }
      u.vs.w[t] &= mask;
    }
  }
  const float m_new = fmaxf(st.m, rows4_max(top));
  const float mu = m_new == kNegInf ? 0.f : m_new;
  const float alpha = fast_exp2(st.m - mu);
  float sum = 0.f;
#pragma unroll
  for (int t = 0; t < kTiles; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      p[t][i] = fast_exp2(p[t][i] - mu);
      sum += p[t][i];
    }
  sum = rows4_sum(sum);
  st.l = fmaf(st.l, alpha, sum);
  // logits that are all NaN leave no maximum: 0 in its place keeps their sum in the merges
  st.m = m_new == kNegInf && sum != 0.f ? 0.f : m_new;
#pragma unroll
  for (int e = 0; e < State<D>::kE; ++e)
#pragma unroll
    for (int i = 0; i < 4; ++i) st.acc[e][i] *= alpha;
  pv_unit<D, GP>(st, u, p, hd);
}

template <int D, int GP>
__device__ __forceinline__ void store_state(State<D>& st, float (*acc)[D + kPadAcc], float* m, float* l, int hd,
                                            int g) {
  constexpr int kE = D / 16;
  if (kPaired<GP>) {  // the other half's part (row_ror:8)
#pragma unroll
    for (int e = 0; e < kE; ++e)
#pragma unroll
      for (int i = 0; i < 4; ++i) st.acc[e][i] += dpp_move<0x128>(st.acc[e][i]);
  }
  if (hd < GP) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < kE; e += 4)
        *reinterpret_cast<float4*>(&acc[hd][kE * (4 * g + i) + e]) =
            make_float4(st.acc[e][i], st.acc[e + 1][i], st.acc[e + 2][i], st.acc[e + 3][i]);
    if (g == 0) {
      m[hd] = st.m;
      l[hd] = st.l;
    }
  }
}

// The gate joins the two kinds of one (query head, column): maxima, sums and
// unnormalised outputs in, the output out.
struct Joined {
  float gate, fM, fR, inv;  // factors on the main and residual sums, 1 / denominator
};
__device__ __forceinline__ Joined join(const QuantDecodeArgs& a, int qh, float mM, float lM, float mR, float lR) {
  const float tau = a.tau ? a.tau[qh] : a.tau_scalar;
  // p_max = 1 / l_main (the largest term is exactly 1), then the gate
  const float pmax = lM > 0.f ? 1.f / lM : 1.f;
  Joined j;
  j.gate = fmaxf(a.g_min, 1.f / (1.f + expf(-(tau - pmax) * a.alpha)));
  // hardware logarithm and powers (an ulp; the logarithm of a gate below 2^-126 by
  // way of 2^64 of it, weights below 2^-126 are 0)
  const float lg = j.gate > 0.f ? __builtin_amdgcn_logf(j.gate * 0x1p64f) - 64.f : kNegInf;
  const float mRg = (mR == kNegInf || lg == kNegInf) ? kNegInf : mR + lg;
  const float M = fmaxf(mM, mRg);
  j.fM = mM != kNegInf ? fast_exp2(mM - M) : 0.f;
  j.fR = mRg != kNegInf ? fast_exp2(mRg - M) : 0.f;
  const float den = lM * j.fM + lR * j.fR;
  j.inv = den != 0.f ? 1.f / den : 0.f;  // NaN stays NaN
  return j;
}
__device__ __forceinline__ void write_stats(const QuantDecodeArgs& a, int qh, float mM, float lM, float mR, float lR,
                                            float gate) {
  if (a.dbg_lse_main) a.dbg_lse_main[qh] = lM != 0.f ? (mM + log2f(lM)) * kLn2 : kNegInf;
  if (a.dbg_lse_res) a.dbg_lse_res[qh] = lR != 0.f ? (mR + log2f(lR)) * kLn2 : kNegInf;
  if (a.dbg_gate) a.dbg_gate[qh] = gate;
}

// Block p of P of a (b, kv head): its cache blocks [p W, (p + 1) W). kSplit: the
// merged states of both kinds go to records, which decode_quant_combine joins;
// else this block has the whole head and finishes it.
template <typename T, int D, int GP, bool kSplit>
__global__ __launch_bounds__(kThreads) void decode_quant_kernel(QuantDecodeArgs a) {
  using Q = QuantBlock<D>;
  constexpr int NP = sizeof(T) == 2 ? 1 : 3;
  const int kvh = blockIdx.x, b = blockIdx.y, part = kSplit ? blockIdx.z : 0;
  const int bh = b * gridDim.x + kvh;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int hd = lane & 15, g = lane >> 4;

  __shared__ __align__(16) float s_acc[2][kWaves][GP][D + kPadAcc];
  __shared__ float s_m[2][kWaves][GP];  // per kind (0 residual, 1 main), per wave
  __shared__ float s_l[2][kWaves][GP];
  __shared__ float s_w[2][kWaves][GP];
  __shared__ __align__(16) float s_bias[kWaves][kUnit];
  __shared__ __align__(16) uint16_t s_q[NP][GP][D + kPadQ];
  __shared__ double2 s_cs[64];

  // The arguments that the first requests need, read together: left to where
  // each is used, they came in a chain of six reads of up to 500 clocks.
  const int32_t* positions = a.positions;
  const int32_t* res_len = a.res_len;
  const int32_t* main_len = a.main_len;
  const T* qp = static_cast<const T*>(a.q);
  const T* kp = static_cast<const T*>(a.k_new);
  const T* vp = static_cast<const T*>(a.v_new);
  uint8_t* cache = a.cache;
  const float* logc = a.logc;
  const double* freqs = a.rope.freq;
  const int rot = a.rope.rot_dim, layout = a.rope.layout, G = a.G, NB = a.NB, Rcap = a.Rcap, C = a.C, W = a.W;
  asm volatile("" ::"s"(positions), "s"(res_len), "s"(main_len), "s"(qp), "s"(kp), "s"(vp), "s"(cache), "s"(logc),
               "s"(freqs), "s"(rot), "s"(layout), "s"(G), "s"(NB), "s"(Rcap), "s"(C), "s"(W));
  cache += (size_t)bh * NB * Q::kBytes;
  logc += (size_t)bh * Rcap;
  const int begin = part * W;

  // Requests that wait for nothing more, in the order of their use: the queries and
  // this step's token with the partners of their elements, then the wave's first
  // unit. (A wait for one load is a wait for all before it.)
  constexpr int kQ = (GP * D + kThreads - 1) / kThreads;
  const int pos = *(positions ? positions + b : res_len + bh);  // unused without a rotation
  const int r_raw = res_len[bh], n_raw = main_len[bh];
  const PairIndex at(positions ? rot : 0, layout);
  double freq = 0.0;
  if (at.rot) freq = freqs[min(lane, rot / 2 - 1)];
  PairElem<T> qe[kQ], ne[2];
  qp += (size_t)bh * G * D;
#pragma unroll
  for (int k = 0; k < kQ; ++k) {
    const int i = tid + k * kThreads;
    qe[k].load(qp + min(i / D, G - 1) * D, i % D, at);
  }
  const PairIndex at_new(wave ? 0 : at.rot, layout);
  const int l_new = min(lane, D / 2 - 1);
  const T* new_row = kp ? (wave ? vp : kp) + (size_t)bh * D : qp;  // wave 0 has the key, wave 1 the value
  ne[0].load(new_row, 2 * l_new, at_new);
  ne[1].load(new_row, 2 * l_new + 1, at_new);
  Unit<D> u;
  u.load(cache, min(begin + wave, NB - 1), logc, Rcap, lane);
  __builtin_amdgcn_sched_barrier(0);  // no wait for any of them before the last is on its way
  int r, n;
  clamp_lengths(r_raw, n_raw, C, Rcap, r, n);
  const bool app = kp != nullptr && r + n < C;
  const int app_slot = r + n;
  if (app) n += 1;
  const int total = r + n;
  const int end = min(begin + W, (total + kUnit - 1) / kUnit);
  if (kSplit && begin >= end) {  // no live slot here: records without weight
    for (int i = tid; i < 2 * GP; i += kThreads) {
      float* ml = a.rec_ml + (((size_t)bh * a.P + part) * 2 * GP + i) * 2;
      ml[0] = kNegInf;
      ml[1] = 0.f;
    }
    return;
  }
  if (at.rot) {
    if (tid < 64) s_cs[tid] = turn(freq, pos, a.rope.attn_scale);
    __syncthreads();
  }
  // queries, rotated, as bf16 parts
#pragma unroll
  for (int k = 0; k < kQ; ++k) {
    const int i = tid + k * kThreads, h = i / D, e = i % D;
    if (h >= GP) continue;
    float x = h < G ? qe[k].rotated(e, at, s_cs) : 0.f;
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      // truncated: exact in one part or three, and never past the largest number
      const uint32_t w = __float_as_uint(x) & 0xffff0000u;
      s_q[p][h][e] = (uint16_t)(w >> 16);
      x -= __uint_as_float(w);
    }
  }
  const int app_blk = app && app_slot / kUnit >= begin && app_slot / kUnit < end ? app_slot / kUnit : -1;
  if (app_blk >= 0 && wave < 2)
    store_row_quant<D>(cache + (size_t)app_blk * Q::kBytes, app_slot % kUnit, wave == 1,
                       ne[0].rotated(2 * l_new, at_new, s_cs), ne[1].rotated(2 * l_new + 1, at_new, s_cs), lane);
  __syncthreads();
  const int hq = kPaired<GP> ? hd & 7 : hd;  // query head of this lane's column
  if (app_blk == begin + wave) u.load(cache, app_blk, logc, Rcap, lane);  // with the new token

  // Units: the cache blocks in order (their residual slots if they have any), then
  // once more the one that holds slot r, for its main slots. The waves take them in
  // turn, so each meets its residual units first.
  State<D> st;
  st.reset();
  bool in_res = true;
  const bool both = r % kUnit != 0 && n > 0 && r / kUnit >= begin && r / kUnit < end;
  const int units = end - begin + (both ? 1 : 0);
  auto block_of = [&](int i) { return i < end - begin ? begin + i : r / kUnit; };
  auto work = [&](Unit<D>& u, int i) __attribute__((always_inline)) {
    const int s0 = block_of(i) * kUnit;
    const bool is_res = i < end - begin && s0 < r;
    if (!is_res && in_res) {
      store_state<D, GP>(st, s_acc[0][wave], s_m[0][wave], s_l[0][wave], hd, g);
      st.reset();
      in_res = false;
    }
    float p[kTiles][4];
    unit_logits<D, GP, NP>(u, s_q, hq, g, p);
    softmax_pv<D, GP>(st, u, p, is_res ? 0 : r - s0, (is_res ? r : total) - s0, is_res, a.qk_scale, a.beta_log2,
                      s_bias[wave], lane);
  };
  int i = wave;
  if (both && i == units - 1) u.load(cache, r / kUnit, logc, Rcap, lane);
  for (; i + kWaves < units; i += kWaves) {
    work(u, i);
    u.load(cache, block_of(i + kWaves), logc, Rcap, lane);
  }
  if (i < units) work(u, i);
  if (in_res) {
    store_state<D, GP>(st, s_acc[0][wave], s_m[0][wave], s_l[0][wave], hd, g);
    st.reset();
  }
  store_state<D, GP>(st, s_acc[1][wave], s_m[1][wave], s_l[1][wave], hd, g);
  __syncthreads();

  // Weights of the waves' states: 16 lanes a head, lane 8 kind + w of wave w's.
  // Sums within 8 lanes by neighbours, pairs and the mirror of 8, which meets the
  // four lanes that hold the other partial sum.
  if (tid < 16 * GP) {
    const int h = tid >> 4, kind = (tid >> 3) & 1, w = tid & 7;
    const float m = s_m[kind][w][h], l = s_l[kind][w][h];
    float M = m;
    M = fmaxf(M, dpp_move<0xB1>(M));
    M = fmaxf(M, dpp_move<0x4E>(M));
    M = fmaxf(M, dpp_move<0x141>(M));
    const float f = m != kNegInf ? fast_exp2(m - M) : 0.f;
    float L = m != kNegInf ? f * l : 0.f;
    L += dpp_move<0xB1>(L);
    L += dpp_move<0x4E>(L);
    L += dpp_move<0x141>(L);
    if constexpr (kSplit) {
      s_w[kind][w][h] = f;
      if (w == 0) {
        float* ml = a.rec_ml + (((size_t)bh * a.P + part) * 2 * GP + kind * GP + h) * 2;
        ml[0] = M;
        ml[1] = L;
      }
    } else {
      const float Mo = dpp_move<0x128>(M), Lo = dpp_move<0x128>(L);  // the other kind's (row_ror:8)
      const float mM = kind ? M : Mo, lM = kind ? L : Lo, mR = kind ? Mo : M, lR = kind ? Lo : L;
      if (h < G) {
        const int qh = bh * G + h;
        const Joined j = join(a, qh, mM, lM, mR, lR);
        s_w[kind][w][h] = m != kNegInf ? f * (kind ? j.fM : j.fR) * j.inv : 0.f;
        if ((tid & 15) == 0) write_stats(a, qh, mM, lM, mR, lR, j.gate);
      }
    }
  }
  __syncthreads();
  // the outputs, four columns a thread
  const bool has_res = begin * kUnit < r, has_main = end * kUnit > r && total > r;
  auto weighed = [&](int kind, int h, int d) {
    f32x4_t o = zero4();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = s_w[kind][w][h];
      const f32x4_t v = *reinterpret_cast<const f32x4_t*>(&s_acc[kind][w][h][d]);
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = fmaf(f, v[i], o[i]);
    }
    return o;
  };
  for (int i = tid; i < G * (D / 4); i += kThreads) {
    const int h = i / (D / 4), d = i % (D / 4) * 4;
    if constexpr (kSplit) {
      float* rec = a.rec_acc + (((size_t)bh * a.P + part) * 2 * GP + h) * D + d;
      if (has_res) *reinterpret_cast<f32x4_t*>(rec) = weighed(0, h, d);
      if (has_main) *reinterpret_cast<f32x4_t*>(rec + GP * D) = weighed(1, h, d);
    } else {
      f32x4_t o = zero4();
      if (has_main) o = weighed(1, h, d);
      if (has_res) o += weighed(0, h, d);
      float* out = a.out + ((size_t)bh * G + h) * D + d;  // 4-byte aligned
#pragma unroll
      for (int k = 0; k < 4; ++k) out[k] = o[k];
    }
  }
  if (!kSplit && app && tid == 0) a.main_len[bh] = n;
}

// Join the records of one query head: thread = one column (tid % D) of every
// kGroups-th part. Outputs are requested before their weights are known; every
// record has its maximum and sum (those without slots -inf and 0: what is read of
// their outputs does not enter), so the cache lengths are not needed, and main_len
// advances here: by the block of the group's first head, which alone reads it.
constexpr int kJoinThreads = 512;

template <int D, int GP>
__global__ __launch_bounds__(kJoinThreads) void decode_quant_combine(QuantDecodeArgs a) {
  constexpr int kGroups = kJoinThreads / D, kPer = kMaxParts / kGroups;  // parts of a thread
  const int h = blockIdx.x, bh = blockIdx.z * gridDim.y + blockIdx.y;
  const int tid = threadIdx.x, lane = tid & 63, d = tid % D, group = tid / D;
  __shared__ float s_w[2][kMaxParts];
  __shared__ float s_o[kGroups][D];
  const size_t row0 = (size_t)bh * a.P * 2 * GP + h;  // record (part p, kind) is row (2 p + kind) GP further
  const float2* ml = reinterpret_cast<const float2*>(a.rec_ml) + row0;
  const int P = a.P, mine = min(lane, P - 1);
  float2 eR = ml[(size_t)(2 * mine) * GP], eM = ml[(size_t)(2 * mine + 1) * GP];
  const float* acc = a.rec_acc + row0 * D + d;
  float vR[kPer], vM[kPer];
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int p = min(group + k * kGroups, P - 1);
    vR[k] = acc[(size_t)(2 * p) * GP * D];
    vM[k] = acc[(size_t)(2 * p + 1) * GP * D];
  }
  if (lane >= P) eR = eM = make_float2(kNegInf, 0.f);
  const float mR = rows4_max(row16_max(eR.x)), mM = rows4_max(row16_max(eM.x));
  const float fR = eR.x != kNegInf ? fast_exp2(eR.x - mR) : 0.f, fM = eM.x != kNegInf ? fast_exp2(eM.x - mM) : 0.f;
  const float lR = rows4_sum(row16_sum(eR.x != kNegInf ? fR * eR.y : 0.f));
  const float lM = rows4_sum(row16_sum(eM.x != kNegInf ? fM * eM.y : 0.f));
  const int qh = bh * a.G + h;
  const Joined j = join(a, qh, mM, lM, mR, lR);
  if (tid < 64) {  // -1: a record without slots
    s_w[0][lane] = eR.x != kNegInf ? fR * j.fR * j.inv : -1.f;
    s_w[1][lane] = eM.x != kNegInf ? fM * j.fM * j.inv : -1.f;
  }
  __syncthreads();
  float o = 0.f;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int p = group + k * kGroups;
    if (p >= P) continue;
    const float wR = s_w[0][p], wM = s_w[1][p];
    if (!(wR < 0.f)) o = fmaf(wR, vR[k], o);
    if (!(wM < 0.f)) o = fmaf(wM, vM[k], o);
  }
  s_o[group][d] = o;
  __syncthreads();
  if (group == 0) {
    o = s_o[0][d];
#pragma unroll
    for (int g = 1; g < kGroups; ++g) o += s_o[g][d];
    a.out[(size_t)qh * D + d] = o;
  }
  if (tid == 0) {
    write_stats(a, qh, mM, lM, mR, lR, j.gate);
    if (h == 0 && a.k_new) {
      int r, n;
      cache_lengths(a.res_len, a.main_len, bh, a.C, a.Rcap, r, n);
      if (r + n < a.C) a.main_len[bh] = n + 1;
    }
  }
}

template <typename T, int D, int GP>
void launch_kernels(const QuantDecodePlan& pl, const QuantDecodeArgs& da, hipStream_t stream) {
  if (pl.P == 1) {
    hipLaunchKernelGGL((decode_quant_kernel<T, D, GP, false>), dim3(pl.Hkv, pl.B), dim3(kThreads), 0,
                       stream, da);
    return;
  }
  hipLaunchKernelGGL((decode_quant_kernel<T, D, GP, true>), dim3(pl.Hkv, pl.B, pl.P), dim3(kThreads), 0,
                     stream, da);
  hipLaunchKernelGGL((decode_quant_combine<D, GP>), dim3(da.G, pl.Hkv, pl.B), dim3(kJoinThreads), 0, stream, da);
}

template <typename T, int D>
hipError_t launch_gp(const QuantDecodePlan& pl, const QuantDecodeArgs& da, hipStream_t stream) {
  switch (pl.GP) {
    case 1: launch_kernels<T, D, 1>(pl, da, stream); break;
    case 2: launch_kernels<T, D, 2>(pl, da, stream); break;
    case 4: launch_kernels<T, D, 4>(pl, da, stream); break;
    case 8: launch_kernels<T, D, 8>(pl, da, stream); break;
    default: launch_kernels<T, D, 16>(pl, da, stream); break;
  }
  return hipGetLastError();
}

}  // namespace

// One block per (b, kv head), or its cache blocks dealt to several and their records
// joined by a second launch. A block takes 512 slots a round (8 waves of 64), about
// 2 us each while the blocks do not fill the memory's rate; the join and its launch
// cost 3 us, more once 256 blocks stream at once. Blocks past 256 (one a CU at d = 128)
// only wait. Measured at d = 128, bf16, 4 query heads per KV head, every slot live, us one
// block / split so that up to 256 blocks run (lengths uniform in [C/4, C] within 1 us
// of both):
//   pairs     C = 1024     1500       2048       2560       4096       8192
//     1      8.6/ 9.7  10.7/ 9.6  12.6/ 9.6  14.5/ 9.7  20.1/ 9.9  35.3/ 9.9
//    32      8.9/10.0  11.0/10.2  13.0/10.3  15.5/10.8  21.6/12.0  37.9/14.5
//    64      9.1/10.3  11.7/11.4  13.6/12.0  15.7/13.6  22.0/14.4  38.2/19.6
//   128     10.0/12.9  12.2/14.9  14.5/15.2  16.3/19.2  22.5/20.6  46.1/35.2
//   240     11.0/20.4  14.2/22.6  16.7/25.1  18.9/27.6  30.6/38.1  (two or more each)
// (8 query heads 0.5 to 1 us more on both sides; fp32 rows of 64, 32 pairs: 7.6/8.3,
// 9.3/8.4, 10.8/8.3, 12.2/8.6, 17.3/8.6, 31.9/11.2.) So a split has to save two
// rounds, four where the pairs alone fill more than a quarter of the CUs. From 129 to
// 239 pairs, and beyond 256 blocks at d = 64, where a CU holds two, nothing was measured:
// heads stay whole from 129 pairs on, and 256 blocks are the most at both widths.
QuantDecodePlan make_quant_decode_plan(const reskv_shape_t& s) {
  QuantDecodePlan p{};
  p.B = s.batch;
  p.Hkv = s.num_kv_heads;
  const long long BH = (long long)p.B * p.Hkv;
  const int G = s.num_q_heads / s.num_kv_heads;
  p.GP = G <= 1 ? 1 : G <= 2 ? 2 : G <= 4 ? 4 : G <= 8 ? 8 : 16;
  const int NB = (int)(((long long)s.slot_cap + kUnit - 1) / kUnit);
  p.P = 1;
  p.W = NB;
  if (BH <= 128) {
    const int want = 256 / (int)BH < kMaxParts ? 256 / (int)BH : kMaxParts;
    const int rounds = (NB + kWaves - 1) / kWaves, each = (rounds + want - 1) / want;
    if (rounds - each >= (BH <= 64 ? 2 : 4)) {
      p.W = each * kWaves;
      p.P = (NB + p.W - 1) / p.W;
    }
  }
  const size_t rows = p.P > 1 ? (size_t)BH * p.P * 2 * p.GP : 0;
  p.acc_off = align_up(rows * 2 * sizeof(float), 256);
  p.bytes = align_up(p.acc_off + rows * s.head_dim * sizeof(float), 256) + 256;  // never 0
  return p;
}

hipError_t launch_decode_quant(const reskv_shape_t& s, const reskv_gate_t& g, const QuantDecodePlan& pl,
                               const reskv_rope_t* rope, const int32_t* positions, const void* q, void* cache,
                               const float* logc, const int32_t* res_len, int32_t* main_len, const void* k_new,
                               const void* v_new, float* out, float* dbg_lse_main, float* dbg_lse_res,
                               float* dbg_gate, void* workspace, hipStream_t stream) {
  QuantDecodeArgs da{};
  if (rope) da.rope = *rope;
  da.positions = rope ? positions : nullptr;
  da.q = q; da.cache = (uint8_t*)cache; da.logc = logc;
  da.res_len = res_len; da.main_len = main_len; da.k_new = k_new; da.v_new = v_new;
  da.tau = g.tau; da.out = out;
  da.rec_ml = static_cast<float*>(workspace);
  da.rec_acc = reinterpret_cast<float*>(static_cast<char*>(workspace) + pl.acc_off);
  da.P = pl.P; da.W = pl.W;
  da.dbg_lse_main = dbg_lse_main; da.dbg_lse_res = dbg_lse_res; da.dbg_gate = dbg_gate;
  da.G = s.num_q_heads / s.num_kv_heads;
  da.C = s.slot_cap; da.Rcap = s.res_cap; da.NB = (int)(((long long)s.slot_cap + kUnit - 1) / kUnit);
  da.qk_scale = kLog2e / sqrtf((float)s.head_dim);
  da.beta_log2 = g.beta * kLog2e;
  da.tau_scalar = g.tau_scalar; da.alpha = g.alpha; da.g_min = g.g_min;
  const bool bf = s.dtype == RESKV_BF16;
  if (s.head_dim == 128) return bf ? launch_gp<uint16_t, 128>(pl, da, stream) : launch_gp<float, 128>(pl, da, stream);
  return bf ? launch_gp<uint16_t, 64>(pl, da, stream) : launch_gp<float, 64>(pl, da, stream);
}

}  // namespace reskv
