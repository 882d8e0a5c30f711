// 4-bit caches (include/reskv.h): packing a built cache, reading values back,
// appending tokens with the rotation of their keys.
#include "internal.h"
#include "quant.h"
#include "rotate.h"

namespace reskv {

namespace {

constexpr int kThreads = 256;

// Both kernels: thread = 8 elements of a row, 4 lanes a group of 32, the lanes of
// a wave along the rows; blockIdx.y = 2 (kv head) + (0 keys, 1 values), z = sequence.
// The 4 bytes of codes of 8 elements adjoin in the key rows and, at d = 128, in the
// value rows, where four neighbouring slots fill 256 bytes. Memory-bound; a thread
// packs kUnroll units of its block's run so that as many reads are in flight (256 x
// 2048 slots of 128, 340 MB: 69, 68, 64 us at 1, 2, 4; 8 x 512: 2.4, 2.6, 2.9).
constexpr int kUnroll = 4;

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void pack_kernel(const T* kc, const T* vc, const int32_t* res_len,
                                                        const int32_t* main_len, uint8_t* cache, int Hkv, int C,
                                                        int Rcap) {
  using Q = QuantBlock<D>;
  const bool value = blockIdx.y & 1;
  const int bh = blockIdx.z * Hkv + (blockIdx.y >> 1), e = (int)(threadIdx.x % (D / 8)) * 8;
  constexpr int kSlots = kThreads / (D / 8);  // slots of a block's unit
  const long long first = (long long)blockIdx.x * (kSlots * kUnroll) + threadIdx.x / (D / 8);
  int r, n;
  cache_lengths(res_len, main_len, bh, C, Rcap, r, n);
  if (first >= r + n) return;  // the four lanes of a group alike
  const T* src = (value ? vc : kc) + (size_t)bh * C * D + e;
  uint8_t* head = cache + (size_t)bh * (((size_t)C + 63) / 64) * Q::kBytes;
  float x[kUnroll][8];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) load8_f32(src + min(first + u * kSlots, (long long)(r + n - 1)) * D, x[u]);
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const long long slot = first + u * kSlots;
    uint32_t top = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) top = max(top, __float_as_uint(x[u][k]) & 0x7fffffffu);
    top = dpp_umax<0xB1>(top);
    top = dpp_umax<0x4E>(top);
    const uint32_t byte = scale_byte(top);
    const float scale = scale_of(byte);
    const uint32_t w = code_pair(x[u][0], x[u][1], scale) | code_pair(x[u][2], x[u][3], scale) << 8 |
                       code_pair(x[u][4], x[u][5], scale) << 16 | code_pair(x[u][6], x[u][7], scale) << 24;
    if (slot >= r + n) break;
    uint8_t* block = head + (size_t)(slot / 64) * Q::kBytes;
    const int s = (int)(slot % 64);
    if (!value) {
      *reinterpret_cast<uint32_t*>(block + Q::k_code(s) + e / 2) = w;
    } else if (Q::kPiece == 8) {
      *reinterpret_cast<uint32_t*>(block + Q::v_code(s, e / 8)) = w;
    } else {
      *reinterpret_cast<uint16_t*>(block + Q::v_code(s, e / 4)) = (uint16_t)w;
      *reinterpret_cast<uint16_t*>(block + Q::v_code(s, e / 4 + 1)) = (uint16_t)(w >> 16);
    }
    if (e % 32 == 0) block[value ? Q::v_scale(s, e / 32) : Q::k_scale(s, e / 32)] = (uint8_t)byte;
  }
}

// Values of more bytes than the last-level cache holds (256 MB) are stored past the
// caches: they would have left them before they are read again, and are written
// faster so (256 x 2304 rows of 128, 2048 of them live, 268 MB: 76 us through the
// caches, 48 past them, in a replayed graph). Fewer stay where the next call finds
// them. The lengths are on the device, so the bytes are those of the rows asked for,
// live or not.
constexpr double kStreamBytes = 256.0 * 1024 * 1024;

template <bool kStream>
__device__ __forceinline__ void store8_pairs(uint16_t* p, const uint32_t (&v)[4]) {
  store16<kStream>(p, u32x4_t{v[0], v[1], v[2], v[3]});
}
template <bool kStream>
__device__ __forceinline__ void store8_pairs(float* p, const uint32_t (&v)[4]) {
#pragma unroll
  for (int k = 0; k < 2; ++k)
    store16<kStream>(p + 4 * k, u32x4_t{v[2 * k] << 16, v[2 * k] & 0xffff0000u, v[2 * k + 1] << 16,
                                        v[2 * k + 1] & 0xffff0000u});
}

template <typename T, int D, bool kStream>
__global__ __launch_bounds__(kThreads) void unpack_kernel(const uint8_t* cache, const int32_t* res_len,
                                                          const int32_t* main_len, const int32_t* first, int n_rows,
                                                          T* kc, T* vc, int Hkv, int C, int Rcap) {
  using Q = QuantBlock<D>;
  const long long i = blockIdx.x * (long long)kThreads + threadIdx.x;
  const long long row = i / (D / 8);
  const int e = (int)(i % (D / 8)) * 8;
  const bool value = blockIdx.y & 1;
  const int bh = blockIdx.z * Hkv + (blockIdx.y >> 1);
  int r, n;
  cache_lengths(res_len, main_len, bh, C, Rcap, r, n);
  const long long slot = (first ? first[bh] : 0) + row;
  if (row >= n_rows || slot < 0 || slot >= r + n) return;
  const uint8_t* block = cache + ((size_t)bh * (((size_t)C + 63) / 64) + slot / 64) * Q::kBytes;
  const int s = (int)(slot % 64);
  const float scale = scale_of(block[value ? Q::v_scale(s, e / 32) : Q::k_scale(s, e / 32)]);
  uint32_t w;
  if (!value) {
    w = *reinterpret_cast<const uint32_t*>(block + Q::k_code(s) + e / 2);
  } else if (Q::kPiece == 8) {
    w = *reinterpret_cast<const uint32_t*>(block + Q::v_code(s, e / 8));
  } else {
    w = *reinterpret_cast<const uint16_t*>(block + Q::v_code(s, e / 4)) |
        (uint32_t)*reinterpret_cast<const uint16_t*>(block + Q::v_code(s, e / 4 + 1)) << 16;
  }
  const uint32_t v[4] = {value_pair<0>(w, scale), value_pair<1>(w, scale), value_pair<2>(w, scale),
                         value_pair<3>(w, scale)};
  store8_pairs<kStream>((value ? vc : kc) + ((size_t)bh * n_rows + row) * D + e, v);
}

struct AppendArgs {
  reskv_rope_t rope;
  const int32_t* positions;  // NULL: keys are not rotated
  const int32_t* n_tok;
  const void* k_new;
  const void* v_new;
  uint8_t* cache;
  const int32_t* res_len;
  int32_t* main_len;
  int n_new, C, Rcap;
};

// A wave per row (keys and values of a token are two); a block has kTokens tokens
// of one (b, kv head). kAdvance: the block has all of the call's tokens and
// advances main_len itself; else advance_kernel does, once every block has read it.
// us at 4, 8, 16, 32 tokens a block, with two of the four waves turning all keys: 8
// heads of 8 tokens 5.2, 5.0, 5.0, 5.0, of 64 5.1, 6.3, 8.8, 13.8; 256 heads of 16
// 6.3, 6.8, 7.8, 7.8, of 300 44, 40, 40, 43. With the turns dealt to every wave, at 8:
// 4.2, 5.5, 6.4, 39.7 (one token of 8 heads 3.1 -> 3.2). A lane with 8 elements of a
// row in place of 2 took 4.4 us for one token of 8 heads, 37 for 256 heads of 300.
// Rows requested before the lengths are known: no gain, and slower where n_tok leaves
// much of a call out.
constexpr int kTokens = 8;

template <typename T, int D, bool kAdvance>
__global__ __launch_bounds__(kThreads) void append_quant_kernel(AppendArgs a) {
  using Q = QuantBlock<D>;
  const int bh = blockIdx.z * gridDim.y + blockIdx.y, b = blockIdx.z;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  int r, n;
  cache_lengths(a.res_len, a.main_len, bh, a.C, a.Rcap, r, n);
  const int want = a.n_tok ? clampi(a.n_tok[b], 0, a.n_new) : a.n_new;
  const int take = min(want, a.C - r - n);
  const int t0 = blockIdx.x * kTokens, nt = min(kTokens, take - t0);  // below 1: nothing of this block is taken
  uint8_t* head = a.cache + (size_t)bh * (((size_t)a.C + 63) / 64) * Q::kBytes;
  const int l = min(lane, D / 2 - 1);  // lanes past the row do its last pair again and store nothing
  // Row j of the block: the keys of its nt tokens, then their values, wave by wave, so
  // that every wave has an equal part of the turns; two of them at once, because one
  // is a chain of 30 instructions.
  constexpr int kWaves = kThreads / 64, kRows = 2 * kTokens / kWaves, kKeys = kTokens / kWaves;
  static_assert(kKeys == 2, "turns of two keys together");
  const int rot = a.positions ? a.rope.rot_dim : 0;
  const int keys = rot ? nt - wave : 0;  // of this wave: above 0, above kWaves
  __shared__ double2 s_cs[kWaves][kKeys][64];
  PairElem<T> x[kRows], y[kRows];
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    const int j = wave + k * kWaves;
    if (j >= 2 * nt) break;  // wave-uniform
    const bool value = j >= nt;
    const PairIndex at(value ? 0 : rot, a.rope.layout);
    const T* src = static_cast<const T*>(value ? a.v_new : a.k_new) +
                   ((size_t)bh * a.n_new + t0 + (value ? j - nt : j)) * D;
    x[k].load(src, 2 * l, at);
    y[k].load(src, 2 * l + 1, at);
  }
  if (keys > 0) {
    double2* cs = s_cs[wave][0];
    const int32_t* pos = a.positions + (size_t)b * a.n_new + t0 + wave;
    const double freq = a.rope.freq[min(lane, rot / 2 - 1)];
    if (keys > kWaves) {
      const double2 c0 = turn(freq, pos[0], a.rope.attn_scale), c1 = turn(freq, pos[kWaves], a.rope.attn_scale);
      cs[lane] = c0;
      cs[64 + lane] = c1;
    } else {
      cs[lane] = turn(freq, pos[0], a.rope.attn_scale);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    const int j = wave + k * kWaves;
    if (j >= 2 * nt) break;
    const bool value = j >= nt;
    const PairIndex at(value ? 0 : rot, a.rope.layout);
    const double2* cs = s_cs[wave][min(k, kKeys - 1)];  // a key is one of the first rows
    const int slot = r + n + t0 + (value ? j - nt : j);
    store_row_quant<D>(head + (size_t)(slot / 64) * Q::kBytes, slot % 64, value, x[k].rotated(2 * l, at, cs),
                       y[k].rotated(2 * l + 1, at, cs), lane);
  }
  if (kAdvance) {
    __syncthreads();  // every wave has read the lengths
    if (tid == 0 && take > 0) a.main_len[bh] = n + take;
  }
}

__global__ __launch_bounds__(kThreads) void advance_kernel(AppendArgs a, int BH, int Hkv) {
  const int bh = blockIdx.x * kThreads + threadIdx.x;
  if (bh >= BH) return;
  int r, n;
  cache_lengths(a.res_len, a.main_len, bh, a.C, a.Rcap, r, n);
  const int want = a.n_tok ? clampi(a.n_tok[bh / Hkv], 0, a.n_new) : a.n_new;
  const int take = min(want, a.C - r - n);
  if (take > 0) a.main_len[bh] = n + take;
}

unsigned blocks_for(long long threads) { return (unsigned)((threads + kThreads - 1) / kThreads); }

template <typename T, int D>
void launch_pack(const reskv_shape_t& s, const void* kc, const void* vc, const int32_t* res_len,
                 const int32_t* main_len, void* cache, hipStream_t stream) {
  const dim3 grid(blocks_for(((long long)s.slot_cap * (D / 8) + kUnroll - 1) / kUnroll), 2 * s.num_kv_heads, s.batch);
  hipLaunchKernelGGL((pack_kernel<T, D>), grid, dim3(kThreads), 0, stream, (const T*)kc, (const T*)vc, res_len, main_len, (uint8_t*)cache,
                     s.num_kv_heads, s.slot_cap, s.res_cap);
}

template <typename T, int D>
void launch_unpack(const reskv_shape_t& s, const void* cache, const int32_t* res_len, const int32_t* main_len,
                   const int32_t* first, int n_rows, void* kc, void* vc, hipStream_t stream) {
  const dim3 grid(blocks_for((long long)n_rows * (D / 8)), 2 * s.num_kv_heads, s.batch);
  const bool past = 2.0 * sizeof(T) * s.batch * s.num_kv_heads * n_rows * D > kStreamBytes;
  auto kernel = past ? unpack_kernel<T, D, true> : unpack_kernel<T, D, false>;
  hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, stream, (const uint8_t*)cache, res_len, main_len, first, n_rows,
                     (T*)kc, (T*)vc, s.num_kv_heads, s.slot_cap, s.res_cap);
}

template <typename T, int D>
void launch_append(const reskv_shape_t& s, const AppendArgs& aa, hipStream_t stream) {
  const dim3 grid((aa.n_new + kTokens - 1) / kTokens, s.num_kv_heads, s.batch);
  if (grid.x == 1) {
    hipLaunchKernelGGL((append_quant_kernel<T, D, true>), grid, dim3(kThreads), 0, stream, aa);
    return;
  }
  hipLaunchKernelGGL((append_quant_kernel<T, D, false>), grid, dim3(kThreads), 0, stream, aa);
  const int BH = s.batch * s.num_kv_heads;
  hipLaunchKernelGGL(advance_kernel, dim3(blocks_for(BH)), dim3(kThreads), 0, stream, aa, BH, s.num_kv_heads);
}

}  // namespace

size_t quant_cache_bytes(const reskv_shape_t& s) {
  return (size_t)s.batch * s.num_kv_heads * (((size_t)s.slot_cap + 63) / 64) * 68 * s.head_dim;
}

hipError_t launch_pack_quant(const reskv_shape_t& s, const void* kc, const void* vc, const int32_t* res_len,
                             const int32_t* main_len, void* cache, hipStream_t stream) {
  const bool bf = s.dtype == RESKV_BF16;
  if (s.head_dim == 128)
    bf ? launch_pack<uint16_t, 128>(s, kc, vc, res_len, main_len, cache, stream)
       : launch_pack<float, 128>(s, kc, vc, res_len, main_len, cache, stream);
  else
    bf ? launch_pack<uint16_t, 64>(s, kc, vc, res_len, main_len, cache, stream)
       : launch_pack<float, 64>(s, kc, vc, res_len, main_len, cache, stream);
  return hipGetLastError();
}

hipError_t launch_unpack_quant(const reskv_shape_t& s, const void* cache, const int32_t* res_len,
                               const int32_t* main_len, const int32_t* first, int n_rows, void* kc, void* vc,
                               hipStream_t stream) {
  const bool bf = s.dtype == RESKV_BF16;
  if (s.head_dim == 128)
    bf ? launch_unpack<uint16_t, 128>(s, cache, res_len, main_len, first, n_rows, kc, vc, stream)
       : launch_unpack<float, 128>(s, cache, res_len, main_len, first, n_rows, kc, vc, stream);
  else
    bf ? launch_unpack<uint16_t, 64>(s, cache, res_len, main_len, first, n_rows, kc, vc, stream)
       : launch_unpack<float, 64>(s, cache, res_len, main_len, first, n_rows, kc, vc, stream);
  return hipGetLastError();
}

hipError_t launch_append_quant(const reskv_shape_t& s, const reskv_rope_t* rope, const int32_t* positions, int n_new,
                               const int32_t* n_tok, const void* k_new, const void* v_new, void* cache,
                               const int32_t* res_len, int32_t* main_len, hipStream_t stream) {
  AppendArgs aa{};
  if (rope) aa.rope = *rope;
  aa.positions = rope ? positions : nullptr;
  aa.n_tok = n_tok; aa.k_new = k_new; aa.v_new = v_new; aa.cache = (uint8_t*)cache;
  aa.res_len = res_len; aa.main_len = main_len;
  aa.n_new = n_new; aa.C = s.slot_cap; aa.Rcap = s.res_cap;
  const bool bf = s.dtype == RESKV_BF16;
  if (s.head_dim == 128) bf ? launch_append<uint16_t, 128>(s, aa, stream) : launch_append<float, 128>(s, aa, stream);
  else bf ? launch_append<uint16_t, 64>(s, aa, stream) : launch_append<float, 64>(s, aa, stream);
  return hipGetLastError();
}

}  // namespace reskv
