// 4-bit caches (include/reskv.h): packing a built cache, reading values back,
// appending tokens with the rotation of their keys.
#include "internal.h"
#include "quant.h"
#include "rotate.h"

namespace reskv {

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ void load32_f32(const uint16_t* p, float (&x)[32]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) load8_f32(p + 8 * j, reinterpret_cast<float(&)[8]>(x[8 * j]));
}
__device__ __forceinline__ void load32_f32(const float* p, float (&x)[32]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) load8_f32(p + 8 * j, reinterpret_cast<float(&)[8]>(x[8 * j]));
}

// Thread = one group of 32 elements of one row (index: pair, keys or values,
// slot, group).
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void pack_kernel(const T* kc, const T* vc, const int32_t* res_len,
                                                        const int32_t* main_len, uint8_t* cache, int BH, int C,
                                                        int Rcap) {
  using Q = QuantBlock<D>;
  const long long i = blockIdx.x * (long long)kThreads + threadIdx.x;
  const int c = (int)(i % Q::kGroups);
  long long rest = i / Q::kGroups;
  const int slot = (int)(rest % C);
  rest /= C;
  const bool value = rest & 1;
  const long long bh = rest >> 1;
  if (bh >= BH) return;
  int r, n;
  cache_lengths(res_len, main_len, (int)bh, C, Rcap, r, n);
  if (slot >= r + n) return;
  float x[32];
  load32_f32((value ? vc : kc) + ((size_t)bh * C + slot) * D + 32 * c, x);
  uint32_t top = 0;
#pragma unroll
  for (int k = 0; k < 32; ++k) top = max(top, __float_as_uint(x[k]) & 0x7fffffffu);
  const uint32_t byte = scale_byte(top);
  uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
  for (int k = 0; k < 16; ++k) w[k / 4] |= code_pair(x[2 * k], x[2 * k + 1], scale_of(byte)) << (8 * (k % 4));
  uint8_t* block = cache + ((size_t)bh * ((C + 63) / 64) + slot / 64) * Q::kBytes;
  const int s = slot % 64;
  if (value) {
    constexpr int kW = Q::kPiece / 2;  // bytes of a piece: 4 or 2
#pragma unroll
    for (int k = 0; k < 16 / kW; ++k) {
      uint8_t* at = block + Q::v_code(s, 32 * c / Q::kPiece + k);
      if (kW == 4) *reinterpret_cast<uint32_t*>(at) = w[k % 4];
      else *reinterpret_cast<uint16_t*>(at) = (uint16_t)(w[k / 2] >> (16 * (k % 2)));
    }
  } else {
    *reinterpret_cast<uint4*>(block + Q::k_code(s) + 16 * c) = make_uint4(w[0], w[1], w[2], w[3]);
  }
  block[value ? Q::v_scale(s, c) : Q::k_scale(s, c)] = (uint8_t)byte;
}

__device__ __forceinline__ void store8_pairs(uint16_t* p, const uint32_t (&v)[4]) {
  *reinterpret_cast<uint4*>(p) = make_uint4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ void store8_pairs(float* p, const uint32_t (&v)[4]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(bf16_lo(v[0]), bf16_hi(v[0]), bf16_lo(v[1]), bf16_hi(v[1]));
  reinterpret_cast<float4*>(p)[1] = make_float4(bf16_lo(v[2]), bf16_hi(v[2]), bf16_lo(v[3]), bf16_hi(v[3]));
}

// Thread = one group of 32 elements of one output row.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void unpack_kernel(const uint8_t* cache, const int32_t* res_len,
                                                          const int32_t* main_len, const int32_t* first, int n_rows,
                                                          T* kc, T* vc, int BH, int C, int Rcap) {
  using Q = QuantBlock<D>;
  const long long i = blockIdx.x * (long long)kThreads + threadIdx.x;
  const int c = (int)(i % Q::kGroups);
  long long rest = i / Q::kGroups;
  const int row = (int)(rest % n_rows);
  rest /= n_rows;
  const bool value = rest & 1;
  const long long bh = rest >> 1;
  if (bh >= BH) return;
  int r, n;
  cache_lengths(res_len, main_len, (int)bh, C, Rcap, r, n);
  const long long slot = (first ? first[bh] : 0) + (long long)row;
  if (slot < 0 || slot >= r + n) return;
  const uint8_t* block = cache + ((size_t)bh * ((C + 63) / 64) + slot / 64) * Q::kBytes;
  const int s = (int)(slot % 64);
  const float scale = scale_of(block[value ? Q::v_scale(s, c) : Q::k_scale(s, c)]);
  T* out = (value ? vc : kc) + ((size_t)bh * n_rows + row) * D + 32 * c;
#pragma unroll
  for (int k = 0; k < 4; ++k) {  // 8 elements: 4 bytes of codes
    uint32_t w;
    if (!value) {
      w = *reinterpret_cast<const uint32_t*>(block + Q::k_code(s) + 16 * c + 4 * k);
    } else if (Q::kPiece == 8) {
      w = *reinterpret_cast<const uint32_t*>(block + Q::v_code(s, 4 * c + k));
    } else {
      w = *reinterpret_cast<const uint16_t*>(block + Q::v_code(s, 8 * c + 2 * k)) |
          (uint32_t)*reinterpret_cast<const uint16_t*>(block + Q::v_code(s, 8 * c + 2 * k + 1)) << 16;
    }
    const uint32_t v[4] = {value_pair<0>(w, scale), value_pair<1>(w, scale), value_pair<2>(w, scale),
                           value_pair<3>(w, scale)};
    store8_pairs(out + 8 * k, v);
  }
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
  int n_new, Hkv, C, Rcap;
};

// One block per (b, kv head), a wave per row: keys and values of token 0, of
// token 1, ...
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void append_quant_kernel(AppendArgs a) {
  using Q = QuantBlock<D>;
  const int bh = blockIdx.x, b = bh / a.Hkv, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  int r, n;
  cache_lengths(a.res_len, a.main_len, bh, a.C, a.Rcap, r, n);
  const int want = a.n_tok ? clampi(a.n_tok[b], 0, a.n_new) : a.n_new;
  const int take = min(want, a.C - r - n);
  uint8_t* head = a.cache + (size_t)bh * ((a.C + 63) / 64) * Q::kBytes;
  const int l = min(lane, D / 2 - 1);  // lanes past the row do its last pair again and store nothing
  __shared__ double2 s_cs[kThreads / 64][64];
  for (int row = wave; row < 2 * take; row += kThreads / 64) {  // wave-uniform
    const int t = row >> 1;
    const bool value = row & 1;
    const T* src = static_cast<const T*>(value ? a.v_new : a.k_new) + ((size_t)bh * a.n_new + t) * D;
    const PairIndex at(!value && a.positions ? a.rope.rot_dim : 0, a.rope.layout);
    PairElem<T> x, y;
    x.load(src, 2 * l, at);
    y.load(src, 2 * l + 1, at);
    if (at.rot) {
      if (lane < a.rope.rot_dim / 2)
        s_cs[wave][lane] = turn(a.rope.freq[lane], a.positions[(size_t)b * a.n_new + t], a.rope.attn_scale);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
    const int slot = r + n + t;
    store_row_quant<D>(head + (size_t)(slot / 64) * Q::kBytes, slot % 64, value,
                       x.rotated(2 * l, at, s_cs[wave]), y.rotated(2 * l + 1, at, s_cs[wave]), lane);
    __builtin_amdgcn_wave_barrier();
  }
  __syncthreads();  // every wave has read the lengths
  if (tid == 0 && take > 0) a.main_len[bh] = n + take;
}

unsigned blocks_for(long long threads) { return (unsigned)((threads + kThreads - 1) / kThreads); }

template <typename T, int D>
void launch_pack(const reskv_shape_t& s, const void* kc, const void* vc, const int32_t* res_len,
                 const int32_t* main_len, void* cache, hipStream_t stream) {
  const int BH = s.batch * s.num_kv_heads;
  hipLaunchKernelGGL((pack_kernel<T, D>), dim3(blocks_for(2LL * BH * s.slot_cap * (D / 32))), dim3(kThreads), 0, stream,
                     (const T*)kc, (const T*)vc, res_len, main_len, (uint8_t*)cache, BH, s.slot_cap, s.res_cap);
}

template <typename T, int D>
void launch_unpack(const reskv_shape_t& s, const void* cache, const int32_t* res_len, const int32_t* main_len,
                   const int32_t* first, int n_rows, void* kc, void* vc, hipStream_t stream) {
  const int BH = s.batch * s.num_kv_heads;
  hipLaunchKernelGGL((unpack_kernel<T, D>), dim3(blocks_for(2LL * BH * n_rows * (D / 32))), dim3(kThreads), 0, stream,
                     (const uint8_t*)cache, res_len, main_len, first, n_rows, (T*)kc, (T*)vc, BH, s.slot_cap,
                     s.res_cap);
}

template <typename T, int D>
void launch_append(const AppendArgs& aa, int BH, hipStream_t stream) {
  hipLaunchKernelGGL((append_quant_kernel<T, D>), dim3(BH), dim3(kThreads), 0, stream, aa);
}

}  // namespace

size_t quant_cache_bytes(const reskv_shape_t& s) {
  return (size_t)s.batch * s.num_kv_heads * ((s.slot_cap + 63) / 64) * 68 * s.head_dim;
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
  aa.n_new = n_new; aa.Hkv = s.num_kv_heads; aa.C = s.slot_cap; aa.Rcap = s.res_cap;
  const bool bf = s.dtype == RESKV_BF16;
  const int BH = s.batch * s.num_kv_heads;
  if (s.head_dim == 128) bf ? launch_append<uint16_t, 128>(aa, BH, stream) : launch_append<float, 128>(aa, BH, stream);
  else bf ? launch_append<uint16_t, 64>(aa, BH, stream) : launch_append<float, 64>(aa, BH, stream);
  return hipGetLastError();
}

}  // namespace reskv
