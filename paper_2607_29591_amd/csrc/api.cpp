// C ABI of the ResKV hot path: argument validation, workspace sizing and
// launch on the caller's stream. Every check runs on the host before any
// kernel is enqueued.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>
#include <string.h>

#include "internal.h"

using namespace reskv;

namespace {

thread_local char g_last_error[512] = "";

reskv_status_t fail(reskv_status_t st, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
reskv_status_t fail(reskv_status_t st, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_last_error, sizeof(g_last_error), fmt, ap);
  va_end(ap);
  return st;
}

reskv_status_t ok() {
  g_last_error[0] = '\0';
  return RESKV_OK;
}

reskv_status_t check_shape(const reskv_shape_t* s) {
  if (!s) return fail(RESKV_ERR_INVALID_ARG, "shape is NULL");
  if (s->batch < 1) return fail(RESKV_ERR_INVALID_ARG, "batch must be >= 1 (got %d)", s->batch);
  if (s->num_kv_heads < 1 || s->num_q_heads < 1)
    return fail(RESKV_ERR_INVALID_ARG, "head counts must be >= 1 (Hq=%d, Hkv=%d)", s->num_q_heads, s->num_kv_heads);
  if (s->num_q_heads % s->num_kv_heads != 0)
    return fail(RESKV_ERR_INVALID_ARG, "Hq (%d) must be a multiple of Hkv (%d)", s->num_q_heads, s->num_kv_heads);
  if (s->num_q_heads / s->num_kv_heads > 16)
    return fail(RESKV_ERR_UNSUPPORTED, "group size Hq/Hkv = %d > 16", s->num_q_heads / s->num_kv_heads);
  if (s->head_dim != 64 && s->head_dim != 128)
    return fail(RESKV_ERR_UNSUPPORTED, "head_dim %d not in {64, 128}", s->head_dim);
  if (s->dtype != RESKV_F32 && s->dtype != RESKV_BF16)
    return fail(RESKV_ERR_UNSUPPORTED, "dtype %d not in {F32, BF16}", s->dtype);
  if (s->slot_cap < 1) return fail(RESKV_ERR_INVALID_ARG, "slot_cap must be >= 1 (got %d)", s->slot_cap);
  if (s->res_cap < 1) return fail(RESKV_ERR_INVALID_ARG, "res_cap must be >= 1 (got %d)", s->res_cap);
  const double cells = (double)s->batch * s->num_kv_heads * s->slot_cap * s->head_dim;
  if (cells > 4.0e12) return fail(RESKV_ERR_INVALID_ARG, "cache of %.3g elements is too large", cells);
  return RESKV_OK;
}

reskv_status_t check_gate(const reskv_gate_t* g) {
  if (!g) return fail(RESKV_ERR_INVALID_ARG, "gate is NULL");
  if (!(g->g_min >= 0.f && g->g_min <= 1.f)) return fail(RESKV_ERR_INVALID_ARG, "g_min %g outside [0, 1]", g->g_min);
  if (!isfinite(g->alpha) || !isfinite(g->beta) || !isfinite(g->tau_scalar))
    return fail(RESKV_ERR_INVALID_ARG, "gate parameters must be finite");
  if (g->beta < 0.f) return fail(RESKV_ERR_INVALID_ARG, "beta %g must be >= 0", g->beta);
  return RESKV_OK;
}

// Workspace that a decode call writes: one block per head leaves no records.
size_t decode_records_bytes(const DecodePlan& plan) { return plan.whole_head ? 0 : plan.bytes; }

}  // namespace

extern "C" {

const char* reskv_status_string(reskv_status_t st) {
  switch (st) {
    case RESKV_OK: return "ok";
    case RESKV_ERR_INVALID_ARG: return "invalid argument";
    case RESKV_ERR_UNSUPPORTED: return "unsupported configuration";
    case RESKV_ERR_WORKSPACE: return "workspace missing or too small";
    case RESKV_ERR_HIP: return "HIP runtime error";
  }
  return "unknown status";
}

const char* reskv_last_error(void) { return g_last_error; }

size_t reskv_decode_workspace_size(const reskv_shape_t* shape) {
  if (check_shape(shape) != RESKV_OK) return 0;
  const DecodePlan plan = make_decode_plan(*shape);
  if ((size_t)plan.GP * plan.P * sizeof(float) > decode_max_lds_weights()) return 0;
  return plan.bytes;
}

reskv_status_t reskv_decode_attn(const reskv_shape_t* shape, const reskv_gate_t* gate, const void* q,
                                 void* kc, void* vc, const float* logc,
                                 const int32_t* res_len, int32_t* main_len,
                                 const void* k_new, const void* v_new, float* out,
                                 float* dbg_lse_main, float* dbg_lse_res, float* dbg_gate,
                                 void* workspace, size_t workspace_bytes, void* stream) {
  reskv_status_t st = check_shape(shape);
  if (st != RESKV_OK) return st;
  if ((st = check_gate(gate)) != RESKV_OK) return st;
  if (!q || !kc || !vc || !logc || !res_len || !main_len || !out)
    return fail(RESKV_ERR_INVALID_ARG, "a required pointer is NULL");
  if ((k_new == nullptr) != (v_new == nullptr))
    return fail(RESKV_ERR_INVALID_ARG, "k_new and v_new must both be given or both be NULL");
  const DecodePlan plan = make_decode_plan(*shape);
  if ((size_t)plan.GP * plan.P * sizeof(float) > decode_max_lds_weights())
    return fail(RESKV_ERR_UNSUPPORTED, "%d split-K records per head do not fit the combine", plan.P);
  if (!workspace || workspace_bytes < plan.bytes)
    return fail(RESKV_ERR_WORKSPACE, "decode needs %zu workspace bytes, got %zu", plan.bytes,
                workspace ? workspace_bytes : (size_t)0);
  hipError_t e = launch_decode(*shape, *gate, plan, q, kc, vc, logc, res_len, main_len, k_new, v_new, out,
                               dbg_lse_main, dbg_lse_res, dbg_gate, workspace, (hipStream_t)stream);
  if (e != hipSuccess) return fail(RESKV_ERR_HIP, "decode launch failed: %s", hipGetErrorString(e));
  return ok();
}

reskv_status_t reskv_decode_attn_static(const reskv_shape_t* shape, const reskv_gate_t* gate, const void* q,
                                        void* kc, void* vc, const float* logc, const int32_t* res_len,
                                        int32_t* main_len, const void* k_new, const void* v_new, float* out,
                                        float* dbg_lse_main, float* dbg_lse_res, float* dbg_gate, void* stream) {
  reskv_status_t st = check_shape(shape);
  if (st != RESKV_OK) return st;
  if ((st = check_gate(gate)) != RESKV_OK) return st;
  if (!q || !kc || !vc || !logc || !res_len || !main_len || !out)
    return fail(RESKV_ERR_INVALID_ARG, "a required pointer is NULL");
  if ((k_new == nullptr) != (v_new == nullptr))
    return fail(RESKV_ERR_INVALID_ARG, "k_new and v_new must both be given or both be NULL");
  const DecodePlan plan = make_decode_plan(*shape);
  if ((size_t)plan.GP * plan.P * sizeof(float) > decode_max_lds_weights())
    return fail(RESKV_ERR_UNSUPPORTED, "%d split-K records per head do not fit the combine", plan.P);
  // from 256 (b, kv head) pairs on no capacity needs split-K records; below,
  // the limit is that of the split path whichever path a capacity takes
  const size_t need = plan.no_records ? 0 : plan.bytes;
  if (need > kStaticScratchBytes)
    return fail(RESKV_ERR_WORKSPACE,
                "this shape needs %zu bytes of split-K scratch, above the %zu bytes of the library's static "
                "scratch; use reskv_decode_attn with a workspace",
                need, kStaticScratchBytes);
  void* ws = nullptr;
  hipError_t e = static_scratch(&ws);
  if (e != hipSuccess) return fail(RESKV_ERR_HIP, "static scratch lookup failed: %s", hipGetErrorString(e));
  e = launch_decode(*shape, *gate, plan, q, kc, vc, logc, res_len, main_len, k_new, v_new, out, dbg_lse_main,
                    dbg_lse_res, dbg_gate, ws, (hipStream_t)stream);
  if (e != hipSuccess) return fail(RESKV_ERR_HIP, "decode launch failed: %s", hipGetErrorString(e));
  return ok();
}

size_t reskv_decode_ragged_workspace_size(const reskv_shape_t* shape) {
  if (check_shape(shape) != RESKV_OK) return 0;
  RaggedPlan plan;
  if (!make_ragged_plan(*shape, &plan)) return 0;
  const size_t other = ragged_takes_decode(*shape) ? decode_records_bytes(make_decode_plan(*shape)) : 0;
  return plan.bytes > other ? plan.bytes : other;
}

reskv_status_t reskv_decode_attn_ragged(const reskv_shape_t* shape, const reskv_gate_t* gate, const void* q,
                                        void* kc, void* vc, const float* logc, const int32_t* res_len,
                                        int32_t* main_len, const void* k_new, const void* v_new, float* out,
                                        float* dbg_lse_main, float* dbg_lse_res, float* dbg_gate, void* workspace,
                                        size_t workspace_bytes, void* stream) {
  reskv_status_t st = check_shape(shape);
  if (st != RESKV_OK) return st;
  if ((st = check_gate(gate)) != RESKV_OK) return st;
  if (!q || !kc || !vc || !logc || !res_len || !main_len || !out)
    return fail(RESKV_ERR_INVALID_ARG, "a required pointer is NULL");
  if ((k_new == nullptr) != (v_new == nullptr))
    return fail(RESKV_ERR_INVALID_ARG, "k_new and v_new must both be given or both be NULL");
  RaggedPlan plan;
  if (!make_ragged_plan(*shape, &plan))
    return fail(RESKV_ERR_UNSUPPORTED,
                "the ragged schedule takes group sizes up to 8, at most 2048 (sequence, KV head) pairs, slot "
                "capacities up to 64960 and bf16 rows (fp32 rows of 64)");
  if (!workspace || workspace_bytes < plan.bytes)
    return fail(RESKV_ERR_WORKSPACE, "ragged decode needs %zu workspace bytes, got %zu", plan.bytes,
                workspace ? workspace_bytes : (size_t)0);
  if (ragged_takes_decode(*shape)) {
    const DecodePlan dp = make_decode_plan(*shape);
    if (workspace_bytes >= decode_records_bytes(dp)) {  // a smaller one holds the equal ranges' records
      const hipError_t e = launch_decode(*shape, *gate, dp, q, kc, vc, logc, res_len, main_len, k_new, v_new, out,
                                         dbg_lse_main, dbg_lse_res, dbg_gate, workspace, (hipStream_t)stream);
      if (e != hipSuccess) return fail(RESKV_ERR_HIP, "decode launch failed: %s", hipGetErrorString(e));
      return ok();
    }
  }
  hipError_t e = launch_decode_ragged(*shape, *gate, plan, q, kc, vc, logc, res_len, main_len, k_new, v_new, out,
                                      dbg_lse_main, dbg_lse_res, dbg_gate, workspace, (hipStream_t)stream);
  if (e != hipSuccess) return fail(RESKV_ERR_HIP, "decode launch failed: %s", hipGetErrorString(e));
  return ok();
}

reskv_status_t reskv_decode_branches(const reskv_shape_t* shape, const reskv_gate_t* gate, const void* q,
                                     const void* kc, const void* vc, const float* logc, const int32_t* res_len,
                                     const int32_t* main_len, float* out_main, float* lse_main, float* out_res,
                                     float* lse_res, float* gate_out, void* workspace, size_t workspace_bytes,
                                     void* stream) {
  reskv_status_t st = check_shape(shape);
  if (st != RESKV_OK) return st;
  if ((st = check_gate(gate)) != RESKV_OK) return st;
  if (!q || !kc || !vc || !logc || !res_len || !main_len || !out_main || !lse_main || !out_res || !lse_res ||
      !gate_out)
    return fail(RESKV_ERR_INVALID_ARG, "a required pointer is NULL");
  const DecodePlan plan = make_decode_plan(*shape, true);
  if ((size_t)plan.GP * plan.P * sizeof(float) > decode_max_lds_weights())
    return fail(RESKV_ERR_UNSUPPORTED, "%d split-K records per head do not fit the combine", plan.P);
  if (!workspace || workspace_bytes < plan.bytes)
    return fail(RESKV_ERR_WORKSPACE, "decode needs %zu workspace bytes, got %zu", plan.bytes,
                workspace ? workspace_bytes : (size_t)0);
  hipError_t e = launch_decode_branches(*shape, *gate, plan, q, kc, vc, logc, res_len, main_len, out_main, lse_main,
                                        out_res, lse_res, gate_out, workspace, (hipStream_t)stream);
  if (e != hipSuccess) return fail(RESKV_ERR_HIP, "decode launch failed: %s", hipGetErrorString(e));
  return ok();
}

int reskv_internal_decode_kernels(const reskv_shape_t* shape, int entry) {
  if (entry < 0 || entry > 2 || check_shape(shape) != RESKV_OK) return -1;
  if (entry == 2) {
    RaggedPlan rp;
    if (!make_ragged_plan(*shape, &rp)) return -1;
    if (!ragged_takes_decode(*shape)) return kEqualRanges;
  }
  const DecodePlan plan = make_decode_plan(*shape, entry == 1);
  if ((size_t)plan.GP * plan.P * sizeof(float) > decode_max_lds_weights()) return -1;
  return plan.whole_head ? kOneBlockPerHead : kSplitCombine;
}

reskv_status_t reskv_merge_branches(const reskv_shape_t* shape, int32_t mode, const float* out_main,
                                    const float* lse_main, const float* out_res, const float* lse_res,
                                    const float* gate, float* out, void* stream) {
  reskv_status_t st = check_shape(shape);
  if (st != RESKV_OK) return st;
  if (mode != RESKV_MERGE_SHARED && mode != RESKV_MERGE_SEPARATE)
    return fail(RESKV_ERR_INVALID_ARG, "merge mode %d is neither SHARED (0) nor SEPARATE (1)", mode);
  if (!out_main || !lse_main || !out_res || !lse_res || !gate || !out)
    return fail(RESKV_ERR_INVALID_ARG, "a required pointer is NULL");
  if (out == out_main || out == out_res) return fail(RESKV_ERR_INVALID_ARG, "out must not alias a branch output");
  hipError_t e = launch_merge_branches(*shape, mode, out_main, lse_main, out_res, lse_res, gate, out,
                                       (hipStream_t)stream);
  if (e != hipSuccess) return fail(RESKV_ERR_HIP, "merge launch failed: %s", hipGetErrorString(e));
  return ok();
}

reskv_status_t reskv_append_kv(const reskv_shape_t* shape, const void* k_new, const void* v_new, void* kc,
                               void* vc, const int32_t* res_len, int32_t* main_len, void* stream) {
  reskv_status_t st = check_shape(shape);
  if (st != RESKV_OK) return st;
  if (!k_new || !v_new || !kc || !vc || !res_len || !main_len)
    return fail(RESKV_ERR_INVALID_ARG, "a required pointer is NULL");
  hipError_t e = launch_append(*shape, k_new, v_new, kc, vc, res_len, main_len, (hipStream_t)stream);
  if (e != hipSuccess) return fail(RESKV_ERR_HIP, "append launch failed: %s", hipGetErrorString(e));
  return ok();
}

// Rows of a call of the rotation, the append or the read-back: a launch has fewer
// than 2^32 threads along a dimension, and indices of rows stay within 32 bits.
constexpr int64_t kMaxRows = 1 << 26;

// Row accesses move 16 bytes.
static bool aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

reskv_status_t reskv_rope_init(const reskv_rope_params_t* p, reskv_rope_t* rope, double* freq_host) {
  if (!p || !rope || !freq_host) return fail(RESKV_ERR_INVALID_ARG, "params, rope or freq_host is NULL");
  if (p->rot_dim < 16 || p->rot_dim > 128 || p->rot_dim % 16 != 0)
    return fail(RESKV_ERR_UNSUPPORTED, "rot_dim %d is not a multiple of 16 in [16, 128]", p->rot_dim);
  if (p->layout != RESKV_ROPE_HALF && p->layout != RESKV_ROPE_INTERLEAVED)
    return fail(RESKV_ERR_INVALID_ARG, "layout %d is neither HALF (0) nor INTERLEAVED (1)", p->layout);
  if (p->scaling < RESKV_ROPE_NONE || p->scaling > RESKV_ROPE_YARN)
    return fail(RESKV_ERR_INVALID_ARG, "scaling %d outside [0, 4]", p->scaling);
  if (!(p->theta > 1.0) || !isfinite(p->theta)) return fail(RESKV_ERR_INVALID_ARG, "theta %g must be > 1", p->theta);
  if (p->scaling != RESKV_ROPE_NONE && !(p->factor >= 1.0 && isfinite(p->factor)))
    return fail(RESKV_ERR_INVALID_ARG, "factor %g must be >= 1", p->factor);
  if (p->scaling >= RESKV_ROPE_LLAMA3 && !(p->original_len > 0.0 && isfinite(p->original_len)))
    return fail(RESKV_ERR_INVALID_ARG, "original_len %g must be > 0", p->original_len);
  if (p->scaling == RESKV_ROPE_LLAMA3 &&
      !(p->low_freq_factor > 0.0 && p->high_freq_factor > p->low_freq_factor && isfinite(p->high_freq_factor)))
    return fail(RESKV_ERR_INVALID_ARG, "frequency factors must satisfy 0 < low (%g) < high (%g)", p->low_freq_factor,
                p->high_freq_factor);
  if (p->scaling == RESKV_ROPE_YARN && !(p->beta_slow > 0.0 && p->beta_fast > p->beta_slow && isfinite(p->beta_fast)))
    return fail(RESKV_ERR_INVALID_ARG, "betas must satisfy beta_fast (%g) > beta_slow (%g) > 0", p->beta_fast,
                p->beta_slow);
  if (!(p->attn_scale >= 0.0) || !isfinite(p->attn_scale))
    return fail(RESKV_ERR_INVALID_ARG, "attn_scale %g must be >= 0", p->attn_scale);
  make_rope(*p, rope, freq_host);
  return ok();
}

// A plan of reskv_rope_init with its frequencies on the device, for rows of `shape`.
static reskv_status_t check_rope(const reskv_shape_t* s, const reskv_rope_t* rope) {
  if (rope->rot_dim < 16 || rope->rot_dim % 16 != 0 || rope->rot_dim > s->head_dim)
    return fail(RESKV_ERR_INVALID_ARG, "rot_dim %d of the plan is not a multiple of 16 in [16, head_dim = %d]",
                rope->rot_dim, s->head_dim);
  if (rope->layout != RESKV_ROPE_HALF && rope->layout != RESKV_ROPE_INTERLEAVED)
    return fail(RESKV_ERR_INVALID_ARG, "layout %d of the plan is neither HALF (0) nor INTERLEAVED (1)", rope->layout);
  if (!isfinite(rope->attn_scale)) return fail(RESKV_ERR_INVALID_ARG, "attn_scale of the plan must be finite");
  if (!rope->freq) return fail(RESKV_ERR_INVALID_ARG, "the plan has no frequencies on the device");
  return RESKV_OK;
}

// Rows of one operand, in bytes.
struct RowSet {
  int64_t first;
  int64_t stride[3], extent[3];  // batch, head, row
};

// Whether a row of a and a row of b have bytes in common: a sum z_0 s_0 + z_1 s_1 + ...
// of strides that moves a's first row to less than a row's bytes from b's. A stride
// that both have is one term, their places' difference; else each has its own. Terms
// are chosen by falling stride, only where what the smaller ones reach, and what is a
// multiple of all of them, can still come near enough: a few tries where every stride
// passes what the smaller ones span, as in tensors and slices of tensors.
enum Overlap { kApart = 0, kCommon = 1, kUntold = 2 };  // kUntold: given up
struct OverlapSearch {
  int64_t bytes;  // of a row
  int terms = 0, tries = 0;
  int64_t s[6], lo[6], hi[6];
  int64_t least[7], most[7], unit[7];  // of the sums of terms t and on; what they are multiples of

  void add(int64_t stride, int64_t from, int64_t to) {
    if (stride == 0 || from == to) return;
    int t = terms++;
    for (; t > 0 && s[t - 1] < stride; --t) s[t] = s[t - 1], lo[t] = lo[t - 1], hi[t] = hi[t - 1];
    s[t] = stride, lo[t] = from, hi[t] = to;
  }
  static int64_t down(int64_t a, int64_t b) { return a / b - (a % b < 0 ? 1 : 0); }  // floor(a / b), b > 0
  Overlap from(int t, int64_t d) {
    if (d + most[t] <= -bytes || d + least[t] >= bytes) return kApart;
    if (t == terms) return kCommon;
    const int64_t past = d - unit[t] * down(d, unit[t]);
    if (past >= bytes && unit[t] - past >= bytes) return kApart;
    if (++tries > 100000) return kUntold;
    int64_t z0 = -down(bytes - 1 + most[t + 1] + d, s[t]), z1 = down(bytes - 1 - least[t + 1] - d, s[t]);
    if (z0 < lo[t]) z0 = lo[t];
    if (z1 > hi[t]) z1 = hi[t];
    for (int64_t z = z0; z <= z1; ++z) {
      const Overlap o = from(t + 1, d + z * s[t]);
      if (o != kApart) return o;
    }
    return kApart;
  }
};

static Overlap rows_overlap(const RowSet& a, const RowSet& b, int64_t bytes) {
  OverlapSearch f{bytes};
  for (int i = 0; i < 3; ++i) {
    if (a.stride[i] == b.stride[i]) {
      f.add(a.stride[i], 1 - b.extent[i], a.extent[i] - 1);
    } else {
      f.add(a.stride[i], 0, a.extent[i] - 1);
      f.add(b.stride[i], 1 - b.extent[i], 0);
    }
  }
  f.least[f.terms] = f.most[f.terms] = f.unit[f.terms] = 0;
  for (int t = f.terms - 1; t >= 0; --t) {
    f.least[t] = f.least[t + 1] + f.lo[t] * f.s[t];
    f.most[t] = f.most[t + 1] + f.hi[t] * f.s[t];
    int64_t x = f.s[t], y = f.unit[t + 1];
    while (y) {
      const int64_t m = x % y;
      x = y;
      y = m;
    }
    f.unit[t] = x;
  }
  return f.from(0, a.first - b.first);
}

static RowSet row_set(const reskv_shape_t* s, int heads, int n, const void* p, const reskv_rows_t* at) {
  const int64_t e = s->dtype == RESKV_BF16 ? 2 : 4;
  RowSet r{(int64_t)reinterpret_cast<uintptr_t>(p), {at->batch, at->head, at->row}, {s->batch, heads, n}};
  for (int i = 0; i < 3; ++i) r.stride[i] = r.extent[i] > 1 ? r.stride[i] * e : 0;  // an unused one may be anything
  return r;
}

int reskv_internal_rows_overlap(const int64_t* a, const int64_t* b, int64_t bytes) {
  return rows_overlap({a[0], {a[1], a[2], a[3]}, {a[4], a[5], a[6]}}, {b[0], {b[1], b[2], b[3]}, {b[4], b[5], b[6]}},
                      bytes);
}

// No row of an output over a row of another operand.
static reskv_status_t check_apart(const reskv_shape_t* s, const RowSet& out, const char* name, const char* role,
                                  const RowSet& other, const char* other_name, const char* other_role) {
  switch (rows_overlap(out, other, s->head_dim * (s->dtype == RESKV_BF16 ? 2 : 4))) {
    case kApart: return RESKV_OK;
    case kCommon:
      return fail(RESKV_ERR_INVALID_ARG, "rows of the %s %s overlap those of the %s %s", name, role, other_name,
                  other_role);
    case kUntold: break;
  }
  return fail(RESKV_ERR_INVALID_ARG, "the %s %s and the %s %s interleave by strides that are not told apart", name,
              role, other_name, other_role);
}

// Input and output rows of one kind of heads.
static reskv_status_t check_rows(const reskv_shape_t* s, const char* name, int heads, int n, const void* in,
                                 const reskv_rows_t* from, void* out, const reskv_rows_t* to) {
  if (!in && !out) return RESKV_OK;
  if (!in || !out || !from || !to)
    return fail(RESKV_ERR_INVALID_ARG, "%s needs its input, its output and the strides of both", name);
  if (!aligned(in) || !aligned(out)) return fail(RESKV_ERR_INVALID_ARG, "%s pointers must be aligned to 16 bytes", name);
  const int64_t unit = s->dtype == RESKV_BF16 ? 8 : 4, extent[3] = {s->batch, heads, n};
  const int64_t* st[2] = {&from->batch, &to->batch};
  for (int k = 0; k < 2; ++k) {
    for (int i = 0; i < 3; ++i) {
      if (extent[i] <= 1 && st[k][i] >= 0) continue;  // not used
      if (st[k][i] < 0 || st[k][i] % unit != 0 || st[k][i] > ((int64_t)1 << 48) / (extent[i] - 1))
        return fail(RESKV_ERR_INVALID_ARG, "%s stride %lld is not a multiple of 16 bytes >= 0 within 2^48 elements",
                    name, (long long)st[k][i]);
    }
  }
  // output rows apart from each other: by rising stride, each passes what the ones before it span
  int order[3] = {0, 1, 2};
  for (int i = 0; i < 2; ++i)
    for (int j = 0; j < 2 - i; ++j)
      if (st[1][order[j]] > st[1][order[j + 1]]) {
        const int x = order[j];
        order[j] = order[j + 1];
        order[j + 1] = x;
      }
  int64_t used = s->head_dim;
  for (int i = 0; i < 3; ++i) {
    const int o = order[i];
    if (extent[o] <= 1) continue;
    if (st[1][o] < used) return fail(RESKV_ERR_INVALID_ARG, "%s output rows overlap", name);
    used += (extent[o] - 1) * st[1][o];
  }
  bool same = in == out;
  for (int i = 0; i < 3; ++i) same = same && (extent[i] <= 1 || st[0][i] == st[1][i]);
  if (same) return RESKV_OK;
  return check_apart(s, row_set(s, heads, n, out, to), name, "output", row_set(s, heads, n, in, from), name, "input");
}

reskv_status_t reskv_rope(const reskv_shape_t* shape, const reskv_rope_t* rope, int32_t n_rows,
                          const int32_t* positions, const int32_t* n_tok, const void* q, const reskv_rows_t* q_at,
                          void* q_out, const reskv_rows_t* q_out_at, const void* k, const reskv_rows_t* k_at,
                          void* k_out, const reskv_rows_t* k_out_at, void* stream) {
  reskv_shape_t rows{};  // the shape without the cache's sizes, which a rotation does not use
  if (shape) {
    rows = *shape;
    rows.slot_cap = rows.res_cap = 1;
  }
  reskv_status_t st = check_shape(shape ? &rows : nullptr);
  if (st != RESKV_OK) return st;
  if (n_rows < 0) return fail(RESKV_ERR_INVALID_ARG, "n_rows %d must be >= 0", n_rows);
  if (n_rows == 0) return ok();  // tensors without elements may have no address
  if (shape->batch * (int64_t)n_rows > kMaxRows)
    return fail(RESKV_ERR_UNSUPPORTED, "%d sequences of %d rows are more than 2^26", shape->batch, n_rows);
  // head numbers stay within 32 bits, also those of the few heads past the last that a wave names
  if ((int64_t)shape->num_q_heads + shape->num_kv_heads > kMaxRows)
    return fail(RESKV_ERR_UNSUPPORTED, "%d query and %d KV heads are more than 2^26", shape->num_q_heads,
                shape->num_kv_heads);
  if (!rope || !positions) return fail(RESKV_ERR_INVALID_ARG, "rope or positions is NULL");
  if ((st = check_rope(shape, rope)) != RESKV_OK) return st;
  if (!q && !q_out && !k && !k_out) return fail(RESKV_ERR_INVALID_ARG, "neither queries nor keys are given");
  if ((st = check_rows(shape, "q", shape->num_q_heads, n_rows, q, q_at, q_out, q_out_at)) != RESKV_OK) return st;
  if ((st = check_rows(shape, "k", shape->num_kv_heads, n_rows, k, k_at, k_out, k_out_at)) != RESKV_OK) return st;
  if (q && k) {
    const RowSet q0 = row_set(shape, shape->num_q_heads, n_rows, q, q_at);
    const RowSet q1 = row_set(shape, shape->num_q_heads, n_rows, q_out, q_out_at);
    const RowSet k0 = row_set(shape, shape->num_kv_heads, n_rows, k, k_at);
    const RowSet k1 = row_set(shape, shape->num_kv_heads, n_rows, k_out, k_out_at);
    if ((st = check_apart(shape, q1, "q", "output", k0, "k", "input")) != RESKV_OK) return st;
    if ((st = check_apart(shape, k1, "k", "output", q0, "q", "input")) != RESKV_OK) return st;
    if ((st = check_apart(shape, q1, "q", "output", k1, "k", "output")) != RESKV_OK) return st;
  }
  hipError_t e = launch_rope(*shape, *rope, n_rows, positions, n_tok, q, q_at, q_out, q_out_at, k, k_at, k_out,
                             k_out_at, (hipStream_t)stream);
  if (e != hipSuccess) return fail(RESKV_ERR_HIP, "rope launch failed: %s", hipGetErrorString(e));
  return ok();
}

// Shapes of the 4-bit caches: sequences and heads are dimensions of the grids.
static reskv_status_t check_quant_shape(const reskv_shape_t* s) {
  reskv_status_t st = check_shape(s);
  if (st != RESKV_OK) return st;
  if (s->batch > 65535 || s->num_kv_heads > 32767)
    return fail(RESKV_ERR_UNSUPPORTED, "batch %d above 65535 or %d KV heads above 32767", s->batch, s->num_kv_heads);
  if (s->slot_cap > 1 << 29) return fail(RESKV_ERR_UNSUPPORTED, "slot_cap %d above 2^29", s->slot_cap);
  return RESKV_OK;
}

size_t reskv_quant_cache_size(const reskv_shape_t* shape) {
  return check_quant_shape(shape) == RESKV_OK ? quant_cache_bytes(*shape) : 0;
}

reskv_status_t reskv_pack_quant(const reskv_shape_t* shape, const void* kc, const void* vc, const int32_t* res_len,
                                const int32_t* main_len, void* cache, void* stream) {
  reskv_status_t st = check_quant_shape(shape);
  if (st != RESKV_OK) return st;
  if (!kc || !vc || !res_len || !main_len || !cache) return fail(RESKV_ERR_INVALID_ARG, "a required pointer is NULL");
  if (!aligned(kc) || !aligned(vc) || !aligned(cache))
    return fail(RESKV_ERR_INVALID_ARG, "kc, vc and cache must be aligned to 16 bytes");
  hipError_t e = launch_pack_quant(*shape, kc, vc, res_len, main_len, cache, (hipStream_t)stream);
  if (e != hipSuccess) return fail(RESKV_ERR_HIP, "pack launch failed: %s", hipGetErrorString(e));
  return ok();
}

reskv_status_t reskv_unpack_quant(const reskv_shape_t* shape, const void* cache, const int32_t* res_len,
                                  const int32_t* main_len, const int32_t* first_slot, int32_t n_rows, void* kc,
                                  void* vc, void* stream) {
  reskv_status_t st = check_quant_shape(shape);
  if (st != RESKV_OK) return st;
  if (n_rows < 0) return fail(RESKV_ERR_INVALID_ARG, "n_rows %d must be >= 0", n_rows);
  if (n_rows == 0) return ok();
  if (n_rows > kMaxRows) return fail(RESKV_ERR_UNSUPPORTED, "n_rows %d above 2^26", n_rows);
  if (!cache || !res_len || !main_len || !kc || !vc) return fail(RESKV_ERR_INVALID_ARG, "a required pointer is NULL");
  if (!aligned(kc) || !aligned(vc) || !aligned(cache))
    return fail(RESKV_ERR_INVALID_ARG, "kc, vc and cache must be aligned to 16 bytes");
  hipError_t e = launch_unpack_quant(*shape, cache, res_len, main_len, first_slot, n_rows, kc, vc,
                                     (hipStream_t)stream);
  if (e != hipSuccess) return fail(RESKV_ERR_HIP, "unpack launch failed: %s", hipGetErrorString(e));
  return ok();
}

// Rotation arguments of the calls where it is optional.
static reskv_status_t check_turn(const reskv_shape_t* shape, const reskv_rope_t* rope, const int32_t* positions) {
  if ((rope == nullptr) != (positions == nullptr))
    return fail(RESKV_ERR_INVALID_ARG, "rope and positions must both be given or both be NULL");
  return rope ? check_rope(shape, rope) : RESKV_OK;
}

reskv_status_t reskv_append_kv_quant(const reskv_shape_t* shape, const reskv_rope_t* rope, const int32_t* positions,
                                     int32_t n_new, const int32_t* n_tok, const void* k_new, const void* v_new,
                                     void* cache, const int32_t* res_len, int32_t* main_len, void* stream) {
  reskv_status_t st = check_quant_shape(shape);
  if (st != RESKV_OK) return st;
  if (n_new < 0) return fail(RESKV_ERR_INVALID_ARG, "n_new %d must be >= 0", n_new);
  if (n_new == 0) return ok();
  if (n_new > kMaxRows) return fail(RESKV_ERR_UNSUPPORTED, "n_new %d above 2^26", n_new);
  if (!k_new || !v_new || !cache || !res_len || !main_len)
    return fail(RESKV_ERR_INVALID_ARG, "a required pointer is NULL");
  if ((st = check_turn(shape, rope, positions)) != RESKV_OK) return st;
  if (!aligned(k_new) || !aligned(v_new) || !aligned(cache))
    return fail(RESKV_ERR_INVALID_ARG, "k_new, v_new and cache must be aligned to 16 bytes");
  hipError_t e = launch_append_quant(*shape, rope, positions, n_new, n_tok, k_new, v_new, cache, res_len, main_len,
                                     (hipStream_t)stream);
  if (e != hipSuccess) return fail(RESKV_ERR_HIP, "append launch failed: %s", hipGetErrorString(e));
  return ok();
}

size_t reskv_decode_quant_workspace_size(const reskv_shape_t* shape) {
  return check_quant_shape(shape) == RESKV_OK ? make_quant_decode_plan(*shape).bytes : 0;
}

int reskv_internal_quant_parts(const reskv_shape_t* shape) {
  return check_quant_shape(shape) == RESKV_OK ? make_quant_decode_plan(*shape).P : -1;
}

reskv_status_t reskv_decode_attn_quant(const reskv_shape_t* shape, const reskv_gate_t* gate, const reskv_rope_t* rope,
                                       const int32_t* positions, const void* q, void* cache, const float* logc,
                                       const int32_t* res_len, int32_t* main_len, const void* k_new,
                                       const void* v_new, float* out, float* dbg_lse_main, float* dbg_lse_res,
                                       float* dbg_gate, void* workspace, size_t workspace_bytes, void* stream) {
  reskv_status_t st = check_quant_shape(shape);
  if (st != RESKV_OK) return st;
  if ((st = check_gate(gate)) != RESKV_OK) return st;
  if (!q || !cache || !logc || !res_len || !main_len || !out)
    return fail(RESKV_ERR_INVALID_ARG, "a required pointer is NULL");
  if ((st = check_turn(shape, rope, positions)) != RESKV_OK) return st;
  if ((k_new == nullptr) != (v_new == nullptr))
    return fail(RESKV_ERR_INVALID_ARG, "k_new and v_new must both be given or both be NULL");
  if (!aligned(q) || !aligned(cache) || !aligned(k_new) || !aligned(v_new) || !aligned(workspace))
    return fail(RESKV_ERR_INVALID_ARG, "q, k_new, v_new, cache and workspace must be aligned to 16 bytes");
  const QuantDecodePlan plan = make_quant_decode_plan(*shape);
  if (!workspace || workspace_bytes < plan.bytes)
    return fail(RESKV_ERR_WORKSPACE, "decode needs %zu workspace bytes, got %zu", plan.bytes,
                workspace ? workspace_bytes : (size_t)0);
  hipError_t e = launch_decode_quant(*shape, *gate, plan, rope, positions, q, cache, logc, res_len, main_len, k_new,
                                     v_new, out, dbg_lse_main, dbg_lse_res, dbg_gate, workspace, (hipStream_t)stream);
  if (e != hipSuccess) return fail(RESKV_ERR_HIP, "decode launch failed: %s", hipGetErrorString(e));
  return ok();
}

static reskv_status_t check_build(const reskv_shape_t* shape, const reskv_build_params_t* p,
                                  const int32_t* seq_len, const int32_t* budget, const int32_t* res_count) {
  reskv_status_t st = check_shape(shape);
  if (st != RESKV_OK) return st;
  if (!p) return fail(RESKV_ERR_INVALID_ARG, "params is NULL");
  if (!seq_len || !budget || !res_count) return fail(RESKV_ERR_INVALID_ARG, "a host length array is NULL");
  if (p->max_seq_len < 1) return fail(RESKV_ERR_INVALID_ARG, "max_seq_len must be >= 1");
  if (p->obs_window < 1 || p->obs_window > p->max_seq_len)
    return fail(RESKV_ERR_INVALID_ARG, "obs_window %d outside [1, %d]", p->obs_window, p->max_seq_len);
  if (p->recent_window < 0) return fail(RESKV_ERR_INVALID_ARG, "recent_window must be >= 0");
  if (p->lloyd_iters < 1 || p->lloyd_iters > 64) return fail(RESKV_ERR_INVALID_ARG, "lloyd_iters %d outside [1, 64]", p->lloyd_iters);
  if (p->pool_kernel < 0 || p->pool_kernel > 31 || (p->pool_kernel > 0 && p->pool_kernel % 2 == 0))
    return fail(RESKV_ERR_INVALID_ARG, "pool_kernel %d must be 0 (= 5) or odd in [1, 31]", p->pool_kernel);
  if (p->fit_rows < 0 || p->fit_rows > p->obs_window)
    return fail(RESKV_ERR_INVALID_ARG, "fit_rows %d outside [0, obs_window=%d]", p->fit_rows, p->obs_window);
  const int rows = p->fit_rows > 0 ? p->fit_rows : p->obs_window;
  if ((long long)rows * (shape->num_q_heads / shape->num_kv_heads) > 1024)
    return fail(RESKV_ERR_UNSUPPORTED, "scoring rows per KV head (G*%d = %d) above 1024", rows,
                rows * (shape->num_q_heads / shape->num_kv_heads));
  if (shape->res_cap > 4096) return fail(RESKV_ERR_UNSUPPORTED, "res_cap %d above 4096", shape->res_cap);
  const int Hkv = shape->num_kv_heads;
  for (int b = 0; b < shape->batch; ++b) {
    const int s = seq_len[b];
    if (s < p->obs_window || s > p->max_seq_len)
      return fail(RESKV_ERR_INVALID_ARG, "seq_len[%d] = %d outside [obs_window=%d, max_seq_len=%d]", b, s, p->obs_window, p->max_seq_len);
    if (budget[b] < 1 || budget[b] > shape->slot_cap)
      return fail(RESKV_ERR_INVALID_ARG, "budget[%d] = %d outside [1, slot_cap=%d]", b, budget[b], shape->slot_cap);
    for (int h = 0; h < Hkv; ++h) {
      const int r = res_count[b * Hkv + h];
      if (r < 0 || r >= budget[b] || r > shape->res_cap)
        return fail(RESKV_ERR_INVALID_ARG, "res_count[%d] = %d must satisfy 0 <= r < budget (%d) and r <= res_cap (%d)",
                    b * Hkv + h, r, budget[b], shape->res_cap);
      const int m = budget[b] - r;
      const int main_len = s <= m ? s : m;
      if (r + main_len > shape->slot_cap)
        return fail(RESKV_ERR_INVALID_ARG, "r + main slots (%d) exceed slot_cap (%d)", r + main_len, shape->slot_cap);
    }
  }
  return RESKV_OK;
}

size_t reskv_build_workspace_size(const reskv_shape_t* shape, const reskv_build_params_t* params,
                                  const int32_t* seq_len_host, const int32_t* budget_host,
                                  const int32_t* res_count_host) {
  if (check_build(shape, params, seq_len_host, budget_host, res_count_host) != RESKV_OK) return 0;
  BuildPlan plan;
  if (!make_build_plan(*shape, *params, seq_len_host, budget_host, res_count_host, &plan)) return 0;
  return plan.bytes;
}

int reskv_internal_build_rules(const reskv_shape_t* shape, const reskv_build_params_t* params,
                               const int32_t* seq_len, const int32_t* budget, const int32_t* res_count,
                               BuildRules* rules) {
  if (check_build(shape, params, seq_len, budget, res_count) != RESKV_OK) return 1;
  BuildPlan pl;
  if (!make_build_plan(*shape, *params, seq_len, budget, res_count, &pl)) return 1;
  *rules = BuildRules{pl.deal_rows, pl.KG, pl.NSEL, pl.count_sel};
  return 0;
}

reskv_status_t reskv_build_cache(const reskv_shape_t* shape, const reskv_build_params_t* params, const void* k,
                                 const void* v, const int32_t* seq_len_host, const void* q_obs,
                                 const int32_t* budget_host, const int32_t* res_count_host, void* kc, void* vc,
                                 float* logc, int32_t* main_idx, int32_t* res_len, int32_t* main_len,
                                 float* dbg_scores, int32_t* dbg_assign, float* dbg_centers, void* workspace,
                                 size_t workspace_bytes, void* stream) {
  reskv_status_t st = check_build(shape, params, seq_len_host, budget_host, res_count_host);
  if (st != RESKV_OK) return st;
  if (!k || !v || !q_obs || !kc || !vc || !logc || !main_idx || !res_len || !main_len)
    return fail(RESKV_ERR_INVALID_ARG, "a required pointer is NULL");
  BuildPlan plan;
  if (!make_build_plan(*shape, *params, seq_len_host, budget_host, res_count_host, &plan))
    return fail(RESKV_ERR_UNSUPPORTED, "construction plan could not be formed for these sizes");
  if (!workspace || workspace_bytes < plan.bytes)
    return fail(RESKV_ERR_WORKSPACE, "build needs %zu workspace bytes, got %zu", plan.bytes,
                workspace ? workspace_bytes : (size_t)0);
  hipError_t e = launch_build(*shape, *params, plan, k, v, seq_len_host, q_obs, budget_host, res_count_host, kc,
                              vc, logc, main_idx, res_len, main_len, dbg_scores, dbg_assign, dbg_centers,
                              workspace, (hipStream_t)stream);
  if (e != hipSuccess) return fail(RESKV_ERR_HIP, "build launch failed: %s", hipGetErrorString(e));
  return ok();
}

static reskv_status_t check_adakv(const reskv_shape_t* shape, double safeguard, int32_t decode_reserve,
                                  const int32_t* budget) {
  if (!(safeguard >= 0.0 && safeguard <= 1.0))
    return fail(RESKV_ERR_INVALID_ARG, "safeguard %g outside [0, 1]", safeguard);
  if (decode_reserve < 0) return fail(RESKV_ERR_INVALID_ARG, "decode_reserve %d must be >= 0", decode_reserve);
  for (int b = 0; b < shape->batch; ++b)
    if ((long long)budget[b] + decode_reserve > shape->slot_cap)
      return fail(RESKV_ERR_INVALID_ARG, "budget[%d] + decode_reserve = %lld exceeds slot_cap (%d)", b,
                  (long long)budget[b] + decode_reserve, shape->slot_cap);
  if (shape->num_kv_heads > kAdaMaxHeads)
    return fail(RESKV_ERR_UNSUPPORTED, "cross-head allocation over %d KV heads (at most %d)", shape->num_kv_heads,
                kAdaMaxHeads);
  return RESKV_OK;
}

size_t reskv_build_adakv_workspace_size(const reskv_shape_t* shape, const reskv_build_params_t* params,
                                        double safeguard, int32_t decode_reserve, const int32_t* seq_len_host,
                                        const int32_t* budget_host, const int32_t* res_count_host) {
  if (check_build(shape, params, seq_len_host, budget_host, res_count_host) != RESKV_OK) return 0;
  if (check_adakv(shape, safeguard, decode_reserve, budget_host) != RESKV_OK) return 0;
  BuildPlan plan;
  if (!make_build_plan_adakv(*shape, *params, safeguard, decode_reserve, seq_len_host, budget_host, res_count_host,
                             &plan))
    return 0;
  return plan.bytes;
}

reskv_status_t reskv_build_cache_adakv(const reskv_shape_t* shape, const reskv_build_params_t* params,
                                       double safeguard, int32_t decode_reserve, const void* k, const void* v,
                                       const int32_t* seq_len_host, const void* q_obs, const int32_t* budget_host,
                                       const int32_t* res_count_host, void* kc, void* vc, float* logc,
                                       int32_t* main_idx, int32_t* res_len, int32_t* main_len, float* dbg_scores,
                                       int32_t* dbg_assign, float* dbg_centers, void* workspace,
                                       size_t workspace_bytes, void* stream) {
  reskv_status_t st = check_build(shape, params, seq_len_host, budget_host, res_count_host);
  if (st != RESKV_OK) return st;
  if ((st = check_adakv(shape, safeguard, decode_reserve, budget_host)) != RESKV_OK) return st;
  if (!k || !v || !q_obs || !kc || !vc || !logc || !main_idx || !res_len || !main_len)
    return fail(RESKV_ERR_INVALID_ARG, "a required pointer is NULL");
  BuildPlan plan;
  if (!make_build_plan_adakv(*shape, *params, safeguard, decode_reserve, seq_len_host, budget_host, res_count_host,
                             &plan))
    return fail(RESKV_ERR_UNSUPPORTED, "construction plan could not be formed for these sizes");
  if (!workspace || workspace_bytes < plan.bytes)
    return fail(RESKV_ERR_WORKSPACE, "build needs %zu workspace bytes, got %zu", plan.bytes,
                workspace ? workspace_bytes : (size_t)0);
  hipError_t e = launch_build_adakv(*shape, *params, safeguard, decode_reserve, plan, k, v, seq_len_host, q_obs,
                                    budget_host, res_count_host, kc, vc, logc, main_idx, res_len, main_len,
                                    dbg_scores, dbg_assign, dbg_centers, workspace, (hipStream_t)stream);
  if (e != hipSuccess) return fail(RESKV_ERR_HIP, "build launch failed: %s", hipGetErrorString(e));
  return ok();
}

// Proxy arguments, then every candidate count through the construction
// checks with the fit rows in place.
static reskv_status_t check_proxy(const reskv_shape_t* shape, const reskv_build_params_t* p,
                                  const reskv_proxy_params_t* x, const int32_t* seq_len, const int32_t* budget,
                                  reskv_build_params_t* pf) {
  reskv_status_t st = check_shape(shape);
  if (st != RESKV_OK) return st;
  if (!p || !x) return fail(RESKV_ERR_INVALID_ARG, "params or proxy params is NULL");
  if (!seq_len || !budget) return fail(RESKV_ERR_INVALID_ARG, "a host length array is NULL");
  if (!x->grid_host) return fail(RESKV_ERR_INVALID_ARG, "grid_host is NULL");
  if (x->n_grid < 1 || x->n_grid > kProxyMaxGrid)
    return fail(RESKV_ERR_INVALID_ARG, "n_grid %d outside [1, %d]", x->n_grid, kProxyMaxGrid);
  bool has_zero = false;
  for (int c = 0; c < x->n_grid; ++c) {
    const double f = x->grid_host[c];
    if (!(f >= 0.0 && f < 1.0)) return fail(RESKV_ERR_INVALID_ARG, "grid[%d] = %g outside [0, 1)", c, f);
    has_zero |= f == 0.0;
  }
  if (!has_zero) return fail(RESKV_ERR_INVALID_ARG, "the grid must contain the fraction 0 (the pure-main cache)");
  if (x->val_rows < 1 || x->val_rows >= p->obs_window)
    return fail(RESKV_ERR_INVALID_ARG, "val_rows %d outside [1, obs_window - 1 = %d]", x->val_rows,
                p->obs_window - 1);
  if (p->fit_rows != 0 && p->fit_rows != p->obs_window - x->val_rows)
    return fail(RESKV_ERR_INVALID_ARG, "fit_rows %d must be 0 or obs_window - val_rows = %d", p->fit_rows,
                p->obs_window - x->val_rows);
  if (!(x->delta >= 0.f && x->delta <= 1.f)) return fail(RESKV_ERR_INVALID_ARG, "delta %g outside [0, 1]", x->delta);
  *pf = *p;
  pf->fit_rows = p->obs_window - x->val_rows;
  const int Hkv = shape->num_kv_heads;
  std::vector<int32_t> counts((size_t)shape->batch * Hkv);
  for (int c = 0; c < x->n_grid; ++c) {
    for (int b = 0; b < shape->batch; ++b) {
      const double r = floor(x->grid_host[c] * (double)budget[b] + 0.5);
      if (budget[b] >= 1 && r >= budget[b])
        return fail(RESKV_ERR_INVALID_ARG, "grid[%d] = %g gives r = %.0f >= budget[%d] = %d", c, x->grid_host[c],
                    r, b, budget[b]);
      for (int h = 0; h < Hkv; ++h) counts[(size_t)b * Hkv + h] = (int32_t)r;
    }
    if ((st = check_build(shape, pf, seq_len, budget, counts.data())) != RESKV_OK) return st;
  }
  return RESKV_OK;
}

size_t reskv_build_proxy_workspace_size(const reskv_shape_t* shape, const reskv_build_params_t* params,
                                        const reskv_proxy_params_t* proxy, const int32_t* seq_len_host,
                                        const int32_t* budget_host) {
  reskv_build_params_t pf;
  if (check_proxy(shape, params, proxy, seq_len_host, budget_host, &pf) != RESKV_OK) return 0;
  ProxyPlan plan;
  if (!make_proxy_plan(*shape, pf, *proxy, seq_len_host, budget_host, true, &plan)) return 0;
  return plan.bytes;
}

int reskv_internal_proxy_rules(const reskv_shape_t* shape, const reskv_build_params_t* params,
                               const reskv_proxy_params_t* proxy, const int32_t* seq_len, const int32_t* budget,
                               ProxyRules* rules) {
  reskv_build_params_t pf;
  if (check_proxy(shape, params, proxy, seq_len, budget, &pf) != RESKV_OK) return 1;
  ProxyPlan all, least;
  if (!make_proxy_plan(*shape, pf, *proxy, seq_len, budget, true, &all) ||
      !make_proxy_plan(*shape, pf, *proxy, seq_len, budget, false, &least))
    return 1;
  *rules = ProxyRules{all.build.NC, least.bytes};
  return 0;
}

reskv_status_t reskv_build_cache_proxy(const reskv_shape_t* shape, const reskv_build_params_t* params,
                                       const reskv_proxy_params_t* proxy, const reskv_gate_t* gate, const void* k,
                                       const void* v, const int32_t* seq_len_host, const void* q_obs,
                                       const int32_t* budget_host, void* kc, void* vc, float* logc,
                                       int32_t* main_idx, int32_t* res_len, int32_t* main_len, float* val_loss,
                                       void* workspace, size_t workspace_bytes, void* stream) {
  reskv_build_params_t pf;
  reskv_status_t st = check_proxy(shape, params, proxy, seq_len_host, budget_host, &pf);
  if (st != RESKV_OK) return st;
  if ((st = check_gate(gate)) != RESKV_OK) return st;
  if (!k || !v || !q_obs || !kc || !vc || !logc || !main_idx || !res_len || !main_len)
    return fail(RESKV_ERR_INVALID_ARG, "a required pointer is NULL");
  ProxyPlan plan;
  // a workspace too small for all candidates at once may still hold one at a time
  if (!make_proxy_plan(*shape, pf, *proxy, seq_len_host, budget_host, true, &plan) ||
      (plan.build.NC > 1 && workspace_bytes < plan.bytes &&
       !make_proxy_plan(*shape, pf, *proxy, seq_len_host, budget_host, false, &plan)))
    return fail(RESKV_ERR_UNSUPPORTED, "proxy plan could not be formed for these sizes");
  if (!workspace || workspace_bytes < plan.bytes)
    return fail(RESKV_ERR_WORKSPACE, "proxy build needs %zu workspace bytes, got %zu", plan.bytes,
                workspace ? workspace_bytes : (size_t)0);
  hipError_t e = launch_build_proxy(*shape, pf, *proxy, *gate, plan, k, v, seq_len_host, q_obs, budget_host, kc, vc,
                                    logc, main_idx, res_len, main_len, val_loss, workspace, (hipStream_t)stream);
  if (e != hipSuccess) return fail(RESKV_ERR_HIP, "proxy build launch failed: %s", hipGetErrorString(e));
  return ok();
}

}  // extern "C"
