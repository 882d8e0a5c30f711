"""Python binding of the ResKV C ABI (include/reskv.h).

Argument marshalling only: every step of construction and decode runs in the
HIP kernels of libreskv.so. Torch tensors supply device memory and the
current stream; this module passes their raw pointers through ctypes. If the
library is missing or fails to load, every entry point raises.
"""

import ctypes
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libreskv.so")

RESKV_F32 = 0
RESKV_BF16 = 1

STATUS = {0: "ok", 1: "invalid argument", 2: "unsupported configuration",
          3: "workspace missing or too small", 4: "HIP runtime error"}


class ReskvError(RuntimeError):
    def __init__(self, status, detail):
        super().__init__(f"{STATUS.get(status, status)}: {detail}")
        self.status = status


class Shape(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("num_q_heads", ctypes.c_int32),
                ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("slot_cap", ctypes.c_int32),
                ("res_cap", ctypes.c_int32)]


class BuildParams(ctypes.Structure):
    _fields_ = [("max_seq_len", ctypes.c_int32), ("obs_window", ctypes.c_int32),
                ("recent_window", ctypes.c_int32), ("lloyd_iters", ctypes.c_int32),
                ("fit_rows", ctypes.c_int32), ("pool_kernel", ctypes.c_int32)]


class ProxyParams(ctypes.Structure):
    _fields_ = [("grid_host", ctypes.POINTER(ctypes.c_double)), ("n_grid", ctypes.c_int32),
                ("val_rows", ctypes.c_int32), ("delta", ctypes.c_float)]


class RopeParams(ctypes.Structure):
    _fields_ = [("rot_dim", ctypes.c_int32), ("layout", ctypes.c_int32), ("scaling", ctypes.c_int32),
                ("theta", ctypes.c_double), ("factor", ctypes.c_double), ("original_len", ctypes.c_double),
                ("low_freq_factor", ctypes.c_double), ("high_freq_factor", ctypes.c_double),
                ("beta_fast", ctypes.c_double), ("beta_slow", ctypes.c_double), ("attn_scale", ctypes.c_double)]


class Rope(ctypes.Structure):
    _fields_ = [("rot_dim", ctypes.c_int32), ("layout", ctypes.c_int32), ("attn_scale", ctypes.c_double),
                ("freq", ctypes.c_void_p)]


class Rows(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int64), ("head", ctypes.c_int64), ("row", ctypes.c_int64)]


class Gate(ctypes.Structure):
    _fields_ = [("tau", ctypes.c_void_p), ("tau_scalar", ctypes.c_float),
                ("alpha", ctypes.c_float), ("g_min", ctypes.c_float), ("beta", ctypes.c_float)]


_lib = None

_P = ctypes.c_void_p
_SIG = {
    "reskv_build_cache": (ctypes.c_int, [ctypes.POINTER(Shape), ctypes.POINTER(BuildParams), _P, _P, _P, _P,
                                         _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, ctypes.c_size_t, _P]),
    "reskv_build_workspace_size": (ctypes.c_size_t, [ctypes.POINTER(Shape), ctypes.POINTER(BuildParams),
                                                     _P, _P, _P]),
    "reskv_build_cache_adakv": (ctypes.c_int, [ctypes.POINTER(Shape), ctypes.POINTER(BuildParams), ctypes.c_double,
                                               ctypes.c_int32, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P,
                                               _P, _P, _P, ctypes.c_size_t, _P]),
    "reskv_build_adakv_workspace_size": (ctypes.c_size_t, [ctypes.POINTER(Shape), ctypes.POINTER(BuildParams),
                                                           ctypes.c_double, ctypes.c_int32, _P, _P, _P]),
    "reskv_build_cache_proxy": (ctypes.c_int, [ctypes.POINTER(Shape), ctypes.POINTER(BuildParams),
                                               ctypes.POINTER(ProxyParams), ctypes.POINTER(Gate), _P, _P, _P, _P,
                                               _P, _P, _P, _P, _P, _P, _P, _P, _P, ctypes.c_size_t, _P]),
    "reskv_build_proxy_workspace_size": (ctypes.c_size_t, [ctypes.POINTER(Shape), ctypes.POINTER(BuildParams),
                                                           ctypes.POINTER(ProxyParams), _P, _P]),
    "reskv_decode_attn": (ctypes.c_int, [ctypes.POINTER(Shape), ctypes.POINTER(Gate), _P, _P, _P, _P, _P, _P,
                                         _P, _P, _P, _P, _P, _P, _P, ctypes.c_size_t, _P]),
    "reskv_decode_workspace_size": (ctypes.c_size_t, [ctypes.POINTER(Shape)]),
    "reskv_decode_attn_ragged": (ctypes.c_int, [ctypes.POINTER(Shape), ctypes.POINTER(Gate), _P, _P, _P, _P, _P,
                                                _P, _P, _P, _P, _P, _P, _P, _P, ctypes.c_size_t, _P]),
    "reskv_decode_ragged_workspace_size": (ctypes.c_size_t, [ctypes.POINTER(Shape)]),
    "reskv_decode_attn_static": (ctypes.c_int, [ctypes.POINTER(Shape), ctypes.POINTER(Gate), _P, _P, _P, _P, _P,
                                                _P, _P, _P, _P, _P, _P, _P, _P]),
    "reskv_decode_branches": (ctypes.c_int, [ctypes.POINTER(Shape), ctypes.POINTER(Gate), _P, _P, _P, _P, _P, _P,
                                             _P, _P, _P, _P, _P, _P, ctypes.c_size_t, _P]),
    "reskv_merge_branches": (ctypes.c_int, [ctypes.POINTER(Shape), ctypes.c_int32, _P, _P, _P, _P, _P, _P, _P]),
    "reskv_append_kv": (ctypes.c_int, [ctypes.POINTER(Shape), _P, _P, _P, _P, _P, _P, _P]),
    "reskv_rope_init": (ctypes.c_int, [ctypes.POINTER(RopeParams), ctypes.POINTER(Rope), _P]),
    "reskv_rope": (ctypes.c_int, [ctypes.POINTER(Shape), ctypes.POINTER(Rope), ctypes.c_int32, _P, _P, _P,
                                  ctypes.POINTER(Rows), _P, ctypes.POINTER(Rows), _P, ctypes.POINTER(Rows), _P,
                                  ctypes.POINTER(Rows), _P]),
    "reskv_quant_cache_size": (ctypes.c_size_t, [ctypes.POINTER(Shape)]),
    "reskv_pack_quant": (ctypes.c_int, [ctypes.POINTER(Shape), _P, _P, _P, _P, _P, _P]),
    "reskv_unpack_quant": (ctypes.c_int, [ctypes.POINTER(Shape), _P, _P, _P, _P, ctypes.c_int32, _P, _P, _P]),
    "reskv_append_kv_quant": (ctypes.c_int, [ctypes.POINTER(Shape), ctypes.POINTER(Rope), _P, ctypes.c_int32, _P, _P,
                                             _P, _P, _P, _P, _P]),
    "reskv_decode_attn_quant": (ctypes.c_int, [ctypes.POINTER(Shape), ctypes.POINTER(Gate), ctypes.POINTER(Rope), _P,
                                               _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, ctypes.c_size_t, _P]),
    "reskv_decode_quant_workspace_size": (ctypes.c_size_t, [ctypes.POINTER(Shape)]),
    "reskv_status_string": (ctypes.c_char_p, [ctypes.c_int]),
    "reskv_last_error": (ctypes.c_char_p, []),
}


def lib():
    """The loaded library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python -m paper_2607_29591_amd.build_lib` (or __graft_entry__.build())")
        L = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIG.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


def _check(status):
    if status != 0:
        raise ReskvError(status, lib().reskv_last_error().decode())


def _ptr(t):
    """Raw device pointer of a contiguous tensor (None -> NULL)."""
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("tensors passed to the ResKV library must be contiguous")
    return t.data_ptr()


_raw_stream = None


def _stream(stream):
    """HIP stream handle; None is the current stream of the current device."""
    if stream is not None:
        return stream.cuda_stream
    global _raw_stream
    if _raw_stream is None:
        import torch
        # the handle itself: building torch's Stream object for it took 2.7 us
        # of a 7 us call, this 0.3 us
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        dev = torch.cuda.current_device
        _raw_stream = (lambda: raw(dev())) if raw else (lambda: torch.cuda.current_stream().cuda_stream)
    return _raw_stream()


def make_shape(batch, num_q_heads, num_kv_heads, head_dim, dtype, slot_cap, res_cap):
    dt = {"f32": RESKV_F32, "bf16": RESKV_BF16}.get(dtype, dtype)
    return Shape(batch, num_q_heads, num_kv_heads, head_dim, dt, slot_cap, res_cap)


def make_gate(tau=None, tau_scalar=0.25, alpha=12.0, g_min=0.0, beta=1.0):
    g = Gate(_ptr(tau), tau_scalar, alpha, g_min, beta)
    g.tau_tensor = tau  # keep the thresholds alive with the struct
    return g


def _host_i32(x):
    a = np.ascontiguousarray(np.asarray(x, dtype=np.int32).reshape(-1))
    return a, a.ctypes.data_as(ctypes.c_void_p)


def reskv_build_workspace_size(shape, params, seq_len, budget, res_count):
    sl, slp = _host_i32(seq_len)
    bu, bup = _host_i32(budget)
    rc, rcp = _host_i32(res_count)
    return lib().reskv_build_workspace_size(ctypes.byref(shape), ctypes.byref(params), slp, bup, rcp)


def reskv_build_cache(shape, params, k, v, seq_len, q_obs, budget, res_count, kc, vc, logc, main_idx,
                      res_len, main_len, workspace, dbg_scores=None, dbg_assign=None, dbg_centers=None,
                      stream=None):
    sl, slp = _host_i32(seq_len)
    bu, bup = _host_i32(budget)
    rc, rcp = _host_i32(res_count)
    _check(lib().reskv_build_cache(ctypes.byref(shape), ctypes.byref(params), _ptr(k), _ptr(v), slp,
                                   _ptr(q_obs), bup, rcp, _ptr(kc), _ptr(vc), _ptr(logc), _ptr(main_idx),
                                   _ptr(res_len), _ptr(main_len), _ptr(dbg_scores), _ptr(dbg_assign),
                                   _ptr(dbg_centers), _ptr(workspace), workspace.numel() * workspace.element_size(),
                                   _stream(stream)))


def reskv_build_adakv_workspace_size(shape, params, safeguard, decode_reserve, seq_len, budget, res_count):
    sl, slp = _host_i32(seq_len)
    bu, bup = _host_i32(budget)
    rc, rcp = _host_i32(res_count)
    return lib().reskv_build_adakv_workspace_size(ctypes.byref(shape), ctypes.byref(params), float(safeguard),
                                                  int(decode_reserve), slp, bup, rcp)


def reskv_build_cache_adakv(shape, params, safeguard, decode_reserve, k, v, seq_len, q_obs, budget, res_count, kc,
                            vc, logc, main_idx, res_len, main_len, workspace, dbg_scores=None, dbg_assign=None,
                            dbg_centers=None, stream=None):
    sl, slp = _host_i32(seq_len)
    bu, bup = _host_i32(budget)
    rc, rcp = _host_i32(res_count)
    _check(lib().reskv_build_cache_adakv(ctypes.byref(shape), ctypes.byref(params), float(safeguard),
                                         int(decode_reserve), _ptr(k), _ptr(v), slp, _ptr(q_obs), bup, rcp, _ptr(kc),
                                         _ptr(vc), _ptr(logc), _ptr(main_idx), _ptr(res_len), _ptr(main_len),
                                         _ptr(dbg_scores), _ptr(dbg_assign), _ptr(dbg_centers), _ptr(workspace),
                                         workspace.numel() * workspace.element_size(), _stream(stream)))


def make_proxy(grid=(0.0, 0.05, 0.10, 0.15, 0.20), val_rows=8, delta=0.01):
    """Proxy parameters; the grid array lives on the returned object."""
    g = (ctypes.c_double * len(grid))(*[float(f) for f in grid])
    x = ProxyParams(ctypes.cast(g, ctypes.POINTER(ctypes.c_double)), len(grid), val_rows, delta)
    x._grid = g  # keep the host array alive with the struct
    return x


def reskv_build_proxy_workspace_size(shape, params, proxy, seq_len, budget):
    sl, slp = _host_i32(seq_len)
    bu, bup = _host_i32(budget)
    return lib().reskv_build_proxy_workspace_size(ctypes.byref(shape), ctypes.byref(params), ctypes.byref(proxy),
                                                  slp, bup)


def reskv_build_cache_proxy(shape, params, proxy, gate, k, v, seq_len, q_obs, budget, kc, vc, logc, main_idx,
                            res_len, main_len, workspace, val_loss=None, stream=None):
    sl, slp = _host_i32(seq_len)
    bu, bup = _host_i32(budget)
    _check(lib().reskv_build_cache_proxy(ctypes.byref(shape), ctypes.byref(params), ctypes.byref(proxy),
                                         ctypes.byref(gate), _ptr(k), _ptr(v), slp, _ptr(q_obs), bup, _ptr(kc),
                                         _ptr(vc), _ptr(logc), _ptr(main_idx), _ptr(res_len), _ptr(main_len),
                                         _ptr(val_loss), _ptr(workspace),
                                         workspace.numel() * workspace.element_size(), _stream(stream)))


def reskv_decode_workspace_size(shape):
    return lib().reskv_decode_workspace_size(ctypes.byref(shape))


def decode_kernels(shape, entry="attn"):
    """Names of the kernels a decode call of these sizes takes; None where it is refused.
    entry: "attn", "branches", or "ragged" (with the workspace its size query names)."""
    fn = lib().reskv_internal_decode_kernels
    fn.restype, fn.argtypes = ctypes.c_int, [ctypes.POINTER(Shape), ctypes.c_int]
    return {0: "decode_head", 1: "decode_split + decode_combine", 2: "decode_ragged + decode_ragged_combine"}.get(
        fn(ctypes.byref(shape), ("attn", "branches", "ragged").index(entry)))


def reskv_decode_attn(shape, gate, q, kc, vc, logc, res_len, main_len, out, workspace,
                      dbg_lse_main=None, dbg_lse_res=None, dbg_gate=None, k_new=None, v_new=None, stream=None):
    _check(lib().reskv_decode_attn(ctypes.byref(shape), ctypes.byref(gate), _ptr(q), _ptr(kc), _ptr(vc),
                                   _ptr(logc), _ptr(res_len), _ptr(main_len), _ptr(k_new), _ptr(v_new), _ptr(out),
                                   _ptr(dbg_lse_main), _ptr(dbg_lse_res), _ptr(dbg_gate), _ptr(workspace),
                                   workspace.numel() * workspace.element_size(), _stream(stream)))


def reskv_decode_ragged_workspace_size(shape):
    return lib().reskv_decode_ragged_workspace_size(ctypes.byref(shape))


def reskv_decode_attn_ragged(shape, gate, q, kc, vc, logc, res_len, main_len, out, workspace, dbg_lse_main=None,
                             dbg_lse_res=None, dbg_gate=None, k_new=None, v_new=None, stream=None):
    _check(lib().reskv_decode_attn_ragged(ctypes.byref(shape), ctypes.byref(gate), _ptr(q), _ptr(kc), _ptr(vc),
                                          _ptr(logc), _ptr(res_len), _ptr(main_len), _ptr(k_new), _ptr(v_new),
                                          _ptr(out), _ptr(dbg_lse_main), _ptr(dbg_lse_res), _ptr(dbg_gate),
                                          _ptr(workspace), workspace.numel() * workspace.element_size(),
                                          _stream(stream)))


def prepare_decode_attn_ragged(shape, gate, q, kc, vc, logc, res_len, main_len, out, workspace,
                               dbg_lse_main=None, dbg_lse_res=None, dbg_gate=None, k_new=None, v_new=None,
                               stream=None):
    """As prepare_decode_attn, for reskv_decode_attn_ragged."""
    fn = lib().reskv_decode_attn_ragged
    args = (ctypes.byref(shape), ctypes.byref(gate), _ptr(q), _ptr(kc), _ptr(vc), _ptr(logc), _ptr(res_len),
            _ptr(main_len), _ptr(k_new), _ptr(v_new), _ptr(out), _ptr(dbg_lse_main), _ptr(dbg_lse_res),
            _ptr(dbg_gate), _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream))
    keep = (shape, gate)

    def call():
        status = fn(*args)
        if status != 0:
            _check(status)

    call.keep = keep
    return call


def reskv_decode_attn_static(shape, gate, q, kc, vc, logc, res_len, main_len, out, dbg_lse_main=None,
                             dbg_lse_res=None, dbg_gate=None, k_new=None, v_new=None, stream=None):
    _check(lib().reskv_decode_attn_static(ctypes.byref(shape), ctypes.byref(gate), _ptr(q), _ptr(kc), _ptr(vc),
                                          _ptr(logc), _ptr(res_len), _ptr(main_len), _ptr(k_new), _ptr(v_new),
                                          _ptr(out), _ptr(dbg_lse_main), _ptr(dbg_lse_res), _ptr(dbg_gate),
                                          _stream(stream)))


def prepare_decode_attn(shape, gate, q, kc, vc, logc, res_len, main_len, out, workspace,
                        dbg_lse_main=None, dbg_lse_res=None, dbg_gate=None, k_new=None, v_new=None, stream=None):
    """Marshal the arguments of one reskv_decode_attn call once and return a
    function that issues it (for loops that launch the same calls many
    times). The caller keeps the tensors alive and unchanged in place."""
    fn = lib().reskv_decode_attn
    args = (ctypes.byref(shape), ctypes.byref(gate), _ptr(q), _ptr(kc), _ptr(vc), _ptr(logc), _ptr(res_len),
            _ptr(main_len), _ptr(k_new), _ptr(v_new), _ptr(out), _ptr(dbg_lse_main), _ptr(dbg_lse_res),
            _ptr(dbg_gate), _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream))
    keep = (shape, gate)

    def call():
        status = fn(*args)
        if status != 0:
            _check(status)

    call.keep = keep
    return call


RESKV_MERGE_SHARED, RESKV_MERGE_SEPARATE = 0, 1


def reskv_decode_branches(shape, gate, q, kc, vc, logc, res_len, main_len, out_main, lse_main, out_res, lse_res,
                          gate_out, workspace, stream=None):
    _check(lib().reskv_decode_branches(ctypes.byref(shape), ctypes.byref(gate), _ptr(q), _ptr(kc), _ptr(vc),
                                       _ptr(logc), _ptr(res_len), _ptr(main_len), _ptr(out_main), _ptr(lse_main),
                                       _ptr(out_res), _ptr(lse_res), _ptr(gate_out), _ptr(workspace),
                                       workspace.numel() * workspace.element_size(), _stream(stream)))


def reskv_merge_branches(shape, mode, out_main, lse_main, out_res, lse_res, gate, out, stream=None):
    _check(lib().reskv_merge_branches(ctypes.byref(shape), int(mode), _ptr(out_main), _ptr(lse_main), _ptr(out_res),
                                      _ptr(lse_res), _ptr(gate), _ptr(out), _stream(stream)))


def reskv_append_kv(shape, k_new, v_new, kc, vc, res_len, main_len, stream=None):
    _check(lib().reskv_append_kv(ctypes.byref(shape), _ptr(k_new), _ptr(v_new), _ptr(kc), _ptr(vc),
                                 _ptr(res_len), _ptr(main_len), _stream(stream)))


# ------------------------------------- rotary positions, caches in 4 bits

ROPE_LAYOUTS = {"half": 0, "interleaved": 1}
ROPE_SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "llama3": 3, "yarn": 4}


def make_rope(rot_dim, layout="half", theta=10000.0, scaling="none", factor=1.0, original_len=0.0,
              low_freq_factor=1.0, high_freq_factor=4.0, beta_fast=32.0, beta_slow=1.0, attn_scale=0.0):
    """Rotation plan (reskv_rope_init); attn_scale 0 takes the scaling's own factor. The frequencies are on the plan
    as the array freq_host and, where there is a GPU, in a tensor of the current one: make a plan outside of captures."""
    import torch
    p = RopeParams(rot_dim, ROPE_LAYOUTS.get(layout, layout), ROPE_SCALINGS.get(scaling, scaling), theta, factor,
                   original_len, low_freq_factor, high_freq_factor, beta_fast, beta_slow, attn_scale)
    rope, freq = Rope(), np.zeros(64)
    _check(lib().reskv_rope_init(ctypes.byref(p), ctypes.byref(rope), freq.ctypes.data))
    rope.freq_host = freq[:rot_dim // 2].copy()
    if torch.cuda.is_available():
        rope.table = torch.from_numpy(rope.freq_host).to("cuda")
        rope.freq = rope.table.data_ptr()
    return rope


def _rope(rope):
    """Reference to a plan whose frequencies are on the current GPU (None -> NULL)."""
    if rope is None:
        return None
    table = getattr(rope, "table", None)
    if table is not None:
        _tensor("the plan's frequencies", table, table.dtype, rope.rot_dim // 2)
    return ctypes.byref(rope)


def _tensor(name, t, dtype, count, contiguous=True):
    """Pointer of a tensor of the current GPU with `count` elements of `dtype` (None -> NULL)."""
    import torch
    if t is None:
        return None
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if t.numel() != count:
        raise ValueError(f"{name} must have {count} elements, got {tuple(t.shape)}")
    if t.device.type != "cuda" or t.device.index != torch.cuda.current_device():
        raise ValueError(f"{name} must be on the current GPU, got {t.device}")
    if contiguous and not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _order(name, t, *size):
    """Refuse a tensor of as many dimensions as `size` whose dimensions are not these: elements alone do not tell
    heads from tokens. One with fewer dimensions (a single token, a flat buffer) is told by its elements."""
    if t is not None and t.dim() == len(size) and tuple(t.shape) != size:
        raise ValueError(f"{name} must be {list(size)}, got {list(t.shape)}")


def _dtype(shape):
    import torch
    return torch.bfloat16 if shape.dtype == RESKV_BF16 else torch.float32


def _prepared(fn, args, keep):
    """Function that issues fn(*args); `keep` lives as long as it does."""
    def call():
        status = fn(*args)
        if status != 0:
            _check(status)

    call.keep = keep
    return call


def prepare_rope(shape, rope, positions, q=None, q_out=None, k=None, k_out=None, n_tok=None, stream=None):
    """Marshal one reskv_rope call once and return a function that issues it (for loops that launch the same
    calls many times). The caller keeps the tensors alive and unchanged in place. The call goes to `stream`, or to the
    stream that is current now: marshal it on the stream and device on which it will be issued or captured."""
    import torch
    B, d, n = shape.batch, shape.head_dim, int(positions.shape[-1]) if positions.dim() > 1 else 1
    at = []
    for name, x, heads in (("q", q, shape.num_q_heads), ("q_out", q_out, shape.num_q_heads),
                           ("k", k, shape.num_kv_heads), ("k_out", k_out, shape.num_kv_heads)):
        if x is None:
            at += [None, None]
            continue
        if tuple(x.shape) != (B, heads, n, d) or x.stride(3) != 1:
            raise ValueError(f"{name} must be [{B}, {heads}, {n}, {d}] with adjoining elements, got {tuple(x.shape)} "
                             f"by {x.stride()}")
        at += [_tensor(name, x, _dtype(shape), x.numel(), False), ctypes.byref(Rows(*x.stride()[:3]))]
    args = (ctypes.byref(shape), _rope(rope), n, _tensor("positions", positions, torch.int32, B * n),
            _tensor("n_tok", n_tok, torch.int32, B), *at, _stream(stream))
    return _prepared(lib().reskv_rope, args, (shape, rope))


def reskv_rope(shape, rope, positions, q=None, q_out=None, k=None, k_out=None, n_tok=None, stream=None):
    """Rotate q [B, Hq, n, d] and / or k [B, Hkv, n, d] (any strides: pass a transposed view of a token-major
    tensor) into q_out, k_out by positions [B, n]; rows from n_tok [B] on are left as they were."""
    prepare_rope(shape, rope, positions, q, q_out, k, k_out, n_tok, stream)()


def reskv_quant_cache_size(shape):
    return lib().reskv_quant_cache_size(ctypes.byref(shape))


def _quant_lens(shape, cache, res_len, main_len):
    import torch
    pairs = shape.batch * shape.num_kv_heads
    return (_tensor("cache", cache, torch.uint8, reskv_quant_cache_size(shape)),
            _tensor("res_len", res_len, torch.int32, pairs), _tensor("main_len", main_len, torch.int32, pairs))


def prepare_pack_quant(shape, kc, vc, res_len, main_len, cache, stream=None):
    """As prepare_rope, for reskv_pack_quant."""
    for name, x in (("kc", kc), ("vc", vc)):
        _order(name, x, shape.batch, shape.num_kv_heads, shape.slot_cap, shape.head_dim)
    c, rl, ml = _quant_lens(shape, cache, res_len, main_len)
    count = shape.batch * shape.num_kv_heads * shape.slot_cap * shape.head_dim
    args = (ctypes.byref(shape), _tensor("kc", kc, _dtype(shape), count), _tensor("vc", vc, _dtype(shape), count),
            rl, ml, c, _stream(stream))
    return _prepared(lib().reskv_pack_quant, args, (shape,))


def reskv_pack_quant(shape, kc, vc, res_len, main_len, cache, stream=None):
    """Live slots of kc, vc [B, Hkv, C, d] into the 4-bit cache (uint8, reskv_quant_cache_size bytes)."""
    prepare_pack_quant(shape, kc, vc, res_len, main_len, cache, stream)()


def prepare_unpack_quant(shape, cache, res_len, main_len, kc, vc, first_slot=None, stream=None):
    """As prepare_rope, for reskv_unpack_quant."""
    import torch
    pairs, n = shape.batch * shape.num_kv_heads, int(kc.shape[-2])
    for name, x in (("kc", kc), ("vc", vc)):
        _order(name, x, shape.batch, shape.num_kv_heads, n, shape.head_dim)
    c, rl, ml = _quant_lens(shape, cache, res_len, main_len)
    args = (ctypes.byref(shape), c, rl, ml, _tensor("first_slot", first_slot, torch.int32, pairs), n,
            _tensor("kc", kc, _dtype(shape), pairs * n * shape.head_dim),
            _tensor("vc", vc, _dtype(shape), pairs * n * shape.head_dim), _stream(stream))
    return _prepared(lib().reskv_unpack_quant, args, (shape,))


def reskv_unpack_quant(shape, cache, res_len, main_len, kc, vc, first_slot=None, stream=None):
    """Values of the 4-bit cache into kc, vc [B, Hkv, n, d]: row i is slot first_slot + i (0 + i if None); rows
    whose slot is not live are left as they were."""
    prepare_unpack_quant(shape, cache, res_len, main_len, kc, vc, first_slot, stream)()


def _turn(shape, rope, positions, n):
    import torch
    return (_rope(rope),
            _tensor("positions", positions, torch.int32, shape.batch * n))


def prepare_append_kv_quant(shape, k_new, v_new, cache, res_len, main_len, rope=None, positions=None, n_tok=None,
                            stream=None):
    """As prepare_rope, for reskv_append_kv_quant."""
    import torch
    n = int(k_new.shape[2]) if k_new.dim() == 4 else 1
    for name, x in (("k_new", k_new), ("v_new", v_new)):
        _order(name, x, shape.batch, shape.num_kv_heads, n, shape.head_dim)
    if n > 1:
        _order("positions", positions, shape.batch, n)
    c, rl, ml = _quant_lens(shape, cache, res_len, main_len)
    count = shape.batch * shape.num_kv_heads * n * shape.head_dim
    args = (ctypes.byref(shape), *_turn(shape, rope, positions, n), n,
            _tensor("n_tok", n_tok, torch.int32, shape.batch), _tensor("k_new", k_new, _dtype(shape), count),
            _tensor("v_new", v_new, _dtype(shape), count), c, rl, ml, _stream(stream))
    return _prepared(lib().reskv_append_kv_quant, args, (shape, rope))


def reskv_append_kv_quant(shape, k_new, v_new, cache, res_len, main_len, rope=None, positions=None, n_tok=None,
                          stream=None):
    """Append k_new, v_new [B, Hkv, n, d] ([B, Hkv, d] for one token) to the 4-bit cache, keys rotated by
    positions [B, n] where a plan is given; tokens from n_tok [B] on are padding."""
    prepare_append_kv_quant(shape, k_new, v_new, cache, res_len, main_len, rope, positions, n_tok, stream)()


def reskv_decode_quant_workspace_size(shape):
    return lib().reskv_decode_quant_workspace_size(ctypes.byref(shape))


def prepare_decode_attn_quant(shape, gate, q, cache, logc, res_len, main_len, out, workspace, rope=None,
                              positions=None, dbg_lse_main=None, dbg_lse_res=None, dbg_gate=None, k_new=None,
                              v_new=None, stream=None):
    """As prepare_rope, for reskv_decode_attn_quant."""
    import torch
    B, Hq, H, d = shape.batch, shape.num_q_heads, shape.num_kv_heads, shape.head_dim
    dt, f32 = _dtype(shape), torch.float32
    _tensor("the gate's tau", getattr(gate, "tau_tensor", None), f32, B * Hq)
    c, rl, ml = _quant_lens(shape, cache, res_len, main_len)
    args = (ctypes.byref(shape), ctypes.byref(gate), *_turn(shape, rope, positions, 1),
            _tensor("q", q, dt, B * Hq * d), c, _tensor("logc", logc, f32, B * H * shape.res_cap), rl, ml,
            _tensor("k_new", k_new, dt, B * H * d), _tensor("v_new", v_new, dt, B * H * d),
            _tensor("out", out, f32, B * Hq * d), _tensor("dbg_lse_main", dbg_lse_main, f32, B * Hq),
            _tensor("dbg_lse_res", dbg_lse_res, f32, B * Hq), _tensor("dbg_gate", dbg_gate, f32, B * Hq),
            _tensor("workspace", workspace, workspace.dtype, workspace.numel()),
            workspace.numel() * workspace.element_size(), _stream(stream))
    return _prepared(lib().reskv_decode_attn_quant, args, (shape, gate, rope))


def reskv_decode_attn_quant(shape, gate, q, cache, logc, res_len, main_len, out, workspace, rope=None, positions=None,
                            dbg_lse_main=None, dbg_lse_res=None, dbg_gate=None, k_new=None, v_new=None, stream=None):
    """One decode step over the 4-bit cache; with a plan, q and k_new are rotated by positions [B] on the way."""
    prepare_decode_attn_quant(shape, gate, q, cache, logc, res_len, main_len, out, workspace, rope, positions,
                              dbg_lse_main, dbg_lse_res, dbg_gate, k_new, v_new, stream)()


def status_string(status):
    return lib().reskv_status_string(status).decode()


def last_error():
    return lib().reskv_last_error().decode()
