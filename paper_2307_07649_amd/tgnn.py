"""Thin ctypes binding of libtgnn.so.  Argument marshalling only: every step of the training path runs in
the HIP kernels behind the C ABI (include/tgnn.h).  PyTorch supplies device memory and streams.

The library must have been built (python -m paper_2307_07649_amd.build); importing this module raises if
libtgnn.so is missing -- there is no CPU fallback.
"""
from __future__ import annotations

import ctypes as C
import os
from array import array

import numpy as np
import torch

_LIB_PATH = os.environ.get("TGNN_LIB") or os.path.join(os.path.dirname(os.path.abspath(__file__)), "libtgnn.so")
if not os.path.exists(_LIB_PATH):
    raise ImportError(f"{_LIB_PATH} not found: build it with `python -m paper_2307_07649_amd.build`")
_lib = C.CDLL(_LIB_PATH)

PARAM_NAMES = ["time_w", "time_b", "gru_wih", "gru_whh", "gru_bih", "gru_bhh", "wq", "bq", "wk", "bk",
               "wv", "bv", "wo", "bo", "dec_ws", "dec_wd", "dec_b1", "dec_w2", "dec_b2"]
MAX_BATCHES = 16
MAX_STEPS_PER_CALL = 8
FLAG_OVERWRITE_GRADS = 1
FLAG_SIDE_STREAM = 2
FLAG_NO_GRAPH = 4
FLAG_WIDE_ROOT_TILES = 8
FLAG_GENERIC_ATTN = 16


class tgnn_config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_nodes", "d_mem", "d_time", "d_edge", "d_static", "n_heads", "k",
                                         "max_batch", "n_replicas", "dt_source", "flags", "max_neg_sets",
                                         "n_classes")]


class tgnn_graph(C.Structure):
    _fields_ = [("indptr", C.c_void_p), ("nbr", C.c_void_p), ("eid", C.c_void_p), ("ts", C.c_void_p),
                ("efeat", C.c_void_p), ("n_events", C.c_int64)]


class tgnn_state(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("mem", "mem_ts", "mail", "mail_ts", "mail_eid", "stat")]


class tgnn_params(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in PARAM_NAMES]


class tgnn_batch(C.Structure):
    _fields_ = [("src", C.c_void_p), ("dst", C.c_void_p), ("neg", C.c_void_p), ("eid", C.c_void_p),
                ("t", C.c_void_p), ("n", C.c_int32), ("replica", C.c_int32)]


class tgnn_seqs(C.Structure):
    _fields_ = [("indptr", C.c_void_p), ("cnt", C.c_void_p), ("n_rows", C.c_int64), ("n_seqs", C.c_int32), ("max_len", C.c_int32),
                ("newest_first", C.c_int32)]


class tgnn_scan(C.Structure):
    _fields_ = ([(n, C.c_int32) for n in ("dtype", "d", "n_state", "n_groups", "softplus", "n_states")] +
                [(n, C.c_void_p) for n in ("x", "dt", "B", "C", "z")] +
                [(n, C.c_int64) for n in ("ld_x", "ld_dt", "ld_b", "ld_c", "ld_z")] +
                [(n, C.c_void_p) for n in ("A", "D", "dt_bias", "state_in", "state_idx")])


class tgnn_scan_grads(C.Structure):
    _fields_ = ([(n, C.c_void_p) for n in ("dx", "ddt", "dB", "dC", "dz")] +
                [(n, C.c_int64) for n in ("ld_dx", "ld_ddt", "ld_db", "ld_dc", "ld_dz")] +
                [(n, C.c_void_p) for n in ("dA", "dD", "ddt_bias")])


_P = C.c_void_p
_I = C.c_int32
_L = C.c_int64
_SIGS = {
    "tgnn_last_error": (C.c_char_p, []),
    "tgnn_create": (_I, [C.POINTER(tgnn_config), C.POINTER(_P)]),
    "tgnn_destroy": (_I, [_P]),
    "tgnn_workspace_bytes": (C.c_int64, [_P]),
    "tgnn_build_tcsr": (_I, [_P, _P, _P, C.c_int64, _I, _P, _P, _P, _P]),
    "tgnn_state_reset": (_I, [_P, C.POINTER(tgnn_state), _I, _P]),
    "tgnn_sample_recent": (_I, [_P, C.POINTER(tgnn_graph), _P, _P, _I, _P, _P, _P, _P, _P]),
    "tgnn_gather_memory": (_I, [_P, C.POINTER(tgnn_graph), C.POINTER(tgnn_state), _I, _P, _I, _P, _P, _P, _P, _P, _P, _P]),
    "tgnn_gru_update": (_I, [_P, C.POINTER(tgnn_params), _I, _P, _P, _P, _P, _P, _P, _P, _P, _P]),
    "tgnn_temporal_attn_fwd": (_I, [_P, C.POINTER(tgnn_params), _I, _P, _P, _P, _P, _P, _P, _P]),
    "tgnn_temporal_attn_bwd": (_I, [_P, C.POINTER(tgnn_params), _I, _P, C.POINTER(tgnn_params), _P, _P, _P]),
    "tgnn_memory_writeback": (_I, [_P, C.POINTER(tgnn_state), _I, _P, _P, _P, _P, _I, _P, _P, _P, _P, _P, _P]),
    "tgnn_memory_writeback_noalloc": (_I, [_I, _I, C.POINTER(tgnn_state), _P, _P, _P, _P, _I, _P, _P, _P, _P, _P, _P]),
    "tgnn_train_step": (_I, [_P, C.POINTER(tgnn_graph), C.POINTER(tgnn_state), C.POINTER(tgnn_params),
                             C.POINTER(tgnn_params), C.POINTER(tgnn_batch), _I, C.c_float, _P, _P, _P, _P]),
    "tgnn_train_step_epoch_parallel": (_I, [_P, C.POINTER(tgnn_graph), C.POINTER(tgnn_state), C.POINTER(tgnn_params),
                                            C.POINTER(tgnn_params), C.POINTER(tgnn_batch), _I, _I, C.c_float, _P, _P, _P, _P]),
    "tgnn_train_step_edge_class": (_I, [_P, C.POINTER(tgnn_graph), C.POINTER(tgnn_state), C.POINTER(tgnn_params),
                                        C.POINTER(tgnn_params), C.POINTER(tgnn_batch), _I, C.POINTER(_P), C.c_float, _P, _P,
                                        _P, _P]),
    "tgnn_eval_step": (_I, [_P, C.POINTER(tgnn_graph), C.POINTER(tgnn_state), C.POINTER(tgnn_params), C.POINTER(tgnn_batch),
                            _I, _I, _P, _P, _P, _P, _P]),
    "tgnn_eval_step_edge_class": (_I, [_P, C.POINTER(tgnn_graph), C.POINTER(tgnn_state), C.POINTER(tgnn_params),
                                       C.POINTER(tgnn_batch), _I, C.POINTER(_P), _P, _P, _P, _P]),
    "tgnn_train_steps": (_I, [_P, C.POINTER(tgnn_graph), C.POINTER(tgnn_state), C.POINTER(tgnn_params),
                              C.POINTER(tgnn_params), _I, C.POINTER(tgnn_batch), _I, C.c_float, _P, _P]),
    "tgnn_set_optimizer": (_I, [_P, _I, C.POINTER(tgnn_params), C.POINTER(tgnn_params), C.c_float, C.c_float, C.c_float]),
    "tgnn_set_grad_clip": (_I, [_P, C.c_float, _P]),
    "tgnn_train_static": (_I, [_P, _I, _P, C.c_float]),
    "tgnn_debug_read": (_I, [_P, _I, _P, C.c_int64, _P]),
    "tgnn_debug_copy": (_I, [_P, _P, C.c_int64, _P]),
    "tgnn_zero_params": (_I, [_P, C.POINTER(tgnn_params), _P]),
    "tgnn_causal_conv_fwd": (_I, [C.POINTER(tgnn_seqs), _I, _I, _I, _P, _L, _P, _P, _I, _P, _P, _P, _I, _P, _L, _P]),
    "tgnn_causal_conv_step": (_I, [_I, _L, _I, _I, _P, _L, _P, _P, _I, _P, _P, _P, _I, _P, _L, _P]),
    "tgnn_causal_conv_workspace_bytes": (_L, [_I, _I]),
    "tgnn_causal_conv_bwd": (_I, [C.POINTER(tgnn_seqs), _I, _I, _I, _P, _L, _P, _L, _P, _P, _I, _P, _P, _I, _P, _L, _P, _P, _I, _P,
                                  _L, _P]),
    "tgnn_selective_scan_saved_bytes": (_L, [C.POINTER(tgnn_seqs), _I, _I]),
    "tgnn_selective_scan_workspace_bytes": (_L, [C.POINTER(tgnn_seqs), _I, _I, _I, _I, _I]),
    "tgnn_selective_scan_fwd": (_I, [C.POINTER(tgnn_seqs), C.POINTER(tgnn_scan), _P, _L, _P, _P, _L, _P, _L, _P]),
    "tgnn_selective_scan_step": (_I, [C.POINTER(tgnn_scan), _L, _P, _L, _P, _P]),
    "tgnn_selective_scan_bwd": (_I, [C.POINTER(tgnn_seqs), C.POINTER(tgnn_scan), _P, _L, _P, _L, C.POINTER(tgnn_scan_grads), _I, _P,
                                     _L, _P]),
    "tgnn_layer_norm_fwd": (_I, [_I, _L, _I, _P, _L, _P, _P, C.c_float, _P, _L, _P, _P, _P]),
    "tgnn_layer_norm_workspace_bytes": (_L, [_L, _I]),
    "tgnn_layer_norm_bwd": (_I, [_I, _L, _I, _P, _L, _P, _L, _P, _P, _P, _P, _L, _P, _P, _I, _P, _L, _P]),
    "tgnn_clip_workspace_bytes": (_L, [_I]),
    "tgnn_grad_norm": (_I, [_I, _P, _P, _P, _P, _P, _L, _P]),
    "tgnn_clip_grads": (_I, [_I, _P, _P, _P, C.c_float, _P, _P, _P, _L, _P]),
    "tgnn_profile_enable": (_I, [_P, C.c_uint32]),
    "tgnn_profile_every": (_I, [_P, _I]),
    "tgnn_profile_read": (_I, [_P, _I, C.POINTER(_I), C.POINTER(C.c_double)]),
}
EXPORTS = list(_SIGS)
for _name, (_res, _args) in _SIGS.items():
    _fn = getattr(_lib, _name)          # AttributeError here = the library does not export a declared symbol
    _fn.restype = _res
    _fn.argtypes = _args


class TgnnError(RuntimeError):
    def __init__(self, code):
        self.code = code
        super().__init__(f"libtgnn error {code}: {_lib.tgnn_last_error().decode()}")


def _check(rc):
    if rc != 0:
        raise TgnnError(rc)


def _ptr(t):
    if t is None:
        return None
    assert t.is_contiguous(), "tensor must be contiguous"
    return t.data_ptr()


def _stream():
    return torch.cuda.current_stream().cuda_stream


def build_tcsr(src, dst, ts, n_nodes):
    """HOST.  numpy int32/int32/float64 event list -> (indptr i64, nbr i32, eid i32, ts f64) numpy arrays."""
    src = np.ascontiguousarray(src, np.int32); dst = np.ascontiguousarray(dst, np.int32)
    ts = np.ascontiguousarray(ts, np.float64)
    E = len(src)
    indptr = np.empty(n_nodes + 1, np.int64); nbr = np.empty(2 * E, np.int32); eid = np.empty(2 * E, np.int32)
    tso = np.empty(2 * E, np.float64)
    _check(_lib.tgnn_build_tcsr(src.ctypes.data, dst.ctypes.data, ts.ctypes.data, E, n_nodes, indptr.ctypes.data,
                                nbr.ctypes.data, eid.ctypes.data, tso.ctypes.data))
    return indptr, nbr, eid, tso


def tgnn_debug_copy(dst, src):
    """dst[:] = src through the library's plain copy kernel (HBM-traffic counter calibration)."""
    assert dst.numel() * dst.element_size() == src.numel() * src.element_size()
    _check(_lib.tgnn_debug_copy(_ptr(dst), _ptr(src), src.numel() * src.element_size(), _stream()))


def tgnn_memory_writeback_noalloc(st, src, dst, eid, t, s_src, s_dst, tau_src, tau_dst, out_winner):
    """st: a State of one replica; out_winner: int32 device tensor [2 n] (preallocated by the caller: the call
    itself allocates nothing)."""
    n_nodes, d_mem = st.mem.shape
    _check(_lib.tgnn_memory_writeback_noalloc(n_nodes, d_mem, C.byref(st.c), _ptr(src), _ptr(dst), _ptr(eid), _ptr(t),
                                              src.numel(), _ptr(s_src), _ptr(s_dst), _ptr(tau_src), _ptr(tau_dst),
                                              _ptr(out_winner), _stream()))
    return out_winner


# ---- operators on sequences of events: plain functions, no context ----
# Every function looks at its tensors once (types, shapes, strides, device) and hands pointers on; `dev` is the current GPU.
_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


def _device_of(t):
    return torch.cuda.current_device() if t.is_cuda else None


def _elsewhere(t, name):
    return ValueError(f"{name} is on {t.device}: a tensor on the current GPU is needed")


def _int32(n, name):
    """n, which the library takes as an int32 (ctypes would hand on its low 32 bits alone)."""
    if not -0x80000000 <= n <= 0x7fffffff:
        raise ValueError(f"{name} = {n} is outside what 32 bits hold")
    return n


def _rows(t, name, dev, dtype=None, shape=None):
    """(pointer, row distance) of a row array: two dimensions, values of a row next to each other; dtype, shape: what it has to be."""
    s = t.shape
    if len(s) != 2 or t.dtype not in _DTYPES:
        raise ValueError(f"{name}: a two-dimensional tensor of float32, bfloat16 or float16 is needed, not {tuple(s)} {t.dtype}")
    if dtype is not None and (t.dtype != dtype or s != shape):
        raise ValueError(f"{name}: {tuple(shape)} {dtype} is needed, not {tuple(s)} {t.dtype}")
    ld, one = t.stride()
    n, c = s
    if one != 1 and c > 1 and n > 0:
        raise ValueError(f"{name}: the values of a row have to be contiguous")
    if c > 0x7fffffff:
        raise ValueError(f"{name}: {c} columns are more than 32 bits hold")
    if t.get_device() != dev:
        raise _elsewhere(t, name)
    return t.data_ptr(), (ld if n > 1 else c)


def _floats(t, name, dev, shape):
    """Pointer of a contiguous float32 tensor of this shape, None for None."""
    if t is None:
        return None
    if t.dtype != torch.float32 or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name}: a contiguous float32 tensor {tuple(shape)} is needed, not {tuple(t.shape)} {t.dtype}")
    if t.get_device() != dev:
        raise _elsewhere(t, name)
    return t.data_ptr()


def _workspace(n_bytes, device):
    return torch.empty(n_bytes, dtype=torch.uint8, device=device)


def _weight_grads(given, shapes, device):
    """Gradient tensors of weights and whether they are added to: the caller's (all of them or none), or new ones."""
    n = sum(g is not None for g in given)
    if n == 0:
        return [torch.empty(s, dtype=torch.float32, device=device) for s in shapes], 0
    if n != len(given):
        raise ValueError("the gradients of all weights are needed, or of none")
    return given, 1


class Seqs:
    """Sequences of events as rows of row arrays (tgnn_seqs): indptr int64 [n_seqs + 1] or None (slots of max_len rows), cnt
    int32 [n_seqs] or None (slots are full); newest_first: rows as tgnn_sample_recent orders them.  max_len: rows of a slot, or with
    indptr the length of the longest sequence."""

    def __init__(self, n_rows, n_seqs, max_len, indptr=None, cnt=None, newest_first=False):
        for t, name, dtype, n in ((indptr, "indptr", torch.int64, n_seqs + 1), (cnt, "cnt", torch.int32, n_seqs)):
            if t is not None:
                if t.dtype != dtype or t.shape != (n,) or not t.is_contiguous():
                    raise ValueError(f"{name}: a contiguous {dtype} tensor ({n},) is needed, not {tuple(t.shape)} {t.dtype}")
                if t.get_device() != _device_of(t):
                    raise _elsewhere(t, name)
        self.indptr, self.cnt, self.n_rows, self.n_seqs = indptr, cnt, n_rows, n_seqs
        self.dev = next((t.get_device() for t in (indptr, cnt) if t is not None), None)
        self.c = tgnn_seqs(None if indptr is None else indptr.data_ptr(), None if cnt is None else cnt.data_ptr(), n_rows,
                           _int32(n_seqs, "n_seqs"), _int32(max_len, "max_len"), 1 if newest_first else 0)


def _seq_rows(seqs, x):
    if x.dim() == 2 and x.shape[0] != seqs.n_rows:
        raise ValueError(f"x has {x.shape[0]} rows, the sequences {seqs.n_rows}")
    if seqs.dev is not None and x.get_device() != seqs.dev:
        raise ValueError(f"x is on {x.device}, the sequences on cuda:{seqs.dev}")


def _states(state_in, state_out, state_idx, dev, n, shape, dtype):
    """(state_in, state_out, state_idx, n_states) as the library takes them; n: sequences (or rows) of the call."""
    states, ptr = None, []
    for t, name in ((state_in, "state_in"), (state_out, "state_out")):
        if t is not None:
            s = t.shape
            if t.dtype != dtype or len(s) != 3 or s[1:] != shape or not t.is_contiguous() or (states is not None and s[0] != states):
                raise ValueError(f"{name}: a contiguous {dtype} tensor {('n_states',) + shape} is needed, not {tuple(s)} {t.dtype}")
            if t.get_device() != dev:
                raise _elsewhere(t, name)
            states = _int32(s[0], "n_states")
        ptr.append(None if t is None else t.data_ptr())
    if state_idx is not None:
        if state_idx.dtype != torch.int32 or state_idx.shape != (n,) or not state_idx.is_contiguous():
            raise ValueError(f"state_idx: a contiguous int32 tensor ({n},) is needed, not {tuple(state_idx.shape)} {state_idx.dtype}")
        if state_idx.get_device() != dev:
            raise _elsewhere(state_idx, "state_idx")
        ptr.append(state_idx.data_ptr())
    else:
        if states is not None and states != n:
            raise ValueError(f"{'state_in' if state_in is not None else 'state_out'}: {n} states are needed without state_idx, not {states}")
        ptr.append(None)
    return (*ptr, states or 0)


def tgnn_causal_conv_fwd(seqs, x, weight, bias=None, silu=True, state_in=None, state_out=None, state_idx=None, out=None):
    """x [rows, d], float32, bfloat16 or float16; weight [d, width], bias [d] float32; states [n_states, width - 1, d] in x's type
    -> y (without `out` a new tensor, in which rows outside all slots hold nothing in particular)."""
    _seq_rows(seqs, x)
    dev = _device_of(x)
    px, ldx = _rows(x, "x", dev)
    d, w = x.shape[1], _int32(weight.shape[-1], "width")
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device) if out is None else out
    py, ldy = _rows(y, "out", dev, x.dtype, x.shape)
    si, so, ix, ns = _states(state_in, state_out, state_idx, dev, seqs.n_seqs, (w - 1, d), x.dtype)
    _check(_lib.tgnn_causal_conv_fwd(seqs.c, _DTYPES[x.dtype], d, w, px, ldx, _floats(weight, "weight", dev, (d, w)),
                                     _floats(bias, "bias", dev, (d,)), 1 if silu else 0, si, so, ix, ns, py, ldy, _stream()))
    return y


def tgnn_causal_conv_step(x, weight, bias=None, silu=True, state_in=None, state_out=None, state_idx=None, out=None):
    """One event per row of x; state_out may be state_in -> y."""
    dev = _device_of(x)
    px, ldx = _rows(x, "x", dev)
    n, d = x.shape
    w = _int32(weight.shape[-1], "width")
    y = torch.empty(n, d, dtype=x.dtype, device=x.device) if out is None else out
    py, ldy = _rows(y, "out", dev, x.dtype, x.shape)
    si, so, ix, ns = _states(state_in, state_out, state_idx, dev, n, (w - 1, d), x.dtype)
    _check(_lib.tgnn_causal_conv_step(_DTYPES[x.dtype], n, d, w, px, ldx, _floats(weight, "weight", dev, (d, w)),
                                      _floats(bias, "bias", dev, (d,)), 1 if silu else 0, si, so, ix, ns, py, ldy, _stream()))
    return y


def tgnn_causal_conv_bwd(seqs, dy, x, weight, bias=None, silu=True, state_in=None, state_idx=None, d_weight=None, d_bias=None,
                         out=None):
    """-> dx, d_weight, d_bias.  Given d_weight and d_bias are added to; without them new ones are written."""
    _seq_rows(seqs, x)
    dev = _device_of(x)
    px, ldx = _rows(x, "x", dev)
    pdy, lddy = _rows(dy, "dy", dev, x.dtype, x.shape)
    d, w = x.shape[1], _int32(weight.shape[-1], "width")
    dx = torch.empty(x.shape, dtype=x.dtype, device=x.device) if out is None else out
    pdx, lddx = _rows(dx, "out", dev, x.dtype, x.shape)
    (dw, db), add = _weight_grads((d_weight, d_bias), ((d, w), (d,)), x.device)
    si, _, ix, ns = _states(state_in, None, state_idx, dev, seqs.n_seqs, (w - 1, d), x.dtype)
    ws = _workspace(_lib.tgnn_causal_conv_workspace_bytes(d, w), x.device)
    _check(_lib.tgnn_causal_conv_bwd(seqs.c, _DTYPES[x.dtype], d, w, pdy, lddy, px, ldx, _floats(weight, "weight", dev, (d, w)),
                                     _floats(bias, "bias", dev, (d,)), 1 if silu else 0, si, ix, ns, pdx, lddx,
                                     _floats(dw, "d_weight", dev, (d, w)), _floats(db, "d_bias", dev, (d,)), add, ws.data_ptr(),
                                     ws.numel(), _stream()))
    return dx, dw, db


def _scan_args(x, dt, A, B, Cm, D, z, dt_bias, softplus, dev, states):
    px, ldx = _rows(x, "x", dev)
    dtype, shape, bc = x.dtype, x.shape, B.shape
    if A.dim() != 2:
        raise ValueError(f"A: a float32 tensor (d, n_state) is needed, not {tuple(A.shape)} {A.dtype}")
    d, n = A.shape
    if shape[1] != d or n == 0 or len(bc) != 2 or bc[0] != shape[0] or bc[1] % n != 0 or bc[1] == 0:
        raise ValueError(f"x {tuple(shape)}, A {tuple(A.shape)} and B {tuple(bc)} do not belong together")
    pdt, lddt = _rows(dt, "dt", dev, dtype, shape)
    pb, ldb = _rows(B, "B", dev, dtype, bc)
    pc, ldc = _rows(Cm, "C", dev, dtype, bc)
    pz, ldz = (None, 0) if z is None else _rows(z, "z", dev, dtype, shape)
    si, _, ix, ns = states
    return tgnn_scan(_DTYPES[dtype], d, n, bc[1] // n, 1 if softplus else 0, ns, px, pdt, pb, pc, pz, ldx, lddt, ldb, ldc, ldz,
                     _floats(A, "A", dev, (d, n)), _floats(D, "D", dev, (d,)), _floats(dt_bias, "dt_bias", dev, (d,)), si, ix)


def _bytes(n):
    if n < 0:
        raise TgnnError(n)
    return n


def selective_scan_saved(seqs, A):
    """A buffer that tgnn_selective_scan_fwd fills for tgnn_selective_scan_bwd (the states every 32 events)."""
    d, n = A.shape
    need = _bytes(_lib.tgnn_selective_scan_saved_bytes(seqs.c, _int32(d, "d"), _int32(n, "n_state")))
    return torch.empty(need // 4, dtype=torch.float32, device=A.device)


def _saved(saved, dev):
    if saved is None:
        return None, 0
    return _floats(saved, "saved", dev, saved.shape), saved.numel() * 4


def tgnn_selective_scan_fwd(seqs, x, dt, A, B, C, D=None, z=None, dt_bias=None, softplus=True, state_in=None, state_out=None,
                            state_idx=None, saved=None, out=None):
    """x, dt, z [rows, d], B, C [rows, n_groups n_state], float32, bfloat16 or float16; A [d, n_state], D, dt_bias [d] float32;
    states [n_states, d, n_state] float32; saved: selective_scan_saved(...) -> y (without `out` a new tensor, in which rows outside all
    slots hold nothing in particular)."""
    _seq_rows(seqs, x)
    dev = _device_of(x)
    states = _states(state_in, state_out, state_idx, dev, seqs.n_seqs, tuple(A.shape), torch.float32)
    a = _scan_args(x, dt, A, B, C, D, z, dt_bias, softplus, dev, states)
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device) if out is None else out
    py, ldy = _rows(y, "out", dev, x.dtype, x.shape)
    ps, ns = _saved(saved, dev)
    need = _bytes(_lib.tgnn_selective_scan_workspace_bytes(seqs.c, a.d, a.n_state, a.n_groups, 0, 0))
    ws = _workspace(need, x.device) if need else None
    _check(_lib.tgnn_selective_scan_fwd(seqs.c, a, py, ldy, states[1], ps, ns, ws.data_ptr() if need else None, need, _stream()))
    return y


def tgnn_selective_scan_step(x, dt, A, B, C, D=None, z=None, dt_bias=None, softplus=True, state_in=None, state_out=None,
                             state_idx=None, out=None):
    """One event per row; state_out may be state_in -> y."""
    dev = _device_of(x)
    states = _states(state_in, state_out, state_idx, dev, x.shape[0], tuple(A.shape), torch.float32)
    a = _scan_args(x, dt, A, B, C, D, z, dt_bias, softplus, dev, states)
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device) if out is None else out
    py, ldy = _rows(y, "out", dev, x.dtype, x.shape)
    _check(_lib.tgnn_selective_scan_step(a, x.shape[0], py, ldy, states[1], _stream()))
    return y


def tgnn_selective_scan_bwd(seqs, dy, x, dt, A, B, C, D=None, z=None, dt_bias=None, softplus=True, state_in=None, state_idx=None,
                            saved=None, dA=None, dD=None, ddt_bias=None, out=None):
    """-> dict of dx, ddt, dB, dC, dA and, with z, D, dt_bias given, dz, dD, ddt_bias.  Given gradients of the weights (of all
    that there are) are added to; without them new ones are written.  out: a dict of the row arrays to write (dx, ddt, dB, dC, dz)."""
    _seq_rows(seqs, x)
    dev = _device_of(x)
    states = _states(state_in, None, state_idx, dev, seqs.n_seqs, tuple(A.shape), torch.float32)
    a = _scan_args(x, dt, A, B, C, D, z, dt_bias, softplus, dev, states)
    dtype, shape, bc = x.dtype, x.shape, B.shape
    pdy, lddy = _rows(dy, "dy", dev, dtype, shape)
    weights = [(n, g) for n, g, v in (("dA", dA, A), ("dD", dD, D), ("ddt_bias", ddt_bias, dt_bias)) if v is not None]
    if (dD is not None and D is None) or (ddt_bias is not None and dt_bias is None):
        raise ValueError("a gradient of a weight that there is none of")
    w, add = _weight_grads([v for _, v in weights], [A.shape if n == "dA" else (a.d,) for n, _ in weights], x.device)
    like = (("dx", shape), ("ddt", shape), ("dB", bc), ("dC", bc)) + ((("dz", shape),) if z is not None else ())
    g = {n: torch.empty(s, dtype=dtype, device=x.device) if out is None else out[n] for n, s in like}
    rows = [_rows(g[n], n, dev, dtype, s) for n, s in like] + ([] if z is not None else [(None, 0)])
    g.update((n, v) for (n, _), v in zip(weights, w))
    c = tgnn_scan_grads(*[r[0] for r in rows], *[r[1] for r in rows], _floats(g["dA"], "dA", dev, A.shape),
                        _floats(g.get("dD"), "dD", dev, (a.d,)), _floats(g.get("ddt_bias"), "ddt_bias", dev, (a.d,)))
    ps, ns = _saved(saved, dev)
    need = _bytes(_lib.tgnn_selective_scan_workspace_bytes(seqs.c, a.d, a.n_state, a.n_groups, 1, 0 if saved is None else 1))
    ws = _workspace(need, x.device)
    _check(_lib.tgnn_selective_scan_bwd(seqs.c, a, pdy, lddy, ps, ns, c, add, ws.data_ptr(), need, _stream()))
    return g


def tgnn_layer_norm_fwd(x, weight=None, bias=None, eps=1e-5, out=None):
    """x [rows, cols], float32, bfloat16 or float16; weight, bias: float32 [cols] or None -> y, mean, rstd."""
    dev = _device_of(x)
    px, ldx = _rows(x, "x", dev)
    n, c = x.shape
    y = torch.empty(n, c, dtype=x.dtype, device=x.device) if out is None else out
    py, ldy = _rows(y, "out", dev, x.dtype, x.shape)
    mean, rstd = torch.empty(2, n, dtype=torch.float32, device=x.device).unbind(0)
    _check(_lib.tgnn_layer_norm_fwd(_DTYPES[x.dtype], n, c, px, ldx, _floats(weight, "weight", dev, (c,)),
                                    _floats(bias, "bias", dev, (c,)), eps, py, ldy, mean.data_ptr(), rstd.data_ptr(), _stream()))
    return y, mean, rstd


def tgnn_layer_norm_bwd(dy, x, mean, rstd, weight=None, d_weight=None, d_bias=None, out=None):
    """-> dx, d_weight, d_bias.  Given d_weight and d_bias are added to; without them new ones are written."""
    dev = _device_of(x)
    px, ldx = _rows(x, "x", dev)
    pdy, lddy = _rows(dy, "dy", dev, x.dtype, x.shape)
    n, c = x.shape
    dx = torch.empty(n, c, dtype=x.dtype, device=x.device) if out is None else out
    pdx, lddx = _rows(dx, "out", dev, x.dtype, x.shape)
    (dw, db), add = _weight_grads((d_weight, d_bias), ((c,), (c,)), x.device)
    ws = _workspace(_lib.tgnn_layer_norm_workspace_bytes(n, c), x.device)
    _check(_lib.tgnn_layer_norm_bwd(_DTYPES[x.dtype], n, c, pdy, lddy, px, ldx, _floats(mean, "mean", dev, (n,)),
                                    _floats(rstd, "rstd", dev, (n,)), _floats(weight, "weight", dev, (c,)), pdx, lddx,
                                    _floats(dw, "d_weight", dev, (c,)), _floats(db, "d_bias", dev, (c,)), add, ws.data_ptr(),
                                    ws.numel(), _stream()))
    return dx, dw, db


def _tensor_list(tensors, name, like=None):
    """Host arrays (pointers, numbers of elements, types) of a list of contiguous tensors or of a Params set, and the first
    tensor's device; like: the numbers and types that they have to have."""
    ts = list(tensors.t.values() if isinstance(tensors, Params) else tensors)
    if not ts:
        return array("Q"), array("q"), array("i"), None
    # (one pass of a built-in per property: several hundred tensors a call)
    kind = array("i", [_DTYPES.get(t.dtype, -1) for t in ts])
    if not all(map(torch.Tensor.is_contiguous, ts)) or -1 in kind:
        raise ValueError(f"{name}: contiguous tensors of float32, bfloat16 or float16 are needed")
    dev = _device_of(ts[0])
    if set(map(torch.Tensor.get_device, ts)) != {dev}:
        raise ValueError(f"{name}: tensors on the current GPU are needed")
    numel = array("q", map(torch.Tensor.numel, ts))
    if like is not None and (numel != like[1] or kind != like[2]):
        raise ValueError(f"{name}: tensors of the gradients' sizes and types are needed")
    return array("Q", map(torch.Tensor.data_ptr, ts)), numel, kind, ts[0].device


def tgnn_grad_norm(grads, out_norm=None):
    """grads: a list of tensors, or a Params set -> the square root of the sum of all their squares, float32 [1]."""
    ptr, numel, kind, device = _tensor_list(grads, "grads")
    norm = torch.empty(1, dtype=torch.float32, device=device or "cuda") if out_norm is None else out_norm
    ws = _workspace(_lib.tgnn_clip_workspace_bytes(len(ptr)), norm.device)
    _check(_lib.tgnn_grad_norm(len(ptr), ptr.buffer_info()[0], numel.buffer_info()[0], kind.buffer_info()[0],
                               _floats(norm, "out_norm", _device_of(norm), (1,)), ws.data_ptr(), ws.numel(), _stream()))
    return norm


def tgnn_clip_grads(grads, max_norm, out=None, out_norm=None):
    """Scales the gradients to a global norm of at most max_norm, in place or into `out` (tensors of the same sizes and types)
    -> their norm before, float32 [1]."""
    ptr, numel, kind, device = given = _tensor_list(grads, "grads")
    to = None if out is None else _tensor_list(out, "out", given)[0]
    norm = torch.empty(1, dtype=torch.float32, device=device or "cuda") if out_norm is None else out_norm
    ws = _workspace(_lib.tgnn_clip_workspace_bytes(len(ptr)), norm.device)
    _check(_lib.tgnn_clip_grads(len(ptr), ptr.buffer_info()[0], numel.buffer_info()[0], kind.buffer_info()[0], max_norm,
                                None if to is None else to.buffer_info()[0], _floats(norm, "out_norm", _device_of(norm), (1,)),
                                ws.data_ptr(), ws.numel(), _stream()))
    return norm


class Graph:
    """Device-resident temporal CSR + edge features."""

    def __init__(self, src, dst, ts, n_nodes, efeat, device="cuda"):
        indptr, nbr, eid, tso = build_tcsr(src, dst, ts, n_nodes)
        self.n_events = len(src)
        self.indptr = torch.from_numpy(indptr).to(device)
        self.nbr = torch.from_numpy(nbr).to(device)
        self.eid = torch.from_numpy(eid).to(device)
        self.ts = torch.from_numpy(tso).to(device)
        if efeat is None:
            self.efeat = None
        elif isinstance(efeat, torch.Tensor):
            self.efeat = efeat.to(device).contiguous()
        else:
            self.efeat = torch.from_numpy(np.ascontiguousarray(efeat, np.float32)).to(device)
        self.c = tgnn_graph(_ptr(self.indptr), _ptr(self.nbr), _ptr(self.eid), _ptr(self.ts), _ptr(self.efeat),
                            self.n_events)


class State:
    def __init__(self, n_nodes, d_mem, n_replicas=1, static=None, device="cuda"):
        n = n_nodes * n_replicas
        self.mem = torch.zeros(n, d_mem, dtype=torch.float32, device=device)
        self.mem_ts = torch.zeros(n, dtype=torch.float64, device=device)
        self.mail = torch.zeros(n, 2 * d_mem, dtype=torch.float32, device=device)
        self.mail_ts = torch.zeros(n, dtype=torch.float64, device=device)
        self.mail_eid = torch.full((n,), -1, dtype=torch.int32, device=device)
        self.stat = None if static is None else torch.as_tensor(static, dtype=torch.float32).to(device).contiguous()
        self.c = tgnn_state(_ptr(self.mem), _ptr(self.mem_ts), _ptr(self.mail), _ptr(self.mail_ts),
                            _ptr(self.mail_eid), _ptr(self.stat))


class Params:
    """Named float32 device tensors in the layout of tgnn_params."""

    def __init__(self, tensors: dict):
        self.t = {n: tensors[n].contiguous() for n in PARAM_NAMES}
        self.c = tgnn_params(*[_ptr(self.t[n]) for n in PARAM_NAMES])

    @classmethod
    def from_numpy(cls, arrays: dict, device="cuda"):
        return cls({n: torch.from_numpy(np.ascontiguousarray(arrays[n], np.float32)).to(device) for n in PARAM_NAMES})

    @classmethod
    def zeros_like(cls, other: "Params"):
        return cls({n: torch.zeros_like(other.t[n]) for n in PARAM_NAMES})

    def zero_(self):
        for v in self.t.values():
            v.zero_()

    def numpy(self):
        return {n: v.detach().cpu().numpy() for n, v in self.t.items()}


class Batch:
    def __init__(self, src, dst, neg, eid, t, replica=0, device="cuda"):
        def dev(a, dt):
            if isinstance(a, torch.Tensor):
                return a.to(device=device, dtype=dt).contiguous()
            return torch.from_numpy(np.ascontiguousarray(a)).to(device=device, dtype=dt)
        self.src, self.dst, self.neg, self.eid = (dev(a, torch.int32) for a in (src, dst, neg, eid))
        self.t = dev(t, torch.float64)
        self.n = int(self.src.numel())
        self.replica = replica
        self.c = tgnn_batch(_ptr(self.src), _ptr(self.dst), _ptr(self.neg), _ptr(self.eid), _ptr(self.t), self.n, replica)


class Context:
    def __init__(self, n_nodes, d_mem, d_time, d_edge, d_static, n_heads, k, max_batch, n_replicas=1, dt_source=0,
                 flags=0, max_neg_sets=1, n_classes=0):
        self.cfg = tgnn_config(n_nodes, d_mem, d_time, d_edge, d_static, n_heads, k, max_batch, n_replicas, dt_source,
                               flags, max_neg_sets, n_classes)
        self.h = _P()
        _check(_lib.tgnn_create(C.byref(self.cfg), C.byref(self.h)))
        self.d_x = d_mem + d_static

    def close(self):
        if self.h:
            _check(_lib.tgnn_destroy(self.h))
            self.h = _P()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def workspace_bytes(self):
        return _lib.tgnn_workspace_bytes(self.h)

    # ---- entry points (same names as the C ABI) ----
    def tgnn_state_reset(self, st: State, replica=-1):
        _check(_lib.tgnn_state_reset(self.h, C.byref(st.c), replica, _stream()))

    def tgnn_sample_recent(self, g: Graph, node, t):
        n, k = node.numel(), self.cfg.k
        dev = node.device
        nbr = torch.empty(n, k, dtype=torch.int32, device=dev); eid = torch.empty_like(nbr)
        ts = torch.empty(n, k, dtype=torch.float64, device=dev); cnt = torch.empty(n, dtype=torch.int32, device=dev)
        _check(_lib.tgnn_sample_recent(self.h, C.byref(g.c), _ptr(node), _ptr(t), n, _ptr(nbr), _ptr(eid), _ptr(ts),
                                       _ptr(cnt), _stream()))
        return nbr, eid, ts, cnt

    def tgnn_gather_memory(self, g: Graph, st: State, replica, slot_node, out=None):
        n = slot_node.numel(); dev = slot_node.device
        dm, de = self.cfg.d_mem, self.cfg.d_edge
        if out is None:
            out = dict(mem=torch.empty(n, dm, device=dev), mail=torch.empty(n, 2 * dm, device=dev),
                       mail_efeat=torch.empty(n, de, device=dev),
                       mem_ts=torch.empty(n, dtype=torch.float64, device=dev),
                       mail_ts=torch.empty(n, dtype=torch.float64, device=dev),
                       has_mail=torch.empty(n, dtype=torch.int32, device=dev))
        _check(_lib.tgnn_gather_memory(self.h, C.byref(g.c), C.byref(st.c), replica, _ptr(slot_node), n,
                                       _ptr(out["mem"]), _ptr(out["mail"]), _ptr(out["mail_efeat"]) if de else None,
                                       _ptr(out["mem_ts"]), _ptr(out["mail_ts"]), _ptr(out["has_mail"]), _stream()))
        return out

    def tgnn_gru_update(self, p: Params, staged: dict):
        n = staged["mem"].shape[0]; dev = staged["mem"].device
        s_new = torch.empty(n, self.cfg.d_mem, device=dev); tau = torch.empty(n, dtype=torch.float64, device=dev)
        _check(_lib.tgnn_gru_update(self.h, C.byref(p.c), n, _ptr(staged["mem"]), _ptr(staged["mail"]),
                                    _ptr(staged["mail_efeat"]) if self.cfg.d_edge else None, _ptr(staged["mem_ts"]),
                                    _ptr(staged["mail_ts"]), _ptr(staged["has_mail"]), _ptr(s_new), _ptr(tau), _stream()))
        return s_new, tau

    def tgnn_temporal_attn_fwd(self, p: Params, x_root, x_nbr, e_nbr, dt_nbr, cnt):
        R = x_root.shape[0]
        z = torch.empty(R, self.cfg.d_mem, device=x_root.device)
        _check(_lib.tgnn_temporal_attn_fwd(self.h, C.byref(p.c), R, _ptr(x_root), _ptr(x_nbr),
                                           _ptr(e_nbr) if self.cfg.d_edge else None, _ptr(dt_nbr), _ptr(cnt), _ptr(z),
                                           _stream()))
        return z

    def tgnn_temporal_attn_bwd(self, p: Params, dz, grads: Params):
        R = dz.shape[0]; dm = self.cfg.d_mem
        d_root = torch.empty(R, dm, device=dz.device); d_nbr = torch.empty(R * self.cfg.k, dm, device=dz.device)
        _check(_lib.tgnn_temporal_attn_bwd(self.h, C.byref(p.c), R, _ptr(dz), C.byref(grads.c), _ptr(d_root),
                                           _ptr(d_nbr), _stream()))
        return d_root, d_nbr

    def tgnn_memory_writeback(self, st: State, replica, src, dst, eid, t, s_src, s_dst, tau_src, tau_dst):
        n = src.numel()
        win = torch.empty(2 * n, dtype=torch.int32, device=src.device)
        _check(_lib.tgnn_memory_writeback(self.h, C.byref(st.c), replica, _ptr(src), _ptr(dst), _ptr(eid), _ptr(t), n,
                                          _ptr(s_src), _ptr(s_dst), _ptr(tau_src), _ptr(tau_dst), _ptr(win), _stream()))
        return win

    def tgnn_train_step(self, g: Graph, st: State, p: Params, grads: Params, batches, lr=0.0, out_loss=None,
                        out_logits=None, out_winner=None):
        arr = (tgnn_batch * len(batches))(*[b.c for b in batches])
        _check(_lib.tgnn_train_step(self.h, C.byref(g.c), C.byref(st.c), C.byref(p.c), C.byref(grads.c), arr,
                                    len(batches), lr, _ptr(out_loss), _ptr(out_logits), _ptr(out_winner), _stream()))

    def tgnn_train_step_epoch_parallel(self, g: Graph, st: State, p: Params, grads: Params, batches, n_neg_sets, lr=0.0,
                                       out_loss=None, out_logits=None, out_winner=None):
        """Each batch's `neg` holds n_neg_sets sets of n negative destinations, one after the other."""
        arr = (tgnn_batch * len(batches))(*[b.c for b in batches])
        _check(_lib.tgnn_train_step_epoch_parallel(self.h, C.byref(g.c), C.byref(st.c), C.byref(p.c), C.byref(grads.c), arr,
                                                   len(batches), n_neg_sets, lr, _ptr(out_loss), _ptr(out_logits),
                                                   _ptr(out_winner), _stream()))

    def tgnn_train_step_edge_class(self, g: Graph, st: State, p: Params, grads: Params, batches, labels, lr=0.0,
                                   out_loss=None, out_logits=None, out_winner=None):
        """labels: one float32 device tensor [n, n_classes] per batch (the batches' `neg` is not read)."""
        arr = (tgnn_batch * len(batches))(*[b.c for b in batches])
        lab = (_P * len(batches))(*[_ptr(y) for y in labels])
        _check(_lib.tgnn_train_step_edge_class(self.h, C.byref(g.c), C.byref(st.c), C.byref(p.c), C.byref(grads.c), arr,
                                               len(batches), lab, lr, _ptr(out_loss), _ptr(out_logits), _ptr(out_winner),
                                               _stream()))

    def tgnn_eval_step(self, g: Graph, st: State, p: Params, batches, n_neg_sets, out_rank, out_rr_sum, out_logits=None,
                       out_winner=None):
        """Each batch's `neg` holds n_neg_sets sets of n negative destinations; out_rank [sum n] float32, out_rr_sum [1]
        float32 (the sum of 1 / rank is added to it)."""
        arr = (tgnn_batch * len(batches))(*[b.c for b in batches])
        _check(_lib.tgnn_eval_step(self.h, C.byref(g.c), C.byref(st.c), C.byref(p.c), arr, len(batches), n_neg_sets,
                                   _ptr(out_logits), _ptr(out_rank), _ptr(out_rr_sum), _ptr(out_winner), _stream()))

    def tgnn_eval_step_edge_class(self, g: Graph, st: State, p: Params, batches, labels, out_counts, out_logits=None,
                                  out_winner=None):
        """labels: one float32 device tensor [n, n_classes] per batch; out_counts: int32 device tensor [3], the counts
        tp, fp, fn of the predictions logit > 0 are added to it."""
        arr = (tgnn_batch * len(batches))(*[b.c for b in batches])
        lab = (_P * len(batches))(*[_ptr(y) for y in labels])
        _check(_lib.tgnn_eval_step_edge_class(self.h, C.byref(g.c), C.byref(st.c), C.byref(p.c), arr, len(batches), lab,
                                              _ptr(out_logits), _ptr(out_counts), _ptr(out_winner), _stream()))

    def tgnn_train_steps(self, g: Graph, st: State, p: Params, grads: Params, steps, lr=0.0, out_loss=None):
        """steps: a list of steps, each a list of Batch (the same number per step); out_loss: device array [len(steps)]."""
        nb = len(steps[0])
        flat = [b.c for step in steps for b in step]
        arr = (tgnn_batch * len(flat))(*flat)
        _check(_lib.tgnn_train_steps(self.h, C.byref(g.c), C.byref(st.c), C.byref(p.c), C.byref(grads.c), len(steps), arr,
                                     nb, lr, _ptr(out_loss), _stream()))

    def tgnn_set_optimizer(self, kind, m: Params = None, v: Params = None, beta1=0.9, beta2=0.999, eps=1e-8):
        self._opt = (m, v)      # keeps the moment tensors alive
        _check(_lib.tgnn_set_optimizer(self.h, kind, C.byref(m.c) if m else None, C.byref(v.c) if v else None, beta1, beta2,
                                       eps))

    def tgnn_set_grad_clip(self, max_norm, out_norm=None):
        """max_norm of the in-step update's gradients, 0: none; out_norm: float32 device tensor, whose first value is every step's norm."""
        if out_norm is not None and out_norm.numel() == 0:
            raise ValueError("out_norm: a float32 tensor of one value is needed")
        norm = None if out_norm is None else _floats(out_norm, "out_norm", _device_of(out_norm), out_norm.shape)
        _check(_lib.tgnn_set_grad_clip(self.h, max_norm, norm))
        self._clip_norm = out_norm      # keeps it alive

    def tgnn_train_static(self, enable, grad_static=None, lr_static=0.0):
        self._gstat = grad_static
        _check(_lib.tgnn_train_static(self.h, 1 if enable else 0, _ptr(grad_static), lr_static))

    def tgnn_zero_params(self, grads: Params):
        _check(_lib.tgnn_zero_params(self.h, C.byref(grads.c), _stream()))

    def tgnn_profile_enable(self, stage_mask: int):
        _check(_lib.tgnn_profile_enable(self.h, stage_mask))

    def tgnn_profile_every(self, n: int):
        _check(_lib.tgnn_profile_every(self.h, n))

    def tgnn_profile_read(self, stage: int):
        cnt = _I(0); ms = C.c_double(0.0)
        _check(_lib.tgnn_profile_read(self.h, stage, C.byref(cnt), C.byref(ms)))
        return cnt.value, ms.value

    def tgnn_debug_read(self, what, dst):
        _check(_lib.tgnn_debug_read(self.h, what, _ptr(dst), dst.numel() * dst.element_size(), _stream()))
        return dst
