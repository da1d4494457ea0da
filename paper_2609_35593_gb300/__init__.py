"""Python binding of the ReSS C-ABI library (libress.so).

Argument marshalling only: every function here checks the tensors it is given (device,
dtype, contiguity), passes raw pointers and the current CUDA stream to the function of the
same name in include/ress.h, and turns a negative return code into RessError.  All
arithmetic runs in the library's CUDA kernels (the newer operators' questions about tensors
are asked in C++, by _tensors.so); if libress.so is missing the import fails (build it with `python -m paper_2609_35593_gb300.build` or __graft_entry__.build()).
"""
from __future__ import annotations

import ctypes
import os
import re
import struct

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libress.so")
HEADER = os.path.join(os.path.dirname(HERE), "include", "ress.h")

if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is not built; run paper_2609_35593_gb300.build.build() first")
_lib = ctypes.CDLL(LIB_PATH)

HEAD_DIM = 64
BLOCK = 64
MAX_HEADS = 32
MAX_BLOCKS = 4096

STATUS = {0: "RESS_OK", -1: "RESS_EINVAL", -2: "RESS_EWORKSPACE", -3: "RESS_EUNSUPPORTED",
          -4: "RESS_ECUDA", -5: "RESS_ETIMEOUT", -6: "RESS_EDEVICE"}


class RessError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{STATUS.get(code, code)}: {msg}")
        self.code = code


class Dims(ctypes.Structure):
    """ress_dims: one global-attention layer."""
    _fields_ = [("n_tokens", ctypes.c_int32), ("n_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("block", ctypes.c_int32),
                ("n_special", ctypes.c_int32), ("d_model", ctypes.c_int32),
                ("q_block", ctypes.c_int32)]


class Variant(ctypes.Structure):
    """ress_variant: selection variant of the ablations (key: 0 drift, 1 probability,
    2 random; direction: 0 minimise, 1 restoration maximises, 2 everything maximises;
    cdf: 0, or the threshold tau of the CDF rule, which keeps further candidates until the
    kept pooled mass reaches tau)."""
    _fields_ = [("key", ctypes.c_int32), ("direction", ctypes.c_int32), ("seed", ctypes.c_uint64),
                ("cdf", ctypes.c_float), ("reserved", ctypes.c_int32)]


_KEYS = {"drift": 0, "probability": 1, "random": 2}
_DIRECTIONS = {"none": 0, "swap": 1, "full": 2}


def variant(key: str = "drift", maximize: str = "none", seed: int = 0, cdf: float = 0.0) -> Variant:
    """A ress_variant from names: key in {drift, probability, random}, maximize in
    {none, swap, full}; cdf the CDF threshold tau (0: off)."""
    return Variant(_KEYS[key], _DIRECTIONS[maximize], seed, cdf, 0)


class WsLayout(ctypes.Structure):
    """ress_ws_layout: byte offsets of the workspace arrays."""
    _fields_ = [(n, ctypes.c_int64) for n in
                ("status", "counter", "qbar", "kbar", "vbar", "ztil", "ytil", "gtil", "P", "q", "t",
                 "K", "G", "J", "Jbest", "J0", "dmask", "bmask", "plen", "asplit", "ksplit", "zsplit",
                 "cdot", "ny", "nz", "lstat", "kcount", "prow", "ld", "words", "total")]


ROPE_MAX_AXES, ROPE_MAX_DIM = 4, 256
_LAYOUTS = {"sections": 0, "halves": 1, "interleaved": 2}


class RopePlan(ctypes.Structure):
    """ress_rope_plan: which channels of a head rotate with which axis, and how fast."""
    _fields_ = [("head_dim", ctypes.c_int32), ("n_axes", ctypes.c_int32),
                ("axis_dims", ctypes.c_int32 * ROPE_MAX_AXES), ("layout", ctypes.c_int32),
                ("n_pairs", ctypes.c_int32), ("turns", ctypes.c_uint64 * (ROPE_MAX_DIM // 2))]


# ress_norm, ress_head_norm and ress_rope_heads as bytes (in a call of a few microseconds, nested
# ctypes structures would be most of it)
_NORM = struct.Struct("@qiiiif4xqqqq")              # rows, width, types, eps, strides
_HEAD_NORM = struct.Struct("@i4xPP")                # enabled, weight, bias
_ROPE_HEADS = struct.Struct("@i4xi4xPPPqqPqqPqqPP")  # n_heads, norm, x, y, dx, dweight, dbias; for callers with
#                                                       raw pointers (tensors.cpp fills it from tensors)


_c = ctypes
_P = _c.c_void_p
_SIGS = {
    "ress_last_error": (_c.c_char_p, []),
    "ress_abi_version": (_c.c_int32, []),
    "ress_kernel_launches": (_c.c_uint64, []),
    "ress_num_blocks": (_c.c_int32, [_c.POINTER(Dims)]),
    "ress_num_candidates": (_c.c_int32, [_c.POINTER(Dims)]),
    "ress_num_query_blocks": (_c.c_int32, [_c.POINTER(Dims)]),
    "ress_num_query_candidates": (_c.c_int32, [_c.POINTER(Dims)]),
    "ress_workspace_bytes": (_c.c_size_t, [_c.POINTER(Dims)]),
    "ress_workspace_layout": (_c.c_int, [_c.POINTER(Dims), _c.POINTER(WsLayout)]),
    "ress_csr_capacity": (_c.c_int64, [_c.POINTER(Dims), _P]),
    "ress_csr_capacity_variant": (_c.c_int64, [_c.POINTER(Dims), _P, _c.POINTER(Variant)]),
    "ress_prepare_wo": (_c.c_int, [_c.POINTER(Dims), _P, _P, _P]),
    "ress_score": (_c.c_int, [_c.POINTER(Dims), _P, _P, _P, _P, _P, _P, _c.c_size_t, _P]),
    "ress_restore": (_c.c_int, [_c.POINTER(Dims), _P, _c.c_int32, _c.c_float, _P, _c.c_size_t,
                                _P, _P, _c.c_int64, _P, _P, _P]),
    "ress_sparse_attn": (_c.c_int, [_c.POINTER(Dims), _P, _P, _P, _P, _P, _c.c_int64, _P, _P,
                                    _c.c_size_t, _P]),
    "ress_sparse_attn_f32": (_c.c_int, [_c.POINTER(Dims), _P, _P, _P, _P, _P, _c.c_int64, _P, _P,
                                        _c.c_size_t, _P]),
    "ress_forward": (_c.c_int, [_c.POINTER(Dims), _P, _P, _P, _P, _P, _c.c_int32, _c.c_float, _P,
                                _c.c_size_t, _P, _P, _c.c_int64, _P, _P, _P]),
    "ress_forward_host": (_c.c_int, [_c.POINTER(Dims), _P, _P, _P, _P, _P, _P, _P, _P, _P, _P,
                                     _c.c_int32, _c.c_float, _P, _c.c_size_t, _P, _P, _c.c_int64,
                                     _P, _P]),
    "ress_status": (_c.c_int, [_P, _P]),
    "ress_wait_selftest": (_c.c_int, [_P, _c.c_size_t, _c.c_uint32, _P]),
    "ress_score_variant": (_c.c_int, [_c.POINTER(Dims), _P, _P, _P, _P, _P, _c.POINTER(Variant), _P,
                                      _c.c_size_t, _P]),
    "ress_restore_variant": (_c.c_int, [_c.POINTER(Dims), _P, _c.c_int32, _c.c_float,
                                        _c.POINTER(Variant), _P, _c.c_size_t, _P, _P, _c.c_int64,
                                        _P, _P, _P]),
    "ress_out_proj": (_c.c_int, [_c.POINTER(Dims), _P, _P, _P, _P, _P, _c.c_size_t, _P]),
    "ress_token_drift": (_c.c_int, [_c.POINTER(Dims), _P, _P, _P, _P, _P, _c.c_size_t, _P]),
    "ress_sparse_attn_noalloc": (_c.c_int, [_c.POINTER(Dims), _P, _P, _P, _P, _P, _c.c_int64, _P,
                                            _c.c_int32, _P]),
    "ress_layer_norm": (_c.c_int, [_P, _P, _P, _P, _P, _P, _P, _P]),
    "ress_layer_norm_workspace_bytes": (_c.c_size_t, [_P]),
    "ress_layer_norm_bwd": (_c.c_int, [_P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P,
                                       _c.c_size_t, _P]),
    "ress_rope_plan_init": (_c.c_int, [_c.POINTER(RopePlan), _c.c_int32, _c.c_int32, _P, _c.c_int32,
                                       _c.c_double, _P]),
    "ress_rope": (_c.c_int, [_c.POINTER(RopePlan), _c.c_int64, _P, _c.c_int32, _c.c_int32, _c.c_float, _P,
                             _P, _P]),
    "ress_rope_workspace_bytes": (_c.c_size_t, [_c.POINTER(RopePlan), _c.c_int64, _c.c_int32, _c.c_int32]),
    "ress_rope_bwd": (_c.c_int, [_c.POINTER(RopePlan), _c.c_int64, _P, _c.c_int32, _c.c_int32, _c.c_float,
                                 _P, _P, _P, _c.c_size_t, _P]),
    "ress_qkv_proj": (_c.c_int, [_c.POINTER(Dims), _P, _P, _P, _P, _P, _P, _P, _c.POINTER(RopePlan), _P,
                                 _P, _P, _c.c_int32, _c.c_float, _P, _P, _P, _P, _c.c_size_t, _P]),
}
for _name, (_res, _args) in _SIGS.items():
    _f = getattr(_lib, _name)
    _f.restype = _res
    _f.argtypes = _args


def exported_names_in_header(path: str = HEADER) -> list[str]:
    """Function names declared in include/ress.h."""
    text = open(path).read()
    return sorted(set(re.findall(r"\b(ress_[a-z_]+)\s*\(", text)))


def _check(rc: int):
    if rc != 0:
        raise RessError(rc, _lib.ress_last_error().decode())


def dims(n_tokens: int, n_heads: int, n_special: int, d_model: int, q_block: int = 64) -> Dims:
    """ress_dims; q_block 128 selects the paper's grid of 128-token query blocks."""
    return Dims(n_tokens, n_heads, HEAD_DIM, BLOCK, n_special, d_model, q_block)


def kernel_launches() -> int:
    """ress_kernel_launches: kernels this library has enqueued so far in the process."""
    return int(_lib.ress_kernel_launches())


def num_blocks(d: Dims) -> int:
    return _lib.ress_num_blocks(_c.byref(d))


def num_candidates(d: Dims) -> int:
    return _lib.ress_num_candidates(_c.byref(d))


def num_query_blocks(d: Dims) -> int:
    return _lib.ress_num_query_blocks(_c.byref(d))


def num_query_candidates(d: Dims) -> int:
    return _lib.ress_num_query_candidates(_c.byref(d))


def workspace_bytes(d: Dims) -> int:
    n = _lib.ress_workspace_bytes(_c.byref(d))
    if n == 0:
        raise RessError(-1, _lib.ress_last_error().decode())
    return n


def workspace_layout(d: Dims) -> WsLayout:
    L = WsLayout()
    _check(_lib.ress_workspace_layout(_c.byref(d), _c.byref(L)))
    return L


def _budget_array(c_h):
    arr = (_c.c_int32 * len(c_h))(*[int(c) for c in c_h])
    return arr


def csr_capacity(d: Dims, c_h, variant: Variant = None) -> int:
    """col_idx entries the restore may write (every row kept whole under a CDF threshold)."""
    if variant is None:
        n = _lib.ress_csr_capacity(_c.byref(d), _c.cast(_budget_array(c_h), _P))
    else:
        n = _lib.ress_csr_capacity_variant(_c.byref(d), _c.cast(_budget_array(c_h), _P),
                                           _c.byref(variant))
    if n < 0:
        raise RessError(-1, _lib.ress_last_error().decode())
    return n


# ---- tensors -> pointers -------------------------------------------------------------
def _torch():
    import torch
    return torch


def _dev(t, dtypes, name):
    """Device pointer of a contiguous CUDA tensor (None -> NULL)."""
    if t is None:
        return None
    torch = _torch()
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.device.type != "cuda":
        raise ValueError(f"{name} must live on a CUDA device")
    if dtypes and t.dtype not in dtypes:
        raise TypeError(f"{name} has dtype {t.dtype}, expected one of {dtypes}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return _c.c_void_p(t.data_ptr())


def _host(t, dtypes, name):
    """Host pointer of a contiguous CPU tensor (page-locked for asynchronous copies)."""
    torch = _torch()
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.device.type != "cpu":
        raise ValueError(f"{name} must live in host memory")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtypes is not None and t.dtype not in dtypes:
        raise TypeError(f"{name} has dtype {t.dtype}, expected one of {dtypes}")
    return _c.c_void_p(t.data_ptr())


_current_stream = None


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    # the current device's current stream without a Stream object (0.1 us instead of 3)
    global _current_stream
    if _current_stream is None:
        _current_stream = _torch()._C._cuda_getCurrentRawStream
    return _current_stream(-1)


def _bf16():
    torch = _torch()
    return (torch.bfloat16, torch.int16, torch.uint16)


def prepare_wo(d: Dims, W_o, F, stream=None):
    torch = _torch()
    _check(_lib.ress_prepare_wo(_c.byref(d), _dev(W_o, _bf16(), "W_o"), _dev(F, (torch.float32,), "F"),
                                _stream(stream)))


def score(d: Dims, Q, K, V, F, c_h, ws, stream=None, variant: Variant = None):
    """ress_score, or ress_score_variant when a Variant is given."""
    torch = _torch()
    args = (_dev(Q, _bf16(), "Q"), _dev(K, _bf16(), "K"), _dev(V, _bf16(), "V"),
            _dev(F, (torch.float32,), "F"), _c.cast(_budget_array(c_h), _P))
    tail = (_dev(ws, None, "ws"), ws.numel() * ws.element_size(), _stream(stream))
    if variant is None:
        _check(_lib.ress_score(_c.byref(d), *args, *tail))
    else:
        _check(_lib.ress_score_variant(_c.byref(d), *args, _c.byref(variant), *tail))


def restore(d: Dims, c_h, rounds: int, rho: float, ws, row_ptr, col_idx, J_best=None,
            drop_mask=None, stream=None, variant: Variant = None):
    """ress_restore, or ress_restore_variant when a Variant is given."""
    torch = _torch()
    head = (_c.cast(_budget_array(c_h), _P), int(rounds), float(rho))
    tail = (_dev(ws, None, "ws"), ws.numel() * ws.element_size(),
            _dev(row_ptr, (torch.int32,), "row_ptr"), _dev(col_idx, (torch.int32,), "col_idx"),
            col_idx.numel(), _dev(J_best, (torch.float32,), "J_best"),
            _dev(drop_mask, (torch.int32, torch.uint32), "drop_mask"), _stream(stream))
    if variant is None:
        _check(_lib.ress_restore(_c.byref(d), *head, *tail))
    else:
        _check(_lib.ress_restore_variant(_c.byref(d), *head, _c.byref(variant), *tail))


def sparse_attn(d: Dims, Q, K, V, row_ptr, col_idx, O, ws, stream=None):
    torch = _torch()
    _check(_lib.ress_sparse_attn(_c.byref(d), _dev(Q, _bf16(), "Q"), _dev(K, _bf16(), "K"),
                                 _dev(V, _bf16(), "V"), _dev(row_ptr, (torch.int32,), "row_ptr"),
                                 _dev(col_idx, (torch.int32,), "col_idx"), col_idx.numel(),
                                 _dev(O, _bf16(), "O"), _dev(ws, None, "ws"),
                                 ws.numel() * ws.element_size(), _stream(stream)))


def out_proj(d: Dims, O, W_o, x, y, ws, stream=None):
    """ress_out_proj: y = x + O W_o^T (x None: y = O W_o^T); bf16 tensors."""
    _check(_lib.ress_out_proj(_c.byref(d), _dev(O, _bf16(), "O"), _dev(W_o, _bf16(), "W_o"),
                              _dev(x, _bf16(), "x"), _dev(y, _bf16(), "y"), _dev(ws, None, "ws"),
                              ws.numel() * ws.element_size(), _stream(stream)))


def token_drift(d: Dims, O_a, O_b, W_o, drift, ws, stream=None):
    """ress_token_drift: drift[b] = sum over block b's tokens of ||W_o (O_a - O_b)||^2."""
    torch = _torch()
    _check(_lib.ress_token_drift(_c.byref(d), _dev(O_a, _bf16(), "O_a"), _dev(O_b, _bf16(), "O_b"),
                                 _dev(W_o, _bf16(), "W_o"), _dev(drift, (torch.float32,), "drift"),
                                 _dev(ws, None, "ws"), ws.numel() * ws.element_size(),
                                 _stream(stream)))


def sparse_attn_f32(d: Dims, Q, K, V, row_ptr, col_idx, O, ws, stream=None):
    """ress_sparse_attn with a float32 output tensor O [N, H, 64]."""
    torch = _torch()
    _check(_lib.ress_sparse_attn_f32(_c.byref(d), _dev(Q, _bf16(), "Q"), _dev(K, _bf16(), "K"),
                                     _dev(V, _bf16(), "V"), _dev(row_ptr, (torch.int32,), "row_ptr"),
                                     _dev(col_idx, (torch.int32,), "col_idx"), col_idx.numel(),
                                     _dev(O, (torch.float32,), "O"), _dev(ws, None, "ws"),
                                     ws.numel() * ws.element_size(), _stream(stream)))


def forward(d: Dims, Q, K, V, F, c_h, rounds: int, rho: float, ws, row_ptr, col_idx, O,
            J_best=None, stream=None):
    torch = _torch()
    _check(_lib.ress_forward(_c.byref(d), _dev(Q, _bf16(), "Q"), _dev(K, _bf16(), "K"),
                             _dev(V, _bf16(), "V"), _dev(F, (torch.float32,), "F"),
                             _c.cast(_budget_array(c_h), _P), int(rounds), float(rho),
                             _dev(ws, None, "ws"), ws.numel() * ws.element_size(),
                             _dev(row_ptr, (torch.int32,), "row_ptr"),
                             _dev(col_idx, (torch.int32,), "col_idx"), col_idx.numel(),
                             _dev(O, _bf16(), "O"), _dev(J_best, (torch.float32,), "J_best"),
                             _stream(stream)))


def forward_host(d: Dims, Q_host, K_host, V_host, O_host, Q_dev, K_dev, V_dev, O_dev, F, c_h,
                 rounds: int, rho: float, ws, row_ptr, col_idx, J_best=None, stream=None):
    """ress_forward_host: copies of Q, K, V in, the forward, the copy of O out, all enqueued
    on `stream` (host tensors should be pinned)."""
    torch = _torch()
    b = _bf16()
    _check(_lib.ress_forward_host(_c.byref(d), _host(Q_host, b, "Q_host"), _host(K_host, b, "K_host"),
                                  _host(V_host, b, "V_host"), _host(O_host, b, "O_host"),
                                  _dev(Q_dev, b, "Q_dev"), _dev(K_dev, b, "K_dev"),
                                  _dev(V_dev, b, "V_dev"), _dev(O_dev, b, "O_dev"),
                                  _dev(F, (torch.float32,), "F"), _c.cast(_budget_array(c_h), _P),
                                  int(rounds), float(rho), _dev(ws, None, "ws"),
                                  ws.numel() * ws.element_size(),
                                  _dev(row_ptr, (torch.int32,), "row_ptr"),
                                  _dev(col_idx, (torch.int32,), "col_idx"), col_idx.numel(),
                                  _dev(J_best, (torch.float32,), "J_best"), _stream(stream)))


def sparse_attn_noalloc(d: Dims, Q, K, V, row_ptr, col_idx, O, wait: bool = True, stream=None):
    """ress_sparse_attn without a workspace: scratch is the library's built-in device array
    (see include/ress.h for its size limit and the sharing rules)."""
    torch = _torch()
    _check(_lib.ress_sparse_attn_noalloc(_c.byref(d), _dev(Q, _bf16(), "Q"), _dev(K, _bf16(), "K"),
                                         _dev(V, _bf16(), "V"), _dev(row_ptr, (torch.int32,), "row_ptr"),
                                         _dev(col_idx, (torch.int32,), "col_idx"), col_idx.numel(),
                                         _dev(O, _bf16(), "O"), 1 if wait else 0, _stream(stream)))


def wait_selftest(ws, limit_us: int = 20000, stream=None):
    """ress_wait_selftest: a bounded wait that nothing completes, recorded as RESS_ETIMEOUT in
    the workspace status word (read it with status())."""
    _check(_lib.ress_wait_selftest(_dev(ws, None, "ws"), ws.numel() * ws.element_size(),
                                   int(limit_us), _stream(stream)))


def status(ws, stream=None):
    """Synchronise, read and clear the device status word; raise on a device-side error."""
    _check(_lib.ress_status(_dev(ws, None, "ws"), _stream(stream)))


# ---- the input half of the sublayer ---------------------------------------------------
# Small calls take a few microseconds on the GPU, so csrc/tensors.cpp asks a tensor all that matters in one
# call, and why one is not as it should be is found out afterwards.
class _Tensors:
    """Stands in for the module _tensors until its first use: the rest of the binding needs no torch."""

    def __getattr__(self, name):
        _torch()
        from . import _tensors
        globals()["_t"] = _tensors
        return getattr(_tensors, name)


_t = _Tensors()
_ANY, _F32, _BF16 = 0b0111, 0b0100, 0b1001  # bits of ress_dtype; bit 3: 16-bit integers


def _types():
    torch = _torch()
    return (torch.bfloat16, torch.float16, torch.float32)


def _code(t, name):
    code = None if t is None else _t.code(t)
    if code is None:
        _refuse(t, name, dtypes=_types())
    return code


def _refuse(t, name, dtypes=None, shape=None, numel=None):
    """Raises for a tensor that is not on a CUDA device, or not of this kind; else for its layout."""
    if not isinstance(t, _torch().Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must live on a CUDA device")
    if dtypes is not None and t.dtype not in dtypes:
        raise TypeError(f"{name} has dtype {t.dtype}, expected one of {dtypes}")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if numel is not None and t.numel() != numel:
        raise ValueError(f"{name} has {t.numel()} elements, expected {numel}")
    raise ValueError(f"{name} must be contiguous, or have contiguous rows a fixed stride apart")


def _vector(t, n, name):
    """Device pointer of n contiguous elements of one of the types (None -> NULL)."""
    p = _t.vector(t, n, _ANY)
    if p is None:
        _refuse(t, name, _types(), numel=n)
    return p


def _vector_f32(t, n, name):
    p = _t.vector(t, n, _F32)
    if p is None:
        _refuse(t, name, _types()[2:], numel=n)
    return p


def _rows(t, like, name):
    """Device pointer and elements between the rows of a tensor [..., width] of like's shape."""
    r = _t.rows(t, like)
    if r is None:
        _refuse(t, name, shape=like.shape)
    return r


def _param_code(*params):
    """The one ress_dtype of the parameters that are given (float32 if none is)."""
    code = _t.code(*params)
    if code is None:
        for p in params:
            if p is not None:
                _code(p, "weight or bias")
        raise TypeError("weights and biases of different dtypes")
    return code


def _scratch(ws):
    """Pointer and bytes of a workspace (None -> NULL, 0)."""
    s = _t.scratch(ws)
    if s is None:
        _refuse(ws, "ws")
    return s


def _row_shape(x):
    """Rows, width and ress_dtype of x [..., width]."""
    s = _t.shape(x)
    if s is None:
        shape = getattr(x, "shape", (1,))
        if len(shape) < 1 or shape[-1] < 1:
            raise ValueError(f"x has shape {tuple(shape)}, expected [..., width]")
        _refuse(x, "x", _types())
    return s


def layer_norm(x, weight, bias, y, eps: float = 1e-5, mean=None, rstd=None, stream=None):
    """ress_layer_norm over the last dimension of x [..., width] into y of the same shape; weight, bias
    [width] or None; mean, rstd: float32 outputs, one per row, for layer_norm_bwd, or None."""
    rows, width, code = _row_shape(x)
    (px, sx), (py, sy) = _rows(x, x, "x"), _rows(y, x, "y")
    n = _NORM.pack(rows, width, code, _code(y, "y"), _param_code(weight, bias), eps, sx, sy, 0, 0)
    _check(_lib.ress_layer_norm(n, px, _vector(weight, width, "weight"), _vector(bias, width, "bias"), py,
                                _vector_f32(mean, rows, "mean"), _vector_f32(rstd, rows, "rstd"),
                                _stream(stream)))


def layer_norm_workspace_bytes(rows: int, width: int) -> int:
    """Workspace of layer_norm_bwd on rows of this width."""
    n = _lib.ress_layer_norm_workspace_bytes(_NORM.pack(rows, width, 0, 0, 0, 0.0, width, width, width, width))
    if n == 0:
        raise RessError(-1, _lib.ress_last_error().decode())
    return n


def layer_norm_bwd(dy, x, weight, mean, rstd, dx, dweight=None, dbias=None, dres=None, ws=None, stream=None):
    """ress_layer_norm_bwd: dx (+ dres where given) and the float32 gradients of weight and bias
    (None to skip; ws is needed for them) from the gradient dy of layer_norm's y."""
    rows, width, code = _row_shape(x)
    (pdy, sdy), (px, sx), (pdx, sdx) = _rows(dy, x, "dy"), _rows(x, x, "x"), _rows(dx, x, "dx")
    pres, sres = (0, 0) if dres is None else _rows(dres, x, "dres")
    if dx.dtype != x.dtype or (dres is not None and dres.dtype != x.dtype):
        raise TypeError(f"dx and dres must have x's dtype {x.dtype}")
    if mean is None or rstd is None:
        raise ValueError("mean and rstd are those layer_norm saved")
    n = _NORM.pack(rows, width, code, _code(dy, "dy"), _param_code(weight), 0.0, sx, sdy, sdx, sres)
    _check(_lib.ress_layer_norm_bwd(n, pdy, px, _vector(weight, width, "weight"), _vector_f32(mean, rows, "mean"),
                                    _vector_f32(rstd, rows, "rstd"), pres, pdx,
                                    _vector_f32(dweight, width, "dweight"), _vector_f32(dbias, width, "dbias"),
                                    *_scratch(ws), _stream(stream)))


def rope_plan(axis_dims, head_dim: int = HEAD_DIM, base: float = 100.0, layout: str = "sections",
              freq=None) -> RopePlan:
    """ress_rope_plan_init: axis_dims[a] channels of a head rotate with axis a of the positions.
    layout: sections, halves or interleaved (include/ress.h); freq: radians per unit position of
    each pair, or None for base^(-2i / axis_dims[a])."""
    plan = RopePlan()
    axis_dims = [int(a) for a in axis_dims]
    arr = None
    if freq is not None:
        freq = [float(f) for f in freq]
        if len(freq) != sum(a // 2 for a in axis_dims):
            raise ValueError(f"{len(freq)} frequencies for {sum(a // 2 for a in axis_dims)} pairs")
        arr = (_c.c_double * len(freq))(*freq)
    _check(_lib.ress_rope_plan_init(plan, int(head_dim), len(axis_dims), (_c.c_int32 * len(axis_dims))(*axis_dims),
                                    _LAYOUTS[layout], float(base), arr))
    return plan


def _head_norm(norm, n, name):
    """enabled, weight, bias of None or (weight, bias)."""
    if norm is None:
        return 0, 0, 0
    weight, bias = norm
    return 1, _vector(weight, n, name), _vector(bias, n, name)


def _positions(plan, pos, tokens):
    p = _t.positions(pos, tokens, plan.n_axes)
    if p is None:
        _refuse(pos, "pos", (_torch().int32,), (tokens, plan.n_axes))
    return p


def _rope_heads(plan, name, like, y, x, dx, norm, grads, tokens, code):
    """ress_rope_heads of one tensor [tokens, heads, head_dim] of the type of this code, as like is."""
    h = _t.rope_heads(y, x, dx, norm, grads, tokens, plan.head_dim, code)
    if h is None:
        _refuse_heads(plan, name, like, (x, y, dx), norm, grads, tokens, code)
    return h


def _refuse_heads(plan, name, like, tensors, norm, grads, tokens, code):
    hd, shape = plan.head_dim, like.shape
    if len(shape) != 3 or shape[0] != tokens or shape[2] != hd:
        raise ValueError(f"{name}: shape {tuple(shape)}, expected ({tokens}, heads, {hd})")
    for t in tensors:
        if t is not None and (getattr(t, "shape", None) != shape
                              or _t.rope_heads(t, None, None, None, None, tokens, hd, code) is None):
            _refuse(t, name, _types()[code:code + 1], shape)
    _head_norm(norm, hd, name)
    dweight, dbias = (None, None) if grads is None else grads
    _vector_f32(dweight, hd, name), _vector_f32(dbias, hd, name)
    raise ValueError(f"{name}: norms and their gradients are tuples of two")


def _norm_code(q_norm, k_norm):
    return _param_code(*(q_norm or ()), *(k_norm or ()))


def rope(plan: RopePlan, pos, q, q_out, k=None, k_out=None, q_norm=None, k_norm=None, eps: float = 1e-5,
         stream=None):
    """ress_rope: q_out, k_out = the heads of q, k [tokens, heads, head_dim] after a layer norm over
    their channels (q_norm, k_norm: (weight, bias), either may be None; None: no norm) and rotated by
    pos, int32 [tokens, axes]."""
    if q is None or q_out is None or (k is None) != (k_out is None) or (k is None and k_norm is not None):
        raise ValueError("q and q_out are needed, and k and k_out together")
    tokens, code = pos.size(0), _code(q, "q")
    tq = _rope_heads(plan, "q, q_out or q_norm", q, q_out, q, None, q_norm, None, tokens, code)
    tk = None if k is None else _rope_heads(plan, "k, k_out or k_norm", k, k_out, k, None, k_norm, None, tokens, code)
    _check(_lib.ress_rope(plan, tokens, _positions(plan, pos, tokens), code, _norm_code(q_norm, k_norm), eps, tq, tk,
                          _stream(stream)))


def rope_workspace_bytes(plan: RopePlan, n_tokens: int, q_heads: int, k_heads: int = 0) -> int:
    """Workspace of rope_bwd with gradients of the norms' parameters."""
    n = _lib.ress_rope_workspace_bytes(plan, n_tokens, q_heads, k_heads)
    if n == 0:
        raise RessError(-1, _lib.ress_last_error().decode())
    return n


def rope_bwd(plan: RopePlan, pos, dq_out, dq, dk_out=None, dk=None, q=None, k=None, q_norm=None, k_norm=None,
             q_norm_grads=None, k_norm_grads=None, eps: float = 1e-5, ws=None, stream=None):
    """ress_rope_bwd: the gradients dq, dk of rope's q, k from those of its outputs, and, with norms
    (which need q, k again), q_norm_grads, k_norm_grads: float32 (dweight, dbias), either or both None."""
    if dq_out is None or dq is None or (dk_out is None) != (dk is None) or (dk is None and k_norm is not None):
        raise ValueError("dq_out and dq are needed, and dk_out and dk together")
    if dk is None and k_norm_grads is not None:
        raise ValueError("k_norm_grads are written together with dk")
    if (q_norm is not None and q is None) or (k_norm is not None and k is None):
        raise ValueError("a norm's gradient needs the norm's input")
    tokens, code = pos.size(0), _code(dq_out, "dq_out")
    tq = _rope_heads(plan, "q, dq, dq_out, q_norm or its gradients", dq_out, dq_out, q, dq, q_norm, q_norm_grads, tokens,
                     code)
    tk = None if dk is None else _rope_heads(plan, "k, dk, dk_out, k_norm or its gradients", dk_out, dk_out, k, dk,
                                             k_norm, k_norm_grads, tokens, code)
    _check(_lib.ress_rope_bwd(plan, tokens, _positions(plan, pos, tokens), code, _norm_code(q_norm, k_norm), eps, tq,
                              tk, *_scratch(ws), _stream(stream)))


def _dense(t, n, name):
    """Device pointer of n contiguous bf16 elements (None -> NULL)."""
    p = _t.vector(t, n, _BF16)
    if p is None:
        _refuse(t, name, _bf16(), numel=n)
    return p


def qkv_proj(d: Dims, x, W_q, W_k, W_v, Q, K, V, ws, b_q=None, b_k=None, b_v=None, plan: RopePlan = None, pos=None,
             q_norm=None, k_norm=None, eps: float = 1e-5, stream=None):
    """ress_qkv_proj: Q, K, V [N, H, 64] = x W^T + b with q_norm, k_norm and the rotation by plan and pos
    as in rope; bf16 tensors."""
    n, dm, out = d.n_tokens, d.d_model, d.n_heads * HEAD_DIM
    if (plan is None) != (pos is None):
        raise ValueError("plan and pos belong together")
    _check(_lib.ress_qkv_proj(d, _dense(x, n * dm, "x"), _dense(W_q, out * dm, "W_q"), _dense(W_k, out * dm, "W_k"),
                              _dense(W_v, out * dm, "W_v"), _dense(b_q, out, "b_q"), _dense(b_k, out, "b_k"),
                              _dense(b_v, out, "b_v"), plan, None if pos is None else _positions(plan, pos, n),
                              _HEAD_NORM.pack(*_head_norm(q_norm, HEAD_DIM, "q_norm")),
                              _HEAD_NORM.pack(*_head_norm(k_norm, HEAD_DIM, "k_norm")), _norm_code(q_norm, k_norm), eps,
                              _dense(Q, n * out, "Q"), _dense(K, n * out, "K"), _dense(V, n * out, "V"),
                              *_scratch(ws), _stream(stream)))


class Buffers:
    """Device buffers of one layer shape (workspace, F, CSR, output), allocated by torch."""

    def __init__(self, d: Dims, c_h, device="cuda", variant: Variant = None):
        torch = _torch()
        self.d = d
        self.c_h = [int(c) for c in c_h]
        self.nb = num_blocks(d)
        self.nq = num_query_blocks(d)
        H = d.n_heads
        self.ws = torch.zeros(workspace_bytes(d), dtype=torch.uint8, device=device)
        self.F = torch.zeros(H, 64, 64, dtype=torch.float32, device=device)
        self.row_ptr = torch.zeros(H * self.nq + 1, dtype=torch.int32, device=device)
        self.col_idx = torch.zeros(csr_capacity(d, c_h, variant), dtype=torch.int32, device=device)
        self.O = torch.zeros(d.n_tokens, H, 64, dtype=torch.bfloat16, device=device)
        self.J_best = torch.zeros(H * self.nq, dtype=torch.float32, device=device)
        self.layout = workspace_layout(d)

    def ws_view(self, name: str, dtype=None, shape=None):
        """A typed view of one workspace array (see WsLayout)."""
        torch = _torch()
        L = self.layout
        names = [f[0] for f in WsLayout._fields_]
        off = getattr(L, name)
        order = sorted(getattr(L, n) for n in names[:names.index("ld")])
        nxt = min([o for o in order if o > off] + [L.total])
        dtype = dtype or torch.float32
        raw = self.ws[off:nxt]
        t = raw.view(dtype)
        if shape is not None:
            n = 1
            for s in shape:
                n *= s
            t = t[:n].view(*shape)
        return t
