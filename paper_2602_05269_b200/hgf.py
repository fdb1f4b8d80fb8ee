"""Thin binding of libhgf_b200.so: same names as the C ABI, argument marshalling only (ctypes; linear_forward and the cache calls, whose GPU time
can be shorter than that, through the native module _hgf_python, csrc/hgf_python.cpp, where that loads and for the arguments that it takes).

Tensors are torch CUDA tensors used purely as device memory; every step of the layer runs in the
library's kernels.  If the library is missing, or a call fails, this raises: there is no fallback.
"""
from __future__ import annotations

import contextlib
import ctypes
import importlib.machinery
import importlib.util
import os
import warnings

import torch

from . import build as _build

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libhgf_b200.so")

HGF_OK = 0
FLAG_OUT_BF16 = 0x1
FLAG_NO_SILU = 0x2
FLAG_FORCE_GEMM = 0x4
FLAG_NO_PDL = 0x8
FLAG_BASE3 = 0x10
DECODE_MAX_M = 16
PHASE_PROLOGUE = 0x1
PHASE_GEMV = 0x2

# every symbol include/hgf.h declares
EXPORTS = ["hgf_packed_bytes", "hgf_pack_ternary", "hgf_unpack_ternary", "hgf_workspace_bytes",
           "hgf_linear_forward", "hgf_act_quant", "hgf_check_status", "hgf_tmax_tokens_per_s",
           "hgf_launch_count", "hgf_status_string", "hgf_group_create", "hgf_group_forward",
           "hgf_group_destroy", "hgf_group_forward_phases", "hgf_linear_forward_static", "hgf_group_debug",
           "hgf_linear_forward_phases", "hgf_linear_forward_ln",
           "hgf_packed_bytes_b3", "hgf_pack_ternary_b3", "hgf_unpack_ternary_b3",
           "hgf_selftest_wait_timeout", "hgf_group_create_ln",
           "hgf_diff_attention_forward", "hgf_diff_lambda0", "hgf_backward_workspace_bytes", "hgf_linear_backward",
           "hgf_cache_reserve", "hgf_cache_append", "hgf_cache_read", "hgf_cache_fork", "hgf_cache_free",
           "hgf_cached_workspace_bytes", "hgf_diff_attention_cached"]


class HgfError(RuntimeError):
    def __init__(self, call: str, status: int):
        self.status = status
        super().__init__(f"{call} failed: status {status} ({status_string(status)})")


class Problem(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("M", ctypes.c_int64), ("packed", ctypes.c_void_p),
                ("gamma", ctypes.c_float), ("d_in", ctypes.c_int64), ("d_out", ctypes.c_int64),
                ("At", ctypes.c_void_p), ("Bt", ctypes.c_void_p), ("r", ctypes.c_int32),
                ("gate", ctypes.c_void_p), ("y", ctypes.c_void_p)]


class DebugOut(ctypes.Structure):
    _fields_ = [("xq", ctypes.c_void_p), ("gamma_x", ctypes.c_void_p), ("y_int", ctypes.c_void_p),
                ("h", ctypes.c_void_p)]


class Grads(ctypes.Structure):
    _fields_ = [("dx", ctypes.c_void_p), ("dW", ctypes.c_void_p), ("dAt", ctypes.c_void_p), ("dBt", ctypes.c_void_p),
                ("dgate", ctypes.c_void_p)]


class Cache(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("open", ctypes.c_void_p), ("table", ctypes.c_void_p),
                ("held", ctypes.c_void_p), ("length", ctypes.c_void_p), ("refs", ctypes.c_void_p), ("arrivals", ctypes.c_void_p),
                ("n_pages", ctypes.c_int64), ("n_slots", ctypes.c_int64), ("max_pages", ctypes.c_int64),
                ("n_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32)]


class FrontEnd(ctypes.Structure):
    _fields_ = [("ln_weight", ctypes.c_void_p), ("ln_bias", ctypes.c_void_p), ("eps", ctypes.c_float),
                ("gate_group", ctypes.c_int64), ("mean_out", ctypes.c_void_p), ("rstd_out", ctypes.c_void_p)]


_lib = None
_native_forward = None  # linear_forward's marshalling (set with _lib; None: ctypes)
_native_cache = None    # the native module, for the cache calls' (likewise)


def lib() -> ctypes.CDLL:
    """Load the CUDA library (built in-tree by paper_2602_05269_b200.build)."""
    global _lib, _native_forward, _native_cache
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: run `python -m paper_2602_05269_b200.build` "
                               "(there is no CPU fallback)")
        L = ctypes.CDLL(LIB_PATH)
        c = ctypes
        i64, i32, u32, vp, sz = c.c_int64, c.c_int32, c.c_uint32, c.c_void_p, c.c_size_t
        L.hgf_packed_bytes.restype = sz
        L.hgf_packed_bytes.argtypes = [i64, i64]
        L.hgf_pack_ternary.restype = c.c_int
        L.hgf_pack_ternary.argtypes = [vp, i64, i64, vp, c.POINTER(c.c_float), vp]
        L.hgf_unpack_ternary.restype = c.c_int
        L.hgf_unpack_ternary.argtypes = [vp, i64, i64, vp, vp]
        L.hgf_packed_bytes_b3.restype = sz
        L.hgf_packed_bytes_b3.argtypes = [i64, i64]
        L.hgf_pack_ternary_b3.restype = c.c_int
        L.hgf_pack_ternary_b3.argtypes = [vp, i64, i64, vp, c.POINTER(c.c_float), vp]
        L.hgf_unpack_ternary_b3.restype = c.c_int
        L.hgf_unpack_ternary_b3.argtypes = [vp, i64, i64, vp, vp]
        L.hgf_workspace_bytes.restype = sz
        L.hgf_workspace_bytes.argtypes = [i64, i64, i64, i32, u32]
        L.hgf_linear_forward.restype = c.c_int
        L.hgf_linear_forward.argtypes = [vp, i64, vp, c.c_float, i64, i64, vp, vp, i32, vp, vp, vp, sz,
                                         c.POINTER(DebugOut), u32, vp]
        L.hgf_linear_forward_phases.restype = c.c_int
        L.hgf_linear_forward_phases.argtypes = [vp, i64, vp, c.c_float, i64, i64, vp, vp, i32, vp, vp, vp, sz,
                                                c.POINTER(DebugOut), u32, u32, vp]
        L.hgf_linear_forward_ln.restype = c.c_int
        L.hgf_linear_forward_ln.argtypes = [vp, i64, vp, c.c_float, i64, i64, vp, vp, i32, vp, vp, vp, sz,
                                            c.POINTER(DebugOut), c.POINTER(FrontEnd), u32, vp]
        L.hgf_linear_forward_static.restype = c.c_int
        L.hgf_linear_forward_static.argtypes = [vp, i64, vp, c.c_float, i64, i64, vp, vp, i32, vp, vp, u32, vp]
        L.hgf_act_quant.restype = c.c_int
        L.hgf_act_quant.argtypes = [vp, i64, i64, vp, vp, vp, vp]
        L.hgf_selftest_wait_timeout.restype = c.c_int
        L.hgf_selftest_wait_timeout.argtypes = [u32, vp]
        L.hgf_diff_attention_forward.restype = c.c_int
        L.hgf_diff_attention_forward.argtypes = [vp, vp, vp, i64, i64, i32, i32, c.c_float, c.c_float, vp, u32, vp]
        L.hgf_diff_lambda0.restype = c.c_double
        L.hgf_diff_lambda0.argtypes = [c.c_double]
        L.hgf_backward_workspace_bytes.restype = sz
        L.hgf_backward_workspace_bytes.argtypes = [i64, i64, i64, i32]
        L.hgf_linear_backward.restype = c.c_int
        L.hgf_linear_backward.argtypes = [vp, i64, vp, c.c_float, i64, i64, vp, vp, i32, vp, vp, c.POINTER(Grads), vp, sz, u32, vp]
        cache = c.POINTER(Cache)
        L.hgf_cache_reserve.restype = c.c_int
        L.hgf_cache_reserve.argtypes = [cache, vp, vp, i64, vp, vp]
        L.hgf_cache_append.restype = c.c_int
        L.hgf_cache_append.argtypes = [cache, vp, vp, i64, vp, vp, i64, vp, vp]
        L.hgf_cache_read.restype = c.c_int
        L.hgf_cache_read.argtypes = [cache, vp, vp, vp, i64, i64, vp, vp, u32, vp]
        L.hgf_cache_fork.restype = c.c_int
        L.hgf_cache_fork.argtypes = [cache, vp, vp, i64, vp, vp]
        L.hgf_cache_free.restype = c.c_int
        L.hgf_cache_free.argtypes = [cache, vp, i64, vp]
        L.hgf_cached_workspace_bytes.restype = sz
        L.hgf_cached_workspace_bytes.argtypes = [cache, i64, i64, i32]
        L.hgf_diff_attention_cached.restype = c.c_int
        L.hgf_diff_attention_cached.argtypes = [cache, vp, i64, i32, vp, vp, i64, c.c_float, c.c_float, vp, vp, sz, u32, vp]
        L.hgf_check_status.restype = c.c_int
        L.hgf_check_status.argtypes = [vp]
        L.hgf_tmax_tokens_per_s.restype = c.c_double
        L.hgf_tmax_tokens_per_s.argtypes = [c.c_double] * 3
        L.hgf_launch_count.restype = c.c_uint64
        L.hgf_launch_count.argtypes = []
        L.hgf_group_create.restype = c.c_int
        L.hgf_group_create.argtypes = [c.POINTER(Problem), i32, u32, c.POINTER(vp)]
        L.hgf_group_create_ln.restype = c.c_int
        L.hgf_group_create_ln.argtypes = [c.POINTER(Problem), c.POINTER(FrontEnd), i32, u32, c.POINTER(vp)]
        L.hgf_group_forward.restype = c.c_int
        L.hgf_group_forward.argtypes = [vp, vp]
        L.hgf_group_forward_phases.restype = c.c_int
        L.hgf_group_forward_phases.argtypes = [vp, u32, vp]
        L.hgf_group_debug.restype = c.c_int
        L.hgf_group_debug.argtypes = [vp, i32, vp, c.POINTER(DebugOut)]
        L.hgf_group_destroy.restype = None
        L.hgf_group_destroy.argtypes = [vp]
        L.hgf_status_string.restype = c.c_char_p
        L.hgf_status_string.argtypes = [c.c_int]
        native = _native()
        if native is not None:
            native.bind(c.cast(L.hgf_linear_forward, vp).value, c.cast(L.hgf_linear_forward_ln, vp).value)
            _native_forward = native.linear_forward
            native.bind_cache(*(c.cast(f, vp).value for f in (L.hgf_cache_reserve, L.hgf_cache_append, L.hgf_cache_read, L.hgf_cache_fork, L.hgf_cache_free,
                                                              L.hgf_diff_attention_cached)))
            _native_cache = native
        _lib = L
    return _lib


def _native():
    """The native module beside the library, built with it."""
    path = _build.module_path()
    loader = importlib.machinery.ExtensionFileLoader("_hgf_python", path)
    try:
        module = importlib.util.module_from_spec(importlib.util.spec_from_loader("_hgf_python", loader))
        loader.exec_module(module)
    except ImportError as e:
        warnings.warn(f"{path} is missing or does not load ({e}): linear_forward takes some microseconds longer on the host.  Run "
                      "`python -m paper_2602_05269_b200.build`", RuntimeWarning, stacklevel=3)
        return None
    return module


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream=None):
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _check(call, status):
    if status != HGF_OK:
        raise HgfError(call, status)


def status_string(status: int) -> str:
    return lib().hgf_status_string(int(status)).decode()


def packed_bytes(d_out: int, d_in: int, base3: bool = False) -> int:
    return int(lib().hgf_packed_bytes_b3(d_out, d_in) if base3 else lib().hgf_packed_bytes(d_out, d_in))


def pack_ternary(W: torch.Tensor, stream=None, base3: bool = False):
    """W: CUDA fp32 [d_out][d_in] -> (packed uint8 on the device, gamma_W as float): two bits per weight, or
    with base3 the 1.6-bit layout of hgf_pack_ternary_b3 (forward calls then take FLAG_BASE3)."""
    assert W.is_cuda and W.dtype == torch.float32 and W.is_contiguous() and W.dim() == 2
    d_out, d_in = W.shape
    nbytes = packed_bytes(d_out, d_in, base3)
    if nbytes == 0:
        raise HgfError("hgf_packed_bytes", 2)
    packed = torch.empty(nbytes, dtype=torch.uint8, device=W.device)
    gamma = ctypes.c_float(0.0)
    fn = lib().hgf_pack_ternary_b3 if base3 else lib().hgf_pack_ternary
    _check("hgf_pack_ternary", fn(_ptr(W), d_out, d_in, _ptr(packed), ctypes.byref(gamma), _stream(stream)))
    return packed, float(gamma.value)


def unpack_ternary(packed: torch.Tensor, d_out: int, d_in: int, stream=None, base3: bool = False) -> torch.Tensor:
    T = torch.empty((d_out, d_in), dtype=torch.int8, device=packed.device)
    fn = lib().hgf_unpack_ternary_b3 if base3 else lib().hgf_unpack_ternary
    _check("hgf_unpack_ternary", fn(_ptr(packed), d_out, d_in, _ptr(T), _stream(stream)))
    return T


def workspace_bytes(M: int, d_in: int, d_out: int, r: int, flags: int = 0) -> int:
    return int(lib().hgf_workspace_bytes(M, d_in, d_out, r, flags))


def act_quant(x: torch.Tensor, stream=None):
    """x: CUDA bf16 [M][d_in] -> (xq int8 [M][d_in], gamma_x fp32 [M], row_sum int32 [M])."""
    assert x.is_cuda and x.dtype == torch.bfloat16 and x.is_contiguous()
    M, K = x.shape
    xq = torch.empty((M, K), dtype=torch.int8, device=x.device)
    gx = torch.empty(M, dtype=torch.float32, device=x.device)
    rs = torch.empty(M, dtype=torch.int32, device=x.device)
    _check("hgf_act_quant", lib().hgf_act_quant(_ptr(x), M, K, _ptr(xq), _ptr(gx), _ptr(rs), _stream(stream)))
    return xq, gx, rs


def linear_forward(x, packed, gamma, d_in, d_out, At=None, Bt=None, gate=None, *, y=None, workspace=None,
                   debug=False, flags=0, stream=None, phases=None, ln_weight=None, ln_bias=None, eps=1e-5,
                   gate_group=None):
    """Enqueue one layer forward.  Returns y, or (y, dbg dict of device tensors) with debug=True.

    x bf16 [M][d_in]; packed uint8 from pack_ternary; At fp16 [r][d_in]; Bt fp16 [d_out][r];
    gate fp32 [d_out]; y fp32 (or bf16 with FLAG_OUT_BF16) [M][d_out].
    Decode-sized calls (M <= DECODE_MAX_M) start fetching packed, At and Bt before earlier work on the stream
    has finished: these must not be outputs of work still pending there (x, gate and the LayerNorm's parameters
    may be); FLAG_NO_PDL lifts that.
    With ln_weight / ln_bias (fp32 [d_in]) and/or gate_group the call is hgf_linear_forward_ln: LayerNorm
    in front of the quantiser, gate fp32 [ceil(d_out / gate_group)]; debug then also returns mean and rstd.
    """
    assert x.is_cuda and x.dtype == torch.bfloat16 and x.is_contiguous()
    if _lib is None:
        lib()
    native = _native_forward if not debug and phases is None else None
    if y is None or workspace is None or native is None:
        M = x.shape[0]
        r = 0 if At is None else At.shape[0]
    if y is None:
        y = torch.empty((M, d_out), dtype=torch.bfloat16 if flags & FLAG_OUT_BF16 else torch.float32,
                        device=x.device)
    if workspace is None:
        workspace = torch.empty(workspace_bytes(M, d_in, d_out, r, flags), dtype=torch.uint8, device=x.device)
    if native is not None:
        try:
            st = native(x, packed, gamma, d_in, d_out, At, Bt, gate, y, workspace, flags, stream, ln_weight, ln_bias, eps,
                        None if gate_group is None else int(gate_group or 1))
        except TypeError:  # (it takes plain numbers and addresses only; ctypes has the last word)
            M = x.shape[0]
            r = 0 if At is None else At.shape[0]
        else:
            if st != HGF_OK:
                raise HgfError("hgf_linear_forward", st)
            return y
    dbg_struct, dbg = None, None
    if debug:
        dbg = {"xq": torch.empty((M, d_in), dtype=torch.int8, device=x.device),
               "gamma_x": torch.empty(M, dtype=torch.float32, device=x.device),
               "y_int": torch.empty((M, d_out), dtype=torch.int32, device=x.device),
               "h": torch.empty((M, max(r, 1)), dtype=torch.float32, device=x.device)}
        dbg_struct = DebugOut(dbg["xq"].data_ptr(), dbg["gamma_x"].data_ptr(), dbg["y_int"].data_ptr(),
                              dbg["h"].data_ptr())
    dbg_arg = ctypes.byref(dbg_struct) if dbg_struct is not None else None
    if ln_weight is not None or gate_group is not None:
        assert phases is None
        fe = FrontEnd(None if ln_weight is None else ln_weight.data_ptr(), None if ln_bias is None else ln_bias.data_ptr(),
                      float(eps), int(gate_group or 1), None, None)
        if debug:
            dbg["mean"] = torch.empty(M, dtype=torch.float32, device=x.device)
            dbg["rstd"] = torch.empty(M, dtype=torch.float32, device=x.device)
            fe.mean_out, fe.rstd_out = dbg["mean"].data_ptr(), dbg["rstd"].data_ptr()
        st = lib().hgf_linear_forward_ln(_ptr(x), M, _ptr(packed), ctypes.c_float(gamma), d_in, d_out, _ptr(At), _ptr(Bt),
                                         r, _ptr(gate), _ptr(y), _ptr(workspace), workspace.numel(), dbg_arg,
                                         ctypes.byref(fe), flags, _stream(stream))
    elif phases is None:
        st = lib().hgf_linear_forward(_ptr(x), M, _ptr(packed), ctypes.c_float(gamma), d_in, d_out, _ptr(At), _ptr(Bt),
                                      r, _ptr(gate), _ptr(y), _ptr(workspace), workspace.numel(), dbg_arg, flags,
                                      _stream(stream))
    else:   # hgf_linear_forward_phases: the prologue launch and the contraction launch separately
        st = lib().hgf_linear_forward_phases(_ptr(x), M, _ptr(packed), ctypes.c_float(gamma), d_in, d_out, _ptr(At),
                                             _ptr(Bt), r, _ptr(gate), _ptr(y), _ptr(workspace), workspace.numel(),
                                             dbg_arg, flags, phases, _stream(stream))
    _check("hgf_linear_forward", st)
    if debug:
        dbg["h"] = dbg["h"][:, :r]
        return y, dbg
    return y


STATIC_SCRATCH_BYTES = 288 * 1024


def linear_forward_static(x, packed, gamma, d_in, d_out, y, At=None, Bt=None, gate=None, *, flags=0, stream=None):
    """hgf_linear_forward_static: the layer forward for callers that may not allocate device memory.

    Everything, y included, is passed in; the call itself allocates nothing (no workspace tensor, no
    debug outputs): the library uses a scratch array built into its image.  Decode-sized problems
    only; HgfError status 7 if the problem needs more scratch than STATIC_SCRATCH_BYTES.  Calls on
    one device share that array, so they must not overlap on the GPU.
    """
    assert x.is_cuda and x.dtype == torch.bfloat16 and x.is_contiguous() and y.is_cuda and y.is_contiguous()
    r = 0 if At is None else At.shape[0]
    st = lib().hgf_linear_forward_static(_ptr(x), x.shape[0], _ptr(packed), ctypes.c_float(gamma), d_in, d_out,
                                         _ptr(At), _ptr(Bt), r, _ptr(gate), _ptr(y), flags, _stream(stream))
    _check("hgf_linear_forward_static", st)
    return y


class Group:
    """A group of independent decode-sized problems (hgf_group_*).  `problems` is a list of dicts
    with keys x, packed, gamma, d_in, d_out, y and optionally At, Bt, gate (device tensors), and for
    the front end of hgf_group_create_ln: ln_weight, ln_bias (fp32 [d_in]), eps, gate_group, mean_out,
    rstd_out; the tensors are kept alive by this object.  As in linear_forward, packed, At and Bt must not be
    outputs of work still pending on the stream of a forward, unless flags has FLAG_NO_PDL."""

    def __init__(self, problems, flags: int = 0):
        self._keep = problems
        arr = (Problem * len(problems))()
        for i, q in enumerate(problems):
            At = q.get("At")
            arr[i] = Problem(q["x"].data_ptr(), q["x"].shape[0], q["packed"].data_ptr(), float(q["gamma"]),
                             q["d_in"], q["d_out"], None if At is None else At.data_ptr(),
                             None if q.get("Bt") is None else q["Bt"].data_ptr(), 0 if At is None else At.shape[0],
                             None if q.get("gate") is None else q["gate"].data_ptr(), q["y"].data_ptr())
        self._handle = ctypes.c_void_p()
        if any(("ln_weight" in q or "gate_group" in q) for q in problems):
            fes = (FrontEnd * len(problems))()
            for i, q in enumerate(problems):
                fes[i] = FrontEnd(None if q.get("ln_weight") is None else q["ln_weight"].data_ptr(),
                                  None if q.get("ln_bias") is None else q["ln_bias"].data_ptr(), float(q.get("eps", 1e-5)),
                                  int(q.get("gate_group", 1)),
                                  None if q.get("mean_out") is None else q["mean_out"].data_ptr(),
                                  None if q.get("rstd_out") is None else q["rstd_out"].data_ptr())
            _check("hgf_group_create_ln", lib().hgf_group_create_ln(arr, fes, len(problems), flags, ctypes.byref(self._handle)))
            return
        _check("hgf_group_create", lib().hgf_group_create(arr, len(problems), flags, ctypes.byref(self._handle)))

    def forward(self, stream=None) -> None:
        _check("hgf_group_forward", lib().hgf_group_forward(self._handle, _stream(stream)))

    def forward_phases(self, phases: int, stream=None) -> None:
        _check("hgf_group_forward_phases", lib().hgf_group_forward_phases(self._handle, phases, _stream(stream)))

    def debug(self, index: int, y_int=None):
        """hgf_group_debug: route problem `index`'s int32 accumulators to `y_int` (a device int32
        tensor [M][d_out], or None) from the next forward on, and return views (xq int8 [M][d_in],
        gamma_x fp32 [M]) of the group's own workspace for that problem."""
        q = self._keep[index]
        M, K = q["x"].shape[0], q["d_in"]
        views = DebugOut()
        _check("hgf_group_debug", lib().hgf_group_debug(self._handle, index, _ptr(y_int), ctypes.byref(views)))
        c = ctypes

        def view(ptr, nbytes, dtype, shape):
            class _Mem:  # exposes the device range through the CUDA array interface
                __cuda_array_interface__ = {"shape": (nbytes,), "typestr": "|u1", "data": (int(ptr), False), "version": 2}
            return torch.as_tensor(_Mem(), device=q["x"].device).view(dtype).view(shape)

        return {"xq": view(views.xq, M * K, torch.int8, (M, K)), "gamma_x": view(views.gamma_x, M * 4, torch.float32, (M,))}

    def close(self) -> None:
        if self._handle:
            lib().hgf_group_destroy(self._handle)
            self._handle = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def check_status(stream=None) -> None:
    """Synchronise and raise if a bounded device-side wait gave up since the last check."""
    _check("hgf_check_status", lib().hgf_check_status(_stream(stream)))


def backward_workspace_bytes(M, d_in, d_out, r) -> int:
    return int(lib().hgf_backward_workspace_bytes(M, d_in, d_out, r))


def linear_backward(x, packed, gamma, d_in, d_out, dy, At=None, Bt=None, gate=None, *, flags=0, stream=None, want=None,
                    out=None, workspace=None):
    """hgf_linear_backward: straight-through backward pass.  dy bf16 [M][d_out].  Returns a dict of fp32 device
    tensors dx, dW and (with a correction) dAt, dBt, dgate; `want` restricts which are computed.  `out` (a dict
    returned by an earlier call of the same shape) and `workspace` are reused when given."""
    assert x.is_cuda and x.dtype == torch.bfloat16 and dy.dtype == torch.bfloat16 and x.is_contiguous() and dy.is_contiguous()
    M = x.shape[0]
    r = 0 if At is None else At.shape[0]
    names = ["dx", "dW"] + (["dAt", "dBt", "dgate"] if r else [])
    if want is not None:
        names = [n for n in names if n in want]
    shapes = {"dx": (M, d_in), "dW": (d_out, d_in), "dAt": (r, d_in), "dBt": (d_out, r), "dgate": (d_out,)}
    if out is None:
        out = {n: torch.empty(shapes[n], dtype=torch.float32, device=x.device) for n in names}
    else:
        assert all(n in out and tuple(out[n].shape) == shapes[n] and out[n].dtype == torch.float32 for n in names)
        workspace = workspace if workspace is not None else out.get("_workspace")
    g = Grads(*[out[n].data_ptr() if n in out else None for n in ("dx", "dW", "dAt", "dBt", "dgate")])
    need = backward_workspace_bytes(M, d_in, d_out, r)
    ws = workspace if workspace is not None and workspace.numel() >= need else torch.empty(need, dtype=torch.uint8, device=x.device)
    _check("hgf_linear_backward",
           lib().hgf_linear_backward(_ptr(x), M, _ptr(packed), ctypes.c_float(gamma), d_in, d_out, _ptr(At), _ptr(Bt), r, _ptr(gate),
                                     _ptr(dy), ctypes.byref(g), _ptr(ws), ws.numel(), flags, _stream(stream)))
    out = dict(out)
    out["_workspace"] = ws
    return out


def diff_attention_forward(q, k, v, B: int, L: int, n_heads: int, head_dim: int, lam: float, out_scale: float = 1.0, *,
                           out=None, flags: int = 0, stream=None):
    """hgf_diff_attention_forward: q, k bf16 [B*L][2*n_heads*head_dim], v bf16 [B*L][n_heads*head_dim] ->
    out [B*L][n_heads*head_dim] fp32 (bf16 with FLAG_OUT_BF16)."""
    assert q.is_cuda and q.dtype == torch.bfloat16 and q.is_contiguous() and k.is_contiguous() and v.is_contiguous()
    if out is None:
        out = torch.empty((B * L, n_heads * head_dim), dtype=torch.bfloat16 if flags & FLAG_OUT_BF16 else torch.float32,
                          device=q.device)
    _check("hgf_diff_attention_forward",
           lib().hgf_diff_attention_forward(_ptr(q), _ptr(k), _ptr(v), B, L, n_heads, head_dim, ctypes.c_float(lam),
                                            ctypes.c_float(out_scale), _ptr(out), flags, _stream(stream)))
    return out


CACHE_BLOCK = 64
CACHE_MAX_SEQS = 1024


class KVCache:
    """The arrays of an hgf_cache (8-bit paged K/V cache of the differential attention): `n_slots` sequences of up to
    64 * max_pages + 63 tokens, in `n_pages` pages of 64 tokens, for `n_heads` K/V heads.  The arrays are attributes (codes, scales, open, table,
    held, length, refs, arrivals) on one device, to be changed in place only, since the library goes by their addresses; KVCache.of takes ones that exist already."""

    _SHAPES = {"codes": (torch.int8, lambda c: (c.n_pages, c.n_heads, 3 * CACHE_BLOCK * c.head_dim)), "scales": (torch.float32, lambda c: (c.n_pages, c.n_heads, 4)),
               "open": (torch.bfloat16, lambda c: (c.n_slots, c.n_heads, 3, CACHE_BLOCK, c.head_dim)), "table": (torch.int32, lambda c: (c.n_slots, c.max_pages)),
               "held": (torch.int32, lambda c: (c.n_slots,)), "length": (torch.int32, lambda c: (c.n_slots,)), "refs": (torch.int32, lambda c: (c.n_pages,)),
               "arrivals": (torch.int32, lambda c: (c.n_slots,))}

    def __init__(self, n_heads: int, head_dim: int, n_pages: int, n_slots: int, max_pages: int, device="cuda"):
        self.n_heads, self.head_dim, self.n_pages, self.n_slots, self.max_pages = n_heads, head_dim, n_pages, n_slots, max_pages
        self._bind({name: torch.zeros(shape(self), dtype=dtype, device=device) for name, (dtype, shape) in self._SHAPES.items()})

    @classmethod
    def of(cls, n_heads: int, head_dim: int, **arrays):
        """A cache on arrays that exist: every one of codes, scales, open, table, held, length, refs, arrivals."""
        self = cls.__new__(cls)
        self.n_heads, self.head_dim = n_heads, head_dim
        self.n_pages = arrays["codes"].shape[0]
        self.n_slots, self.max_pages = arrays["table"].shape
        self._bind(arrays)
        return self

    def _bind(self, arrays):
        assert set(arrays) == set(self._SHAPES), "the arrays of a cache are " + ", ".join(self._SHAPES)
        for name, (dtype, shape) in self._SHAPES.items():
            a = arrays[name]
            assert a.dtype == dtype and tuple(a.shape) == shape(self) and a.is_contiguous() and a.device == arrays["codes"].device, f"cache array {name}"
            setattr(self, name, a)
        self.device = self.codes.device
        self._index = self.device.index if self.device.type == "cuda" else -1
        self._struct = Cache(*(arrays[n].data_ptr() for n in self._SHAPES), self.n_pages, self.n_slots, self.max_pages, self.n_heads, self.head_dim)
        self._ref = ctypes.byref(self._struct)
        self._at = ctypes.addressof(self._struct)
        self._bound = frozenset((*self._SHAPES, "n_heads", "head_dim", "n_pages", "n_slots", "max_pages", "device", "_index", "_struct", "_ref", "_at", "_bound"))
        lib()

    def __setattr__(self, name, value):
        if name in self.__dict__.get("_bound", ()) and value is not getattr(self, name):  # (`cache.length -= n` assigns the tensor that it changed)
            raise AttributeError(f"{name} of a cache is what the library was given: change the array in place, or make another cache")
        super().__setattr__(name, value)

    def __delattr__(self, name):
        if name in self.__dict__.get("_bound", ()):
            raise AttributeError(f"{name} of a cache is what the library was given")
        super().__delattr__(name)


def _on(stream):
    """What a cache call makes for itself is made on the stream that the call runs on."""
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)


def _done(call, status) -> bool:
    """What a native cache call returned: done, refused, or (-1) not taken, so that the checks here say why."""
    if status > 0:
        raise HgfError(call, status)
    return status == 0


def _list(cache, *tensors):
    """The lists of a cache call: int32 on the cache's device, which has to be the current one, dense."""
    assert cache.device.type == "cuda" and cache.device.index == torch.cuda.current_device(), f"the cache is on {cache.device}, which is not the current device"
    for a in tensors:
        assert a is None or (a.dtype == torch.int32 and a.device == cache.device and a.is_contiguous() and a.dim() == 1), "lists of a cache call are dense int32 on its device"


def cache_reserve(cache: KVCache, slots, tokens, *, granted=None, stream=None):
    """hgf_cache_reserve: pages for slots[i] to grow to tokens[i] tokens.  Returns `granted` (int32 [n], made here if not given): 1 where it has them."""
    if granted is not None and _native_cache and _done("hgf_cache_reserve", _native_cache.cache_reserve(cache._at, cache._index, slots, tokens, granted, stream)):
        return granted
    _list(cache, slots, tokens, granted)
    n = slots.numel()
    if granted is None:
        with _on(stream):
            granted = torch.empty(n, dtype=torch.int32, device=cache.device)
    assert tokens.numel() == n and granted.numel() == n
    _check("hgf_cache_reserve", lib().hgf_cache_reserve(cache._ref, _ptr(slots), _ptr(tokens), n, _ptr(granted), _stream(stream)))
    return granted


def cache_append(cache: KVCache, k, v, slots, starts, *, done=None, stream=None):
    """hgf_cache_append: rows starts[i] .. starts[i + 1] - 1 of k (bf16 [n_rows][2 * n_heads * head_dim]) and v (bf16 [n_rows][n_heads * head_dim])
    to the sequence in slots[i].  Returns `done` (int32 [n_seqs], made here if not given): 1 where they were appended."""
    if done is not None and _native_cache and _done("hgf_cache_append", _native_cache.cache_append(cache._at, cache._index, k, v, slots, starts, done, stream)):
        return done
    _list(cache, slots, starts, done)
    n, width = slots.numel(), cache.n_heads * cache.head_dim
    assert k.device == v.device == cache.device and k.dtype == v.dtype == torch.bfloat16 and k.is_contiguous() and v.is_contiguous()
    assert k.dim() == 2 and k.shape[1] == 2 * width and v.shape == (k.shape[0], width) and starts.numel() == n + 1
    if done is None:
        with _on(stream):
            done = torch.empty(n, dtype=torch.int32, device=cache.device)
    assert done.numel() == n
    _check("hgf_cache_append", lib().hgf_cache_append(cache._ref, _ptr(k), _ptr(v), k.shape[0], _ptr(slots), _ptr(starts), n, _ptr(done), _stream(stream)))
    return done


def cache_read(cache: KVCache, slots, first, starts, n_rows: int | None = None, *, k=None, v=None, flags: int = 0, stream=None):
    """hgf_cache_read: tokens first[i], first[i] + 1, ... of the sequence in slots[i] as rows starts[i] .. starts[i + 1] - 1 of (k, v): fp32, or bf16
    with FLAG_OUT_BF16.  Without k and v, `n_rows` rows are made here, zero where nothing is read."""
    if k is not None and not flags and _native_cache and _done("hgf_cache_read", _native_cache.cache_read(cache._at, cache._index, slots, first, starts, k, v, stream)):
        return k, v
    _list(cache, slots, first, starts)
    n, width = slots.numel(), cache.n_heads * cache.head_dim
    if k is None:
        assert n_rows is not None, "cache_read takes either n_rows or k and v"
        dtype = torch.bfloat16 if flags & FLAG_OUT_BF16 else torch.float32
        with _on(stream):
            k, v = (torch.zeros((n_rows, w), dtype=dtype, device=cache.device) for w in (2 * width, width))
    elif k.dtype == torch.bfloat16:
        flags |= FLAG_OUT_BF16
    assert k.device == v.device == cache.device and k.is_contiguous() and v.is_contiguous()
    assert k.dtype == v.dtype == (torch.bfloat16 if flags & FLAG_OUT_BF16 else torch.float32)
    assert k.dim() == 2 and k.shape[1] == 2 * width and v.shape == (k.shape[0], width) and starts.numel() == n + 1 and first.numel() == n
    _check("hgf_cache_read",
           lib().hgf_cache_read(cache._ref, _ptr(slots), _ptr(first), _ptr(starts), n, k.shape[0], _ptr(k), _ptr(v), flags, _stream(stream)))
    return k, v


def cache_fork(cache: KVCache, src, dst, *, done=None, stream=None):
    """hgf_cache_fork: the empty slot dst[i] becomes a copy of the sequence in src[i].  Returns `done` (int32 [n]; made here if not given)."""
    if done is None:
        with _on(stream):
            done = torch.empty_like(src)
    if _native_cache and _done("hgf_cache_fork", _native_cache.cache_fork(cache._at, cache._index, src, dst, done, stream)):
        return done
    _list(cache, src, dst, done)
    n = src.numel()
    assert dst.numel() == n and done.numel() == n
    _check("hgf_cache_fork", lib().hgf_cache_fork(cache._ref, _ptr(src), _ptr(dst), n, _ptr(done), _stream(stream)))
    return done


def cache_free(cache: KVCache, slots, *, stream=None) -> None:
    """hgf_cache_free: empties the slots and gives their pages back."""
    if _native_cache and _done("hgf_cache_free", _native_cache.cache_free(cache._at, cache._index, slots, stream)):
        return
    _list(cache, slots)
    _check("hgf_cache_free", lib().hgf_cache_free(cache._ref, _ptr(slots), slots.numel(), _stream(stream)))


def cached_workspace_bytes(cache: KVCache, n_seqs: int, n_rows: int, n_heads: int) -> int:
    """hgf_cached_workspace_bytes: for a call of these sizes.  With n_seqs = 1 and the most rows: for every call with up to as many rows."""
    return int(lib().hgf_cached_workspace_bytes(cache._ref, n_seqs, n_rows, n_heads))


def diff_attention_cached(cache: KVCache, q, slots, starts, lam: float, out_scale: float = 1.0, *, out=None, workspace=None, flags: int = 0,
                          stream=None):
    """hgf_diff_attention_cached: rows starts[i] .. starts[i + 1] - 1 of q (bf16 [n_rows][2 * n_heads * head_dim]), the last tokens of the sequence
    in slots[i], attend to what the cache holds of it -> out [n_rows][n_heads * head_dim], fp32 (bf16 with FLAG_OUT_BF16)."""
    if out is not None and workspace is not None and _native_cache and _done(
            "hgf_diff_attention_cached",
            _native_cache.diff_attention_cached(cache._at, cache._index, q, slots, starts, lam, out_scale, out, workspace, flags, stream)):
        return out
    _list(cache, slots, starts)
    assert q.dim() == 2, "q is a matrix"
    n, rows = slots.numel(), q.shape[0]
    heads = q.shape[1] // (2 * cache.head_dim)
    assert q.device == cache.device and q.dtype == torch.bfloat16 and q.is_contiguous() and q.shape[1] == 2 * heads * cache.head_dim and starts.numel() == n + 1
    dtype = torch.bfloat16 if flags & FLAG_OUT_BF16 else torch.float32
    if out is None or workspace is None:
        with _on(stream):
            out = torch.empty((rows, heads * cache.head_dim), dtype=dtype, device=q.device) if out is None else out
            workspace = torch.empty(cached_workspace_bytes(cache, n, rows, heads), dtype=torch.uint8, device=q.device) if workspace is None else workspace
    assert out.device == cache.device and out.dtype == dtype and out.is_contiguous() and out.shape == (rows, heads * cache.head_dim)
    assert workspace.device == cache.device and workspace.dtype == torch.uint8 and workspace.is_contiguous(), "the workspace is dense bytes on the cache's device"
    _check("hgf_diff_attention_cached",
           lib().hgf_diff_attention_cached(cache._ref, _ptr(q), rows, heads, _ptr(slots), _ptr(starts), n, lam, out_scale, _ptr(out), _ptr(workspace),
                                           workspace.numel(), flags, _stream(stream)))
    return out


def diff_lambda0(head_dim: float) -> float:
    return float(lib().hgf_diff_lambda0(float(head_dim)))


def selftest_wait_timeout(limit_us: int = 200, stream=None) -> None:
    """Enqueue the kernel whose bounded wait runs out (hgf_selftest_wait_timeout); the next check_status raises."""
    _check("hgf_selftest_wait_timeout", lib().hgf_selftest_wait_timeout(int(limit_us), _stream(stream)))


def tmax_tokens_per_s(bmem_bytes_per_s: float, params: float, bits: float) -> float:
    return float(lib().hgf_tmax_tokens_per_s(bmem_bytes_per_s, params, bits))


def launch_count() -> int:
    return int(lib().hgf_launch_count())
