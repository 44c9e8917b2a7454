"""Python binding of libvarlen_attn.so: argument marshalling only.

Attention: varlen_attn_fwd, varlen_attn_bwd, varlen_attn_merge.  Around it, on the same packed tokens: varlen_attn_rotary_positions,
varlen_attn_rotary_fwd and _bwd, varlen_attn_norm_fwd and _bwd, varlen_attn_act8_pack and _unpack (activations in 8 bits),
varlen_attn_bwd_act8 (attention's backward pass from them).

Forward, backward and merge are marshalled in native code (csrc/va_host.cpp) where that is built and nothing is unusual about the
call, else here.
Every step of the attention path runs in the library's HIP kernels.  PyTorch is used for device
memory (outputs, workspace) and for the current stream handle, nothing else.  There is no CPU or
eager fallback: if the library is missing or a call fails, this raises.
"""
import ctypes
import importlib.machinery
import importlib.util
import os
import subprocess
import threading
import warnings
from collections import namedtuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libvarlen_attn.so")
_lib = None
_host = None
_host_lock = threading.Lock()

VA_OK = 0
VA_ERR_BAD_CU_SEQLENS = 8


class VarlenAttnError(RuntimeError):
    def __init__(self, status, message):
        super().__init__(f"varlen_attn status {status}: {message}")
        self.status = status


class Params(ctypes.Structure):
    _fields_ = [("total_tokens", ctypes.c_int32), ("num_seqs", ctypes.c_int32),
                ("num_q_heads", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("causal", ctypes.c_int32),
                ("softmax_scale", ctypes.c_float), ("max_seqlen", ctypes.c_int32), ("kv_splits", ctypes.c_int32)]


class RotaryParams(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("total_tokens", "num_q_heads", "num_kv_heads", "head_dim", "num_pairs", "num_axes",
                                              "interleaved")] + \
               [(n, ctypes.c_int64) for n in ("q_stride", "k_stride", "v_stride", "q_out_stride", "k_out_stride", "v_out_stride")]


class Act8Tensor(ctypes.Structure):
    _fields_ = [("values", ctypes.c_void_p), ("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p),
                ("total_tokens", ctypes.c_int32), ("rows_per_token", ctypes.c_int32), ("channels", ctypes.c_int32),
                ("stride", ctypes.c_int64)]


class NormParams(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("total_tokens", "rows_per_token", "channels", "weight_type", "act8_format")] + \
               [("eps", ctypes.c_float)] + [(n, ctypes.c_int64) for n in ("x_stride", "dy_stride", "dx_stride")]


def load():
    """Load the C-ABI library (building it first only when no built library is present)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        from . import build as _build
        _build.build()
    lib = ctypes.CDLL(LIB_PATH)
    vp, sz = ctypes.c_void_p, ctypes.c_size_t
    pp = ctypes.POINTER(Params)
    lib.varlen_attn_fwd_workspace_bytes.argtypes = [pp]
    lib.varlen_attn_fwd_workspace_bytes.restype = sz
    lib.varlen_attn_bwd_workspace_bytes.argtypes = [pp]
    lib.varlen_attn_bwd_workspace_bytes.restype = sz
    lib.varlen_attn_max_work_items.argtypes = [pp, ctypes.c_int]
    lib.varlen_attn_max_work_items.restype = ctypes.c_int64
    lib.varlen_attn_fwd.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.varlen_attn_fwd.restype = ctypes.c_int
    lib.varlen_attn_fwd_static_scratch.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp]
    lib.varlen_attn_fwd_static_scratch.restype = ctypes.c_int
    lib.varlen_attn_bwd.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.varlen_attn_bwd.restype = ctypes.c_int
    lib.varlen_attn_merge.argtypes = [pp, ctypes.c_int32, vp, vp, vp, vp, vp]
    lib.varlen_attn_merge.restype = ctypes.c_int
    lib.varlen_attn_check_cu_seqlens.argtypes = [pp, vp, vp, sz, vp]
    lib.varlen_attn_check_cu_seqlens.restype = ctypes.c_int
    lib.varlen_attn_status_string.argtypes = [ctypes.c_int]
    lib.varlen_attn_status_string.restype = ctypes.c_char_p
    lib.varlen_attn_last_hip_error.argtypes = []
    lib.varlen_attn_last_hip_error.restype = ctypes.c_int
    lib.varlen_attn_balance_partition.argtypes = [vp, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                                  ctypes.c_double, ctypes.c_double, vp, vp]
    lib.varlen_attn_balance_partition.restype = ctypes.c_int
    lib.varlen_attn_profile_enable.argtypes = [ctypes.c_int]
    lib.varlen_attn_profile_enable.restype = ctypes.c_int
    lib.varlen_attn_profile_read.argtypes = [ctypes.c_int, ctypes.POINTER(ctypes.c_double),
                                             ctypes.POINTER(ctypes.c_int64)]
    lib.varlen_attn_profile_read.restype = ctypes.c_int
    lib.varlen_attn_profile_clock_probe.argtypes = [vp]
    lib.varlen_attn_profile_clock_probe.restype = ctypes.c_int
    i32 = ctypes.c_int32
    rp, ap, np_ = ctypes.POINTER(RotaryParams), ctypes.POINTER(Act8Tensor), ctypes.POINTER(NormParams)
    for name, args in (("rotary_positions", [i32, i32, i32, vp, vp, vp, vp, vp]), ("rotary_fwd", [rp, *[vp] * 10]),
                       ("rotary_bwd", [rp, *[vp] * 10]), ("act8_pack", [ap, i32, i32, vp]), ("act8_unpack", [ap, i32, i32, vp]),
                       ("bwd_act8", [pp, i32, *[vp] * 15, sz, vp]), ("norm_fwd", [np_, *[vp] * 11]),
                       ("norm_bwd", [np_, *[vp] * 12, sz, vp])):
        f = getattr(lib, "varlen_attn_" + name)
        f.argtypes, f.restype = args, ctypes.c_int
    for name, arg in (("bwd_act8", pp), ("norm_bwd", np_)):
        f = getattr(lib, f"varlen_attn_{name}_workspace_bytes")
        f.argtypes, f.restype = [arg], sz
    _lib = lib
    return lib


class _PythonHalf:
    """Stands where the native half should: leaves every call to the code below."""

    @staticmethod
    def fwd(*args):
        return NotImplemented

    bwd = merge = positions = rotary = act8_pack = act8_unpack = bwd_act8 = norm_fwd = norm_bwd = fwd


def _load_host():
    """The native half of this module, told where the library's entry points are (building it first only when it is not there).
    Without a compiler, torch's headers or a module that loads, the Python half does all of it, 4-6 us of host time a call slower."""
    global _host
    with _host_lock:
        if _host is not None:
            return _host
        lib = load()
        from . import build as _build
        try:
            path = _build.host_path()
            if not os.path.exists(path):
                _build.build_host()
            loader = importlib.machinery.ExtensionFileLoader("_varlen_attn_host", path)
            host = importlib.util.module_from_spec(importlib.util.spec_from_loader("_varlen_attn_host", loader))
            loader.exec_module(host)
        except (OSError, ImportError, subprocess.SubprocessError) as e:
            warnings.warn(f"the native half of the binding is not available ({e}); calls are marshalled in Python", RuntimeWarning,
                          stacklevel=3)
            host = _PythonHalf
        else:
            address = lambda f: ctypes.cast(f, ctypes.c_void_p).value  # noqa: E731
            host.bind(*map(address, (lib.varlen_attn_fwd_workspace_bytes, lib.varlen_attn_bwd_workspace_bytes, lib.varlen_attn_fwd,
                                     lib.varlen_attn_bwd, lib.varlen_attn_merge)))
            host.bind_block(*map(address, (lib.varlen_attn_rotary_positions, lib.varlen_attn_rotary_fwd, lib.varlen_attn_rotary_bwd,
                                           lib.varlen_attn_act8_pack, lib.varlen_attn_act8_unpack,
                                           lib.varlen_attn_bwd_act8_workspace_bytes, lib.varlen_attn_bwd_act8, lib.varlen_attn_norm_fwd,
                                           lib.varlen_attn_norm_bwd_workspace_bytes, lib.varlen_attn_norm_bwd)), Act8)
        _host = host
    return _host


def status_string(status):
    return load().varlen_attn_status_string(int(status)).decode()


def _check(status):
    if status != VA_OK:
        msg = status_string(status)
        if status == 6:
            msg += f" (hipError_t {load().varlen_attn_last_hip_error()})"
        raise VarlenAttnError(status, msg)


def make_params(total_tokens, num_seqs, num_q_heads, num_kv_heads, head_dim, causal, softmax_scale, kv_splits=0,
                max_seqlen=0):
    return Params(int(total_tokens), int(num_seqs), int(num_q_heads), int(num_kv_heads), int(head_dim),
                  int(bool(causal)), float(softmax_scale), int(max_seqlen), int(kv_splits))


def _params_of(q, k, cu_seqlens, causal, softmax_scale, kv_splits=0, max_seqlen=0):
    T, Hq, D = q.shape
    return make_params(T, cu_seqlens.numel() - 1, Hq, k.shape[1], D, causal, softmax_scale, kv_splits, max_seqlen)


def _require(t, dtype, name):
    if not (t.is_cuda and t.dtype == dtype and t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous {dtype} tensor on the GPU")


def _require_room(t, dtype, name, elements=0):
    """A caller's own buffer (or None): what the kernels write or read by its address alone.  It may be larger than needed or
    shaped otherwise, and in pinned host memory; dtype None: any (a workspace, of which one byte an element is counted on)."""
    if t is None:
        return
    if not ((t.is_cuda or t.is_pinned()) and (dtype is None or t.dtype == dtype) and t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous {'' if dtype is None else f'{dtype} '}tensor on the GPU")
    if t.numel() < elements:
        raise ValueError(f"{name} must hold at least {elements} elements")


def fwd_workspace_bytes(params):
    return int(load().varlen_attn_fwd_workspace_bytes(ctypes.byref(params)))


def bwd_workspace_bytes(params):
    return int(load().varlen_attn_bwd_workspace_bytes(ctypes.byref(params)))


def max_work_items(params, which=0):
    return int(load().varlen_attn_max_work_items(ctypes.byref(params), which))


def _stream_handle(stream):
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


class _Allocating:
    """Allocations for kernels on `stream`, made while this is entered.  They come from that stream's pool: a workspace goes
    back to it as soon as the call returns, with the kernels still to run, and what the current stream's pool hands out may be
    in use by work that is still queued there.  result(t): t is the caller's, who uses it on the current stream and may drop it
    with such work queued."""

    def __init__(self, stream, device):
        self._user = None
        if stream is not None:
            current = torch.cuda.current_stream(device)
            if stream.cuda_stream != current.cuda_stream:
                self._user = current
                self._pool = torch.cuda.stream(stream if isinstance(stream, torch.cuda.Stream) else
                                               torch.cuda.ExternalStream(stream.cuda_stream, device=device))

    def __enter__(self):
        if self._user is not None:
            self._pool.__enter__()
        return self

    def __exit__(self, *error):
        if self._user is not None:
            self._pool.__exit__(*error)

    def result(self, t):
        if self._user is not None:
            t.record_stream(self._user)
        return t


def varlen_attn_fwd(q, k, v, cu_seqlens, causal, softmax_scale, out=None, lse=None, workspace=None,
                    stream=None, kv_splits=0, max_seqlen=0):
    """O bf16 [T,Hq,D] and LSE fp32 [Hq,T] of packed attention; asynchronous on the stream (default: the current one; the
    inputs must be ready there, and what is not given is allocated from its pool).
    kv_splits: 0 automatic, 1 never, 2..8 workgroups sharing the keys of each query tile.
    max_seqlen: 0 unknown, else the caller's promise that no sample is longer (a hint).
    out, lse, workspace: the caller's own buffers, contiguous, large enough, of any shape."""
    done = (_host or _load_host()).fwd(q, k, v, cu_seqlens, bool(causal), float(softmax_scale), out, lse, workspace,
                                       None if stream is None else stream.cuda_stream, int(kv_splits), int(max_seqlen))
    if type(done) is tuple:
        return done
    if done is not NotImplemented:
        _check(done)
    lib = load()
    for t, n in ((q, "q"), (k, "k"), (v, "v")):
        _require(t, torch.bfloat16, n)
    _require(cu_seqlens, torch.int32, "cu_seqlens")
    p = _params_of(q, k, cu_seqlens, causal, softmax_scale, kv_splits, max_seqlen)
    if k.shape != v.shape or k.shape[0] != q.shape[0] or k.shape[2] != q.shape[2]:
        raise ValueError("k and v must be [T, Hkv, D] matching q's T and D")
    _require_room(out, torch.bfloat16, "out", q.numel())
    _require_room(lse, torch.float32, "lse", q.shape[0] * q.shape[1])
    _require_room(workspace, None, "workspace")
    with _Allocating(stream, q.device) as a:
        if out is None:
            out = a.result(torch.empty_like(q))
        if lse is None:
            lse = a.result(torch.empty((q.shape[1], q.shape[0]), dtype=torch.float32, device=q.device))
        if workspace is None:
            workspace = torch.empty(max(fwd_workspace_bytes(p), 16), dtype=torch.uint8, device=q.device)
    _check(lib.varlen_attn_fwd(ctypes.byref(p), q.data_ptr(), k.data_ptr(), v.data_ptr(),
                               cu_seqlens.data_ptr(), out.data_ptr(), lse.data_ptr(),
                               workspace.data_ptr(), workspace.numel(), _stream_handle(stream)))
    return out, lse


STATIC_SCRATCH_BYTES = 32 << 20
VA_ERR_SCRATCH_LIMIT = 9


def varlen_attn_fwd_static_scratch(q, k, v, cu_seqlens, causal, softmax_scale, out, lse, stream=None, kv_splits=0,
                                   max_seqlen=0):
    """varlen_attn_fwd without a workspace: the scratch lives in a static device array of the library.  The
    caller passes the outputs; nothing is allocated here or in the library."""
    lib = load()
    for t, n in ((q, "q"), (k, "k"), (v, "v"), (out, "out")):
        _require(t, torch.bfloat16, n)
    _require(lse, torch.float32, "lse")
    _require(cu_seqlens, torch.int32, "cu_seqlens")
    if k.shape != v.shape or k.shape[0] != q.shape[0] or k.shape[2] != q.shape[2] or out.shape != q.shape:
        raise ValueError("k and v must be [T, Hkv, D] matching q's T and D; out must match q")
    if tuple(lse.shape) != (q.shape[1], q.shape[0]):
        raise ValueError("lse must be [Hq, T]")
    p = _params_of(q, k, cu_seqlens, causal, softmax_scale, kv_splits, max_seqlen)
    _check(lib.varlen_attn_fwd_static_scratch(ctypes.byref(p), q.data_ptr(), k.data_ptr(), v.data_ptr(),
                                              cu_seqlens.data_ptr(), out.data_ptr(), lse.data_ptr(),
                                              _stream_handle(stream)))
    return out, lse


def varlen_attn_bwd(dout, q, k, v, out, lse, cu_seqlens, causal, softmax_scale, dq=None, dk=None,
                    dv=None, workspace=None, stream=None, max_seqlen=0, kv_splits=0):
    """dQ, dK, dV (bf16) from dO and the forward's saved O and LSE; asynchronous on the stream (as varlen_attn_fwd).
    max_seqlen: 0 unknown, else the caller's promise that no sample is longer (a hint; above 1024 a launch too small
    to fill the GPU may cut its tiles into chunks, so that a sample's gradients depend, to rounding, on the launch).
    kv_splits: 1 never does, 0 automatic.
    dq, dk, dv, workspace: the caller's own buffers, contiguous, large enough, of any shape."""
    done = (_host or _load_host()).bwd(dout, q, k, v, out, lse, cu_seqlens, bool(causal), float(softmax_scale), dq, dk, dv,
                                       workspace, None if stream is None else stream.cuda_stream, int(kv_splits),
                                       int(max_seqlen))
    if type(done) is tuple:
        return done
    if done is not NotImplemented:
        _check(done)
    lib = load()
    for t, n in ((dout, "dout"), (q, "q"), (k, "k"), (v, "v"), (out, "out")):
        _require(t, torch.bfloat16, n)
    _require(lse, torch.float32, "lse")
    _require(cu_seqlens, torch.int32, "cu_seqlens")
    p = _params_of(q, k, cu_seqlens, causal, softmax_scale, kv_splits, max_seqlen)
    if dout.shape != q.shape or out.shape != q.shape or k.shape != v.shape:
        raise ValueError("dout and out must match q; k must match v")
    if k.dim() != 3 or k.shape[0] != q.shape[0] or k.shape[2] != q.shape[2]:
        raise ValueError("k and v must be [T, Hkv, D] matching q's T and D")
    _require_room(lse, torch.float32, "lse", q.shape[0] * q.shape[1])
    for t, like, n in ((dq, q, "dq"), (dk, k, "dk"), (dv, v, "dv")):
        _require_room(t, torch.bfloat16, n, like.numel())
    _require_room(workspace, None, "workspace")
    with _Allocating(stream, q.device) as a:
        dq = a.result(torch.empty_like(q)) if dq is None else dq
        dk = a.result(torch.empty_like(k)) if dk is None else dk
        dv = a.result(torch.empty_like(v)) if dv is None else dv
        if workspace is None:
            workspace = torch.empty(max(bwd_workspace_bytes(p), 16), dtype=torch.uint8, device=q.device)
    _check(lib.varlen_attn_bwd(ctypes.byref(p), dout.data_ptr(), q.data_ptr(), k.data_ptr(),
                               v.data_ptr(), out.data_ptr(), lse.data_ptr(), cu_seqlens.data_ptr(),
                               dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), workspace.data_ptr(),
                               workspace.numel(), _stream_handle(stream)))
    return dq, dk, dv


KERNELS = {"sched": 0, "fwd": 1, "dkdv": 2, "dq": 3, "merge": 4, "rotary": 5, "norm": 6, "act8": 7}


def profile_enable(on=True):
    _check(load().varlen_attn_profile_enable(int(bool(on))))


def profile_read():
    """{kernel name: (total milliseconds, launches)} of the launches recorded since profile_enable."""
    out = {}
    for name, kid in KERNELS.items():
        ms, n = ctypes.c_double(0.0), ctypes.c_int64(0)
        _check(load().varlen_attn_profile_read(kid, ctypes.byref(ms), ctypes.byref(n)))
        out[name] = (ms.value, n.value)
    return out


def profile_clock_probe(counters):
    """Attach a zeroed int64 device tensor of 6 counters as the shader-clock probe, or None to detach."""
    if counters is not None and (counters.dtype != torch.int64 or counters.numel() < 6 or not counters.is_cuda
                                 or not counters.is_contiguous()):
        raise ValueError("counters must be a contiguous int64 device tensor of at least 6 elements")
    _check(load().varlen_attn_profile_clock_probe(None if counters is None else counters.data_ptr()))


def varlen_attn_merge(o_parts, lse_parts, out=None, lse=None, stream=None):
    """Merge partial results over key shards: o_parts bf16 [P,T,Hq,D], lse_parts fp32 [P,Hq,T]."""
    done = (_host or _load_host()).merge(o_parts, lse_parts, out, lse, None if stream is None else stream.cuda_stream)
    if type(done) is tuple:
        return done
    if done is not NotImplemented:
        _check(done)
    _require(o_parts, torch.bfloat16, "o_parts")
    _require(lse_parts, torch.float32, "lse_parts")
    P, T, Hq, D = o_parts.shape
    if tuple(lse_parts.shape) != (P, Hq, T):
        raise ValueError("lse_parts must be [P, Hq, T]")
    _require_room(out, torch.bfloat16, "out", T * Hq * D)
    _require_room(lse, torch.float32, "lse", T * Hq)
    p = make_params(T, 1, Hq, Hq, D, False, 1.0)
    with _Allocating(stream, o_parts.device) as a:
        if out is None:
            out = a.result(torch.empty((T, Hq, D), dtype=torch.bfloat16, device=o_parts.device))
        if lse is None:
            lse = a.result(torch.empty((Hq, T), dtype=torch.float32, device=o_parts.device))
    _check(load().varlen_attn_merge(ctypes.byref(p), P, o_parts.data_ptr(), lse_parts.data_ptr(), out.data_ptr(),
                                    lse.data_ptr(), _stream_handle(stream)))
    return out, lse


# ---- around attention: rotary positions, layer norm, activations in 8 bits --------------------------------------------------

Act8 = namedtuple("Act8", ["codes", "scales"])
Act8.__doc__ = """A tensor in 8 bits: codes (torch.int8 or torch.float8_e4m3fn, the tensor's shape) and their fp32 scales, one for each
ACT8_BLOCK channels of a row (the shape without the last dimension, and the number of blocks)."""
NormForward = namedtuple("NormForward", ["out", "mean", "rstd", "summed", "saved"])

ACT8_BLOCK = 128
_ACT8_FORMATS = {"int8": (0, torch.int8), "e4m3": (1, torch.float8_e4m3fn)}
_ACT8_OF_TYPE = {torch.int8: 0, torch.float8_e4m3fn: 1}
_WEIGHT_TYPES = {torch.bfloat16: 0, torch.float32: 1}


def _done(answer):
    """Whether the native half has done the call: an answer that is not NotImplemented, nor a status, which is raised."""
    if type(answer) is int:
        _check(answer)
    return answer is not NotImplemented


class _On:
    """Everything a call is given has to be on one GPU, which is made the current one for it."""

    def __init__(self, first, stream, /, **tensors):
        for name, t in tensors.items():
            if t is not None and t.device != first.device:
                raise ValueError(f"{name} must be on {first.device}")
        self._guard = torch.cuda.device(first.device)
        self._stream, self._device = stream, first.device

    def __enter__(self):
        self._guard.__enter__()
        s = torch.cuda.current_stream(self._device) if self._stream is None else self._stream
        self.stream = ctypes.c_void_p(s.cuda_stream)
        self._alloc = _Allocating(self._stream, self._device)
        self._alloc.__enter__()
        return self

    def __exit__(self, *error):
        self._alloc.__exit__(*error)
        self._guard.__exit__(*error)

    def empty(self, shape, dtype):
        return self._alloc.result(torch.empty(shape, dtype=dtype, device=self._device))

    def scratch(self, n):
        return torch.empty(max(n, 16), dtype=torch.uint8, device=self._device)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _if_on_gpu(t):
    """A caller's own buffer, or None for one in pinned host memory (see _require_room), which is on no GPU."""
    return t if t is not None and t.is_cuda else None


def _require_32_bits(**sizes):
    """Sizes go to the library as 32-bit numbers, into which ctypes puts the low half of a larger one without a word."""
    for name, n in sizes.items():
        if not -2 ** 31 <= n < 2 ** 31:
            raise ValueError(f"{name} must be below 2^31")


def _token_stride(t, name, dims=(3,)):
    """Elements from one token to the next of a bf16 tensor [T, H, D] (or [T, C]) on the GPU, whose channels (and heads) lie side by
    side: contiguous, or a part of a wider tensor."""
    if not (t.is_cuda and t.dtype == torch.bfloat16 and t.dim() in dims):
        raise ValueError(f"{name} must be a torch.bfloat16 tensor of {' or '.join(map(str, dims))} dimensions on the GPU")
    shape, strides = t.shape, t.stride()
    _require_32_bits(**{f"{name}'s every size": max(shape)})
    width = shape[1] if t.dim() == 2 else shape[1] * shape[2]
    if t.numel() == 0:
        return width
    if (shape[-1] > 1 and strides[-1] != 1) or (t.dim() == 3 and shape[1] > 1 and strides[1] != shape[2]) or \
            (shape[0] > 1 and strides[0] < width):
        raise ValueError(f"{name} must hold a token's channels side by side")
    return strides[0] if shape[0] > 1 else width


def _out_like(t, shape, name):
    """A caller's own output tensor: of this shape."""
    if t is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have the shape {tuple(shape)}")


def varlen_attn_rotary_positions(cu_rows, grids, total_tokens, first=None, merge=1, out=None, stream=None):
    """Positions int32 [3, total_tokens] (time, height, width) of packed text, images and video; asynchronous on the stream.
    Segment s holds the tokens [cu_rows[s], cu_rows[s + 1]); grids int32 [S, 3] its time, height and width in patches, laid out in blocks of
    merge x merge (height or width 0: text, whose tokens count up on all axes); first int32 [S]: added to a segment's positions."""
    if stream is None and out is None:
        answer = (_host or _load_host()).positions(cu_rows, grids, total_tokens, first, merge)
        if _done(answer):
            return answer
    for t, n in ((cu_rows, "cu_rows"), (grids, "grids"), (first, "first"), (out, "out")):
        if t is not None:
            _require(t, torch.int32, n)
    segments = cu_rows.numel() - 1
    _require_32_bits(total_tokens=int(total_tokens), merge=int(merge), **{"cu_rows' size": segments})
    if cu_rows.dim() != 1 or segments < 0 or tuple(grids.shape) != (segments, 3):
        raise ValueError("grids must be [S, 3] for the S + 1 elements of cu_rows")
    if first is not None and first.numel() != segments:
        raise ValueError("first must be [S]")
    _out_like(out, (3, int(total_tokens)), "out")
    with _On(cu_rows, stream, grids=grids, first=first, out=out) as on:
        out = on.empty((3, int(total_tokens)), torch.int32) if out is None else out
        _check(load().varlen_attn_rotary_positions(int(total_tokens), segments, int(merge), cu_rows.data_ptr(), grids.data_ptr(),
                                                   _ptr(first), out.data_ptr(), on.stream))
    return out


def _rotary(inverse, names, q, k, v, positions, inv_freq, pair_axis, interleaved, q_out, k_out, v_out, stream):
    if stream is None:
        answer = (_host or _load_host()).rotary(inverse, q, k, v, positions, inv_freq, pair_axis, bool(interleaved), q_out, k_out, v_out)
        if _done(answer):
            return answer
    ins, outs = dict(zip(names, (q, k, v))), dict(zip((n + "_out" for n in names), (q_out, k_out, v_out)))
    strides = [0 if t is None else _token_stride(t, n) for n, t in ins.items()]
    if k.shape[0] != q.shape[0] or k.shape[2] != q.shape[2]:
        raise ValueError(f"{names[1]} must be [T, Hkv, D] matching {names[0]}'s T and D")
    if v is not None and v.shape != k.shape:
        raise ValueError(f"{names[2]} must match {names[1]}")
    if v is None and v_out is not None:
        raise ValueError(f"{names[2]} must be given with {names[2]}_out")
    _require(positions, torch.int32, "positions")
    _require(inv_freq, torch.float32, "inv_freq")
    _require(pair_axis, torch.int32, "pair_axis")
    if positions.dim() != 2 or positions.shape[1] != q.shape[0]:
        raise ValueError("positions must be [axes, T]")
    if inv_freq.dim() != 1 or pair_axis.shape != inv_freq.shape:
        raise ValueError("pair_axis must match inv_freq")
    _require_32_bits(axes=positions.shape[0], pairs=inv_freq.numel())
    for (n, t), like in zip(outs.items(), (q, k, v)):
        if t is not None:
            _out_like(t, like.shape, n)
    out_strides = [0 if like is None else _token_stride(t, n) if t is not None else like.shape[1] * like.shape[2]
                   for (n, t), like in zip(outs.items(), (q, k, v))]
    p = RotaryParams(q.shape[0], q.shape[1], k.shape[1], q.shape[2], inv_freq.numel(), positions.shape[0], int(bool(interleaved)),
                     *strides, *out_strides)
    with _On(q, stream, **ins, **outs, positions=positions, inv_freq=inv_freq, pair_axis=pair_axis) as on:
        made = [like if like is None else on.empty(like.shape, torch.bfloat16) if t is None else t
                for t, like in zip((q_out, k_out, v_out), (q, k, v))]
        f = load().varlen_attn_rotary_bwd if inverse else load().varlen_attn_rotary_fwd
        _check(f(ctypes.byref(p), q.data_ptr(), k.data_ptr(), _ptr(v), positions.data_ptr(), inv_freq.data_ptr(),
                 pair_axis.data_ptr(), *map(_ptr, made), on.stream))
    return tuple(made[:2] if v is None else made)


def varlen_attn_rotary_fwd(q, k, positions, inv_freq, pair_axis, v=None, interleaved=False, q_out=None, k_out=None, v_out=None,
                           stream=None):
    """q and k turned by their tokens' positions, as (q, k), or (q, k, v) with v copied along; asynchronous on the stream.
    q [T, Hq, D], k and v [T, Hkv, D]: bf16, contiguous or parts of the fused projection [T, Hq + 2 Hkv, D].
    positions int32 [axes, T]; inv_freq fp32 [P] and pair_axis int32 [P]: frequency and axis of each pair of channels, (j, j + P), or
    (2j, 2j + 1) if interleaved; channels from 2P on are copied.
    q_out, k_out, v_out: the caller's own tensors of the same shapes, contiguous or parts too; each may be its own input."""
    return _rotary(False, ("q", "k", "v"), q, k, v, positions, inv_freq, pair_axis, interleaved, q_out, k_out, v_out, stream)


def varlen_attn_rotary_bwd(dq, dk, positions, inv_freq, pair_axis, dv=None, interleaved=False, dq_out=None, dk_out=None, dv_out=None,
                           stream=None):
    """The gradients of varlen_attn_rotary_fwd's inputs from those of its outputs; arguments as there."""
    return _rotary(True, ("dq", "dk", "dv"), dq, dk, dv, positions, inv_freq, pair_axis, interleaved, dq_out, dk_out, dv_out, stream)


def _act8_shape(shape):
    return (*shape[:-1], (shape[-1] + ACT8_BLOCK - 1) // ACT8_BLOCK)


def _check_act8(x, name):
    """Format, tokens, rows a token and channels of an Act8."""
    if not isinstance(x, Act8):
        raise ValueError(f"{name} must be an Act8 (codes, scales)")
    codes, scales = x
    if not (codes.is_cuda and codes.dtype in _ACT8_OF_TYPE and codes.is_contiguous() and codes.dim() in (2, 3)):
        raise ValueError(f"{name}.codes must be a contiguous torch.int8 or torch.float8_e4m3fn tensor of 2 or 3 dimensions on the GPU")
    _require_32_bits(**{f"{name}.codes' every size": max(codes.shape)})
    _require(scales, torch.float32, f"{name}.scales")
    if tuple(scales.shape) != _act8_shape(codes.shape) or scales.device != codes.device:
        raise ValueError(f"{name}.scales must be {_act8_shape(codes.shape)} on {codes.device}")
    return _ACT8_OF_TYPE[codes.dtype]


def _act8_tensor(values, stride, codes, scales):
    shape = codes.shape
    return Act8Tensor(values.data_ptr(), codes.data_ptr(), scales.data_ptr(), shape[0], 1 if len(shape) == 2 else shape[1], shape[-1],
                      stride)


def varlen_attn_act8_pack(tensors, format="int8", out=None, stream=None):
    """bf16 tensors [T, C] or [T, H, C] (contiguous or parts of wider ones) in 8 bits, a list of Act8; asynchronous on the stream.
    format: "int8" or "e4m3".  One launch for up to 8 tensors.  out: Act8s of the caller's own."""
    if format not in _ACT8_FORMATS:
        raise ValueError("format must be int8 or e4m3")
    number, code_type = _ACT8_FORMATS[format]
    tensors = list(tensors)
    if stream is None and out is None:
        answer = (_host or _load_host()).act8_pack(tensors, number)
        if _done(answer):
            return answer
    strides = [_token_stride(t, f"tensors[{i}]", (2, 3)) for i, t in enumerate(tensors)]
    if out is not None:
        out = list(out)
        if len(out) != len(tensors):
            raise ValueError("out must match tensors")
        for i, (t, o) in enumerate(zip(tensors, out)):
            if _check_act8(o, f"out[{i}]") != number or o.codes.shape != t.shape:
                raise ValueError(f"out[{i}] must match tensors[{i}] and the format")
    if not tensors:
        return []
    given = {} if out is None else {f"out[{i}]": o.codes for i, o in enumerate(out)}
    with _On(tensors[0], stream, **{f"tensors[{i}]": t for i, t in enumerate(tensors)}, **given) as on:
        if out is None:
            out = [Act8(on.empty(t.shape, code_type), on.empty(_act8_shape(t.shape), torch.float32)) for t in tensors]
        for at in range(0, len(tensors), 8):
            part = [_act8_tensor(t, s, *o) for t, s, o in zip(tensors[at:at + 8], strides[at:at + 8], out[at:at + 8])]
            _check(load().varlen_attn_act8_pack((Act8Tensor * len(part))(*part), len(part), number, on.stream))
    return out


def varlen_attn_act8_unpack(packed, out=None, stream=None):
    """The bf16 tensors that a list of Act8 stands for; asynchronous on the stream.
    out: the caller's own tensors of the same shapes, contiguous or parts of wider ones."""
    packed = list(packed)
    if stream is None and out is None:
        answer = (_host or _load_host()).act8_unpack(packed)
        if _done(answer):
            return answer
    formats = [_check_act8(x, f"packed[{i}]") for i, x in enumerate(packed)]
    if len(set(formats)) > 1:
        raise ValueError("packed must be of one format")
    if out is not None:
        out = list(out)
        if len(out) != len(packed):
            raise ValueError("out must match packed")
        for i, (x, o) in enumerate(zip(packed, out)):
            _out_like(o, x.codes.shape, f"out[{i}]")
    if not packed:
        return []
    strides = [x.codes[0].numel() if x.codes.shape[0] else 1 << 30 for x in packed] if out is None else \
        [_token_stride(o, f"out[{i}]", (2, 3)) for i, o in enumerate(out)]
    given = {} if out is None else {f"out[{i}]": o for i, o in enumerate(out)}
    with _On(packed[0].codes, stream, **{f"packed[{i}]": x.codes for i, x in enumerate(packed)}, **given) as on:
        if out is None:
            out = [on.empty(x.codes.shape, torch.bfloat16) for x in packed]
        for at in range(0, len(packed), 8):
            part = [_act8_tensor(o, s, *x) for x, s, o in zip(packed[at:at + 8], strides[at:at + 8], out[at:at + 8])]
            _check(load().varlen_attn_act8_unpack((Act8Tensor * len(part))(*part), len(part), formats[0], on.stream))
    return out


def bwd_act8_workspace_bytes(params):
    return int(load().varlen_attn_bwd_act8_workspace_bytes(ctypes.byref(params)))


def varlen_attn_bwd_act8(dout, q, k, v, out, lse, cu_seqlens, causal, softmax_scale, dq=None, dk=None, dv=None, workspace=None,
                         stream=None, max_seqlen=0, kv_splits=0):
    """varlen_attn_bwd with q, k, v and out in 8 bits (Act8s of one format, from varlen_attn_act8_pack); the other arguments as there."""
    if stream is None:
        answer = (_host or _load_host()).bwd_act8(dout, q, k, v, out, lse, cu_seqlens, bool(causal), float(softmax_scale), dq, dk, dv,
                                                  workspace, int(kv_splits), int(max_seqlen))
        if _done(answer):
            return answer
    _require(dout, torch.bfloat16, "dout")
    formats = {_check_act8(x, n) for x, n in ((q, "q"), (k, "k"), (v, "v"), (out, "out"))}
    if len(formats) > 1:
        raise ValueError("q, k, v and out must be of one format")
    _require(lse, torch.float32, "lse")
    _require(cu_seqlens, torch.int32, "cu_seqlens")
    qs, ks = q.codes.shape, k.codes.shape
    if dout.dim() != 3 or dout.shape != qs or out.codes.shape != qs:
        raise ValueError("dout and out must match q")
    if len(ks) != 3 or v.codes.shape != ks or ks[0] != qs[0] or ks[2] != qs[2]:
        raise ValueError("k and v must be [T, Hkv, D] matching q's T and D")
    _require_room(lse, torch.float32, "lse", qs[0] * qs[1])
    for t, shape, n in ((dq, qs, "dq"), (dk, ks, "dk"), (dv, ks, "dv")):
        _require_room(t, torch.bfloat16, n, shape.numel())
    _require_room(workspace, None, "workspace")
    _require_32_bits(kv_splits=int(kv_splits), **{"cu_seqlens' size": cu_seqlens.numel()})
    p = _params_of(q.codes, k.codes, cu_seqlens, causal, softmax_scale, kv_splits, min(int(max_seqlen), 2 ** 31 - 1))
    with _On(dout, stream, q=q.codes, k=k.codes, v=v.codes, out=out.codes, lse=lse, cu_seqlens=cu_seqlens, dq=_if_on_gpu(dq),
             dk=_if_on_gpu(dk), dv=_if_on_gpu(dv), workspace=_if_on_gpu(workspace)) as on:
        dq = on.empty(qs, torch.bfloat16) if dq is None else dq
        dk = on.empty(ks, torch.bfloat16) if dk is None else dk
        dv = on.empty(ks, torch.bfloat16) if dv is None else dv
        if workspace is None:
            workspace = on.scratch(bwd_act8_workspace_bytes(p))
        _check(load().varlen_attn_bwd_act8(ctypes.byref(p), formats.pop(), dout.data_ptr(),
                                           *(t.data_ptr() for x in (q, k, v, out) for t in x), lse.data_ptr(), cu_seqlens.data_ptr(),
                                           dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), workspace.data_ptr(), workspace.numel(),
                                           on.stream))
    return dq, dk, dv


def _check_weights(weight, bias, channels):
    if bias is not None and weight is None:
        raise ValueError("weight must be given with bias")
    for t, n in ((weight, "weight"), (bias, "bias")):
        if t is None:
            continue
        if not (t.is_cuda and t.dtype in _WEIGHT_TYPES and t.is_contiguous() and tuple(t.shape) == (channels,)):
            raise ValueError(f"{n} must be a contiguous torch.bfloat16 or torch.float32 tensor [{channels}] on the GPU")
    if bias is not None and bias.dtype != weight.dtype:
        raise ValueError("bias must have weight's type")
    return 0 if weight is None else _WEIGHT_TYPES[weight.dtype]


def _statistics_like(t, shape, name):
    if t is not None:
        _require(t, torch.float32, name)
        _out_like(t, shape[:-1], name)


def _contiguous_like(t, shape, name):
    if t is not None:
        _require(t, torch.bfloat16, name)
        _out_like(t, shape, name)


def _norm_params(shape, weight_type, act8_format, eps, x_stride=0, dy_stride=0, dx_stride=0):
    return NormParams(shape[0], 1 if len(shape) == 2 else shape[1], shape[-1], weight_type, act8_format, float(eps), x_stride, dy_stride,
                      dx_stride)


def varlen_attn_norm_fwd(x, weight=None, bias=None, eps=1e-5, residual=None, save=None, out=None, mean=None, rstd=None, summed=None,
                         saved=None, stream=None):
    """Layer norm over the last dimension of x, bf16 [T, C] or [T, H, C] (contiguous or a part of a wider tensor): a NormForward
    (out bf16, mean and rstd fp32 [T] or [T, H], summed, saved); asynchronous on the stream.
    weight, bias: bf16 or fp32 [C], or None.  residual: contiguous, x's shape; the norm is then of summed = bf16(x + residual).
    save: "int8" or "e4m3": what is normed is left in 8 bits too (saved, an Act8), for varlen_attn_norm_bwd.
    out, mean, rstd, summed (with residual), saved (with save, an Act8): the caller's own, contiguous, of those shapes."""
    if save is not None and save not in _ACT8_FORMATS:
        raise ValueError("save must be int8 or e4m3")
    number, code_type = _ACT8_FORMATS[save or "int8"]
    if stream is None and mean is None and rstd is None and summed is None and saved is None:
        answer = (_host or _load_host()).norm_fwd(x, weight, bias, float(eps), residual, number if save else None, out)
        if _done(answer):
            return NormForward._make(answer)
    stride = _token_stride(x, "x", (2, 3))
    shape = x.shape
    _contiguous_like(residual, shape, "residual")
    _contiguous_like(out, shape, "out")
    _contiguous_like(summed, shape, "summed")
    _statistics_like(mean, shape, "mean")
    _statistics_like(rstd, shape, "rstd")
    if summed is not None and residual is None:
        raise ValueError("residual must be given with summed")
    if saved is not None and (save is None or _check_act8(saved, "saved") != number or saved.codes.shape != shape):
        raise ValueError("saved must match x and save")
    p = _norm_params(shape, _check_weights(weight, bias, shape[-1]), number, eps, x_stride=stride)
    with _On(x, stream, weight=weight, bias=bias, residual=residual, out=out, mean=mean, rstd=rstd, summed=summed,
             saved=None if saved is None else saved.codes) as on:
        out = on.empty(shape, torch.bfloat16) if out is None else out
        mean = on.empty(shape[:-1], torch.float32) if mean is None else mean
        rstd = on.empty(shape[:-1], torch.float32) if rstd is None else rstd
        if residual is not None and summed is None:
            summed = on.empty(shape, torch.bfloat16)
        if save is not None and saved is None:
            saved = Act8(on.empty(shape, code_type), on.empty(_act8_shape(shape), torch.float32))
        codes, scales = saved or (None, None)
        _check(load().varlen_attn_norm_fwd(ctypes.byref(p), x.data_ptr(), _ptr(residual), _ptr(weight), _ptr(bias), out.data_ptr(),
                                           _ptr(summed), mean.data_ptr(), rstd.data_ptr(), _ptr(codes), _ptr(scales), on.stream))
    return NormForward(out, mean, rstd, summed, saved)


def norm_bwd_workspace_bytes(params):
    return int(load().varlen_attn_norm_bwd_workspace_bytes(ctypes.byref(params)))


def varlen_attn_norm_bwd(dy, x, mean, rstd, weight=None, dsummed=None, dx=None, dweight=None, dbias=None, workspace=None, stream=None):
    """(dx bf16, dweight fp32, dbias fp32; the last two None without weight) of varlen_attn_norm_fwd; asynchronous on the stream.
    x: what was normed: the forward's x, its summed where it had a residual, or its saved Act8.  mean, rstd: the forward's.
    dsummed: the gradient that reaches summed on its own way, added to dx (which is the gradient of x and of residual).
    dy, x and dx may be parts of wider tensors; dx, dweight and dbias (with weight), workspace: the caller's own."""
    if stream is None and dweight is None and dbias is None and workspace is None:
        answer = (_host or _load_host()).norm_bwd(dy, x, mean, rstd, weight, dsummed, dx)
        if _done(answer):
            return answer
    dy_stride = _token_stride(dy, "dy", (2, 3))
    shape, packed = dy.shape, isinstance(x, Act8)
    number = _check_act8(x, "x") if packed else 0
    x_stride = 0 if packed else _token_stride(x, "x", (2, 3))
    if (x.codes if packed else x).shape != shape:
        raise ValueError("x must match dy")
    for t, n in ((mean, "mean"), (rstd, "rstd")):
        _require(t, torch.float32, n)
        _out_like(t, shape[:-1], n)
    for t, n in ((dweight, "dweight"), (dbias, "dbias")):
        if t is not None and weight is None:
            raise ValueError(f"weight must be given with {n}")
        if t is not None:
            _require(t, torch.float32, n)
            _out_like(t, shape[-1:], n)
    _contiguous_like(dsummed, shape, "dsummed")
    dx_stride = shape[1:].numel()
    if dx is not None:
        dx_stride = _token_stride(dx, "dx", (2, 3))
        _out_like(dx, shape, "dx")
    _require_room(workspace, None, "workspace")
    p = _norm_params(shape, _check_weights(weight, None, shape[-1]), number, 0.0, x_stride, dy_stride, dx_stride)
    codes, scales = x if packed else (None, None)
    with _On(dy, stream, x=x.codes if packed else x, mean=mean, rstd=rstd, weight=weight, dsummed=dsummed, dx=dx, dweight=dweight,
             dbias=dbias, workspace=_if_on_gpu(workspace)) as on:
        dx = on.empty(shape, torch.bfloat16) if dx is None else dx
        if weight is not None:
            dweight = on.empty(shape[-1:], torch.float32) if dweight is None else dweight
            dbias = on.empty(shape[-1:], torch.float32) if dbias is None else dbias
            if workspace is None:
                workspace = on.scratch(norm_bwd_workspace_bytes(p))
        _check(load().varlen_attn_norm_bwd(ctypes.byref(p), dy.data_ptr(), None if packed else x.data_ptr(), _ptr(codes), _ptr(scales),
                                           mean.data_ptr(), rstd.data_ptr(), _ptr(weight), _ptr(dsummed), dx.data_ptr(), _ptr(dweight),
                                           _ptr(dbias), _ptr(workspace), 0 if workspace is None else workspace.numel(), on.stream))
    return dx, dweight, dbias


def check_cu_seqlens(cu_seqlens, total_tokens, stream=None):
    """True if the device array obeys cu[0] = 0, non-decreasing, cu[-1] = total_tokens.  Synchronises the stream."""
    _require(cu_seqlens, torch.int32, "cu_seqlens")
    p = make_params(total_tokens, cu_seqlens.numel() - 1, 1, 1, 64, False, 1.0)
    with _Allocating(stream, cu_seqlens.device):
        ws = torch.empty(16, dtype=torch.uint8, device=cu_seqlens.device)
    rc = load().varlen_attn_check_cu_seqlens(ctypes.byref(p), cu_seqlens.data_ptr(), ws.data_ptr(), ws.numel(),
                                             _stream_handle(stream))
    if rc == VA_ERR_BAD_CU_SEQLENS:
        return False
    _check(rc)
    return True


PARTITION_KARMARKAR_KARP = 0
PARTITION_LPT = 1


def balance_partition(lengths, bins, method=PARTITION_KARMARKAR_KARP, equal_counts=False, lin_cost=0.0,
                      quad_cost=1.0):
    """Host-side: bin of every sample and the summed cost per bin (numpy arrays)."""
    import numpy as np
    lengths = np.ascontiguousarray(lengths, dtype=np.int32)
    bin_of = np.zeros(lengths.size, dtype=np.int32)
    bin_cost = np.zeros(max(int(bins), 0), dtype=np.float64)
    _check(load().varlen_attn_balance_partition(
        lengths.ctypes.data_as(ctypes.c_void_p), lengths.size, int(bins), int(method), int(bool(equal_counts)),
        float(lin_cost), float(quad_cost), bin_of.ctypes.data_as(ctypes.c_void_p),
        bin_cost.ctypes.data_as(ctypes.c_void_p)))
    return bin_of, bin_cost
