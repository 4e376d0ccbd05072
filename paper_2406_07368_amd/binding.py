"""ctypes binding of liblinattn.so: argument marshalling only.

Every call has the name and argument order of its declaration in ``include/linattn.h``.
Tensors are torch tensors on the GPU (torch is used for device memory and
streams, nothing else); every arithmetic step runs inside the library's
kernels.  If the library is missing or a call is refused, this module raises;
there is no other code path.  The tensor-level calls at the end go through
``csrc/calls.cpp`` where their arguments are what they ordinarily are (it answers
None otherwise): the same marshalling, without the interpreter's time.  Where that module
cannot be built or loaded they are marshalled here, and a warning says so once.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
import warnings

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblinattn.so")
_lib = None
_calls, _bound = None, None         # the native tensor-level calls, and the library they were given

LINATTN_F32, LINATTN_BF16 = 0, 1
LINATTN_PHI_ELU1, LINATTN_PHI_RELU = 0, 1
PHI = {"elu1": LINATTN_PHI_ELU1, "relu": LINATTN_PHI_RELU}
MAX_CONV_K, MAX_CONV_K_PREFILL, MAX_DRAFT, MAX_TREE = 8, 63, 16, 64
SYMBOLS = ("linattn_workspace_bytes", "linattn_prefill", "linattn_prefill_noalloc", "linattn_noalloc_scratch_bytes", "linattn_prefill_grouped", "linattn_backward_workspace_bytes", "linattn_prefill_grouped_backward", "linattn_verify", "linattn_verify_grouped", "linattn_verify_tree", "linattn_decode",
           "linattn_decay_workspace_bytes", "linattn_decay_backward_workspace_bytes", "linattn_decay_prefill", "linattn_decay_backward", "linattn_decay_step",
           "linattn_window_prefill", "linattn_window_backward_workspace_bytes", "linattn_window_backward", "linattn_window_step_workspace_bytes", "linattn_window_step",
           "linattn_set_wait_limit", "linattn_status_string", "linattn_version")


class LinattnError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


class Desc(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("d", ctypes.c_int32),
                ("conv_k", ctypes.c_int32), ("chunk", ctypes.c_int32), ("io_dtype", ctypes.c_int32),
                ("phi", ctypes.c_int32), ("eps", ctypes.c_float),
                ("stride_b", ctypes.c_int64), ("stride_h", ctypes.c_int64), ("stride_t", ctypes.c_int64),
                ("d_v", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("stride_b_v", ctypes.c_int64), ("stride_h_v", ctypes.c_int64), ("stride_t_v", ctypes.c_int64)]


class Strides(ctypes.Structure):
    _fields_ = [("b", ctypes.c_int64), ("h", ctypes.c_int64), ("t", ctypes.c_int64)]


class DecayDesc(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("d", ctypes.c_int32), ("io_dtype", ctypes.c_int32),
                ("scale", ctypes.c_float), ("reserved", ctypes.c_int32),
                *[(n, Strides) for n in ("q", "k", "v", "out", "dout", "dq", "dk", "dv")]]


class WindowDesc(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("H_kv", ctypes.c_int32), ("d", ctypes.c_int32), ("io_dtype", ctypes.c_int32),
                ("window", ctypes.c_int32), ("sinks", ctypes.c_int32), ("scale", ctypes.c_float),
                *[(n, Strides) for n in ("q", "k", "v", "out", "dout", "dq", "dk", "dv")]]


def load():
    """Load the built library (build it first if it has never been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        from . import build as _build
        _build.build(calls=False)
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    dp = ctypes.POINTER(Desc)
    lib.linattn_workspace_bytes.restype = sz
    lib.linattn_workspace_bytes.argtypes = [dp, i32]
    lib.linattn_prefill.restype = ctypes.c_int
    lib.linattn_prefill.argtypes = [dp, i32] + [vp] * 11 + [vp, sz, vp]
    lib.linattn_prefill_noalloc.restype = ctypes.c_int
    lib.linattn_prefill_noalloc.argtypes = [dp, i32] + [vp] * 11 + [vp]
    lib.linattn_noalloc_scratch_bytes.restype = sz
    lib.linattn_noalloc_scratch_bytes.argtypes = []
    lib.linattn_prefill_grouped.restype = ctypes.c_int
    lib.linattn_prefill_grouped.argtypes = [dp, i32, ctypes.c_float] + [vp] * 11 + [vp, sz, vp]
    lib.linattn_backward_workspace_bytes.restype = sz
    lib.linattn_backward_workspace_bytes.argtypes = [dp, i32]
    lib.linattn_prefill_grouped_backward.restype = ctypes.c_int
    lib.linattn_prefill_grouped_backward.argtypes = [dp, i32, ctypes.c_float] + [vp] * 9 + [vp, sz, vp]
    lib.linattn_verify.restype = ctypes.c_int
    lib.linattn_verify.argtypes = [dp, i32] + [vp] * 9 + [vp]
    lib.linattn_verify_grouped.restype = ctypes.c_int
    lib.linattn_verify_grouped.argtypes = [dp, i32, ctypes.c_float] + [vp] * 12 + [vp]
    lib.linattn_verify_tree.restype = ctypes.c_int
    lib.linattn_verify_tree.argtypes = [dp, i32] + [vp] * 10 + [vp]
    lib.linattn_decode.restype = ctypes.c_int
    lib.linattn_decode.argtypes = [dp] + [vp] * 8 + [vp]
    dd = ctypes.POINTER(DecayDesc)
    for f in (lib.linattn_decay_workspace_bytes, lib.linattn_decay_backward_workspace_bytes):
        f.restype, f.argtypes = sz, [dd, i32]
    for f, args in ((lib.linattn_decay_prefill, [dd, i32] + [vp] * 8 + [vp, sz, vp]),
                    (lib.linattn_decay_backward, [dd, i32] + [vp] * 9 + [vp, sz, vp]),
                    (lib.linattn_decay_step, [dd, i32] + [vp] * 7 + [vp])):
        f.restype, f.argtypes = ctypes.c_int, args
    wd = ctypes.POINTER(WindowDesc)
    for f in (lib.linattn_window_backward_workspace_bytes, lib.linattn_window_step_workspace_bytes):
        f.restype, f.argtypes = sz, [wd, i32]
    for f, args in ((lib.linattn_window_prefill, [wd, i32] + [vp] * 10),
                    (lib.linattn_window_backward, [wd, i32] + [vp] * 10 + [vp, sz, vp]),
                    (lib.linattn_window_step, [wd, i32] + [vp] * 8 + [vp, sz, vp])):
        f.restype, f.argtypes = ctypes.c_int, args
    lib.linattn_status_string.restype = ctypes.c_char_p
    lib.linattn_status_string.argtypes = [ctypes.c_int]
    lib.linattn_version.restype = i32
    lib.linattn_set_wait_limit.restype = i32
    lib.linattn_set_wait_limit.argtypes = [i32]
    _lib = lib
    return lib


class _NoCalls:
    """In the place of the native calls where they cannot be had: every call takes the general path."""

    def __getattr__(self, name):
        return lambda *a: None


def _load_calls():
    try:
        from . import build as _build
        if not _build.calls_current():
            _build.build_calls()
        from . import _calls as mod
        return mod
    except (ImportError, OSError, RuntimeError) as e:     # no compiler, another torch, a folder that is read-only
        warnings.warn(f"the native tensor-level calls are not available ({e}); the calls go through ctypes", RuntimeWarning)
        return _NoCalls()


def _native():
    """The native tensor-level calls, bound to the library that is loaded."""
    global _calls, _bound
    lib = load()
    if _bound is not lib:
        if _calls is None:
            _calls = _load_calls()
        f = [lib.linattn_workspace_bytes, lib.linattn_prefill, lib.linattn_prefill_grouped, lib.linattn_backward_workspace_bytes,
             lib.linattn_prefill_grouped_backward, lib.linattn_verify, lib.linattn_verify_grouped, lib.linattn_verify_tree, lib.linattn_decode,
             lib.linattn_decay_workspace_bytes, lib.linattn_decay_prefill, lib.linattn_decay_backward_workspace_bytes, lib.linattn_decay_backward,
             lib.linattn_decay_step, lib.linattn_window_prefill, lib.linattn_window_backward_workspace_bytes, lib.linattn_window_backward,
             lib.linattn_window_step_workspace_bytes, lib.linattn_window_step]
        _calls.bind(tuple(ctypes.cast(x, ctypes.c_void_p).value for x in f), torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream)
        _bound = lib
    return _calls


def _result(r, where: str):
    if type(r) is int:
        raise LinattnError(r, where)
    return r


def status_string(status: int) -> str:
    return load().linattn_status_string(int(status)).decode()


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _stream(stream):
    if stream is None:
        return torch.cuda.current_stream().cuda_stream if torch.cuda.is_available() else None
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _check(status: int, where: str):
    if status != 0:
        raise LinattnError(status, where)


def make_desc(B, H, d, conv_k, chunk=64, io_dtype=torch.bfloat16, eps=0.0, strides=None, L=None, phi="elu1",
              d_v=None, strides_v=None) -> Desc:
    """Descriptor for dense [B,H,L,d] tensors unless ``strides`` (b, h, t) is given.  phi: "elu1" or "relu".
    d_v: width of the value rows when it differs from d (a multiple of d); v and out are then dense [B,H,L,d_v]
    unless ``strides_v`` is given."""
    code = {torch.float32: LINATTN_F32, torch.bfloat16: LINATTN_BF16}[io_dtype]
    Lx = 0 if L is None else int(L)
    if strides is None:
        strides = (H * Lx * d, Lx * d, d)
    if d_v is None or d_v == d:
        return Desc(B, H, d, conv_k, chunk, code, PHI[phi], float(eps), *[int(s) for s in strides], 0, 0, 0, 0, 0)
    if strides_v is None:
        strides_v = (H * Lx * d_v, Lx * d_v, d_v)
    return Desc(B, H, d, conv_k, chunk, code, PHI[phi], float(eps), *[int(s) for s in strides], int(d_v), 0,
                *[int(s) for s in strides_v])


def _ws_bytes(workspace, workspace_bytes) -> int:
    if workspace_bytes is None:
        workspace_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    return int(workspace_bytes)


def make_decay_desc(B, H, d, io_dtype=torch.bfloat16, scale=1.0, **strides) -> DecayDesc:
    """strides: (b, h, t) in elements for each of q, k, v, out (prefill) and dout, dq, dk, dv (gradient) that the call takes."""
    code = {torch.float32: LINATTN_F32, torch.bfloat16: LINATTN_BF16}[io_dtype]
    return DecayDesc(B, H, d, code, float(scale), 0, **{n: Strides(*[int(x) for x in s]) for n, s in strides.items()})


def _int32(name, x) -> int:
    """A field of 32 bits: ctypes would cut off what is above them."""
    x = int(x)
    if not -(1 << 31) <= x < 1 << 31:
        raise ValueError(f"{name} must fit 32 bits")
    return x


def make_window_desc(B, H, H_kv, d, window, sinks=0, io_dtype=torch.bfloat16, scale=1.0, **strides) -> WindowDesc:
    """strides: as for ``make_decay_desc``."""
    code = {torch.float32: LINATTN_F32, torch.bfloat16: LINATTN_BF16}[io_dtype]
    return WindowDesc(B, H, H_kv, d, code, _int32("window", window), _int32("sinks", sinks), float(scale), **{n: Strides(*[int(x) for x in s]) for n, s in strides.items()})


def linattn_set_wait_limit(spins: int) -> int:
    return int(load().linattn_set_wait_limit(int(spins)))


def linattn_workspace_bytes(desc: Desc, L: int) -> int:
    return int(load().linattn_workspace_bytes(ctypes.byref(desc), int(L)))


def linattn_prefill(desc: Desc, L, q, k, v, conv_w, S_in, z_in, hist_in, out, S_out, z_out, hist_out,
                    workspace=None, workspace_bytes=None, stream=None) -> None:
    if workspace_bytes is None:
        workspace_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    st = load().linattn_prefill(ctypes.byref(desc), int(L), _ptr(q), _ptr(k), _ptr(v), _ptr(conv_w),
                                _ptr(S_in), _ptr(z_in), _ptr(hist_in), _ptr(out), _ptr(S_out), _ptr(z_out),
                                _ptr(hist_out), _ptr(workspace), int(workspace_bytes), _stream(stream))
    _check(st, "linattn_prefill")


def linattn_prefill_noalloc(desc: Desc, L, q, k, v, conv_w, S_in, z_in, hist_in, out, S_out, z_out, hist_out, stream=None) -> None:
    st = load().linattn_prefill_noalloc(ctypes.byref(desc), int(L), _ptr(q), _ptr(k), _ptr(v), _ptr(conv_w),
                                        _ptr(S_in), _ptr(z_in), _ptr(hist_in), _ptr(out), _ptr(S_out), _ptr(z_out),
                                        _ptr(hist_out), _stream(stream))
    _check(st, "linattn_prefill_noalloc")


def linattn_noalloc_scratch_bytes() -> int:
    return int(load().linattn_noalloc_scratch_bytes())


def linattn_prefill_grouped(desc: Desc, L, alpha, q, k, v, conv_w, S_in, z_in, hist_in, out, S_out, z_out, hist_out,
                            workspace=None, workspace_bytes=None, stream=None) -> None:
    if workspace_bytes is None:
        workspace_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    st = load().linattn_prefill_grouped(ctypes.byref(desc), int(L), float(alpha), _ptr(q), _ptr(k), _ptr(v), _ptr(conv_w),
                                        _ptr(S_in), _ptr(z_in), _ptr(hist_in), _ptr(out), _ptr(S_out), _ptr(z_out),
                                        _ptr(hist_out), _ptr(workspace), int(workspace_bytes), _stream(stream))
    _check(st, "linattn_prefill_grouped")


def linattn_backward_workspace_bytes(desc: Desc, L) -> int:
    return int(load().linattn_backward_workspace_bytes(ctypes.byref(desc), int(L)))


def linattn_prefill_grouped_backward(desc: Desc, L, alpha, q, k, v, conv_w, dout, dq, dk, dv, dconv_w, workspace,
                                     workspace_bytes=None, stream=None) -> None:
    if workspace_bytes is None:
        workspace_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    st = load().linattn_prefill_grouped_backward(ctypes.byref(desc), int(L), float(alpha), _ptr(q), _ptr(k), _ptr(v),
                                                 _ptr(conv_w), _ptr(dout), _ptr(dq), _ptr(dk), _ptr(dv), _ptr(dconv_w),
                                                 _ptr(workspace), int(workspace_bytes), _stream(stream))
    _check(st, "linattn_prefill_grouped_backward")


def linattn_verify(desc: Desc, kk, q, k, v, conv_w, S, z, hist, n_commit, out, stream=None) -> None:
    st = load().linattn_verify(ctypes.byref(desc), int(kk), _ptr(q), _ptr(k), _ptr(v), _ptr(conv_w),
                               _ptr(S), _ptr(z), _ptr(hist), _ptr(n_commit), _ptr(out), _stream(stream))
    _check(st, "linattn_verify")


def linattn_verify_grouped(desc: Desc, kk, alpha, q, k, v, conv_w, S, z, hist, kwin, vwin, fill, n_commit, out, stream=None) -> None:
    st = load().linattn_verify_grouped(ctypes.byref(desc), int(kk), float(alpha), _ptr(q), _ptr(k), _ptr(v), _ptr(conv_w),
                                       _ptr(S), _ptr(z), _ptr(hist), _ptr(kwin), _ptr(vwin), _ptr(fill), _ptr(n_commit),
                                       _ptr(out), _stream(stream))
    _check(st, "linattn_verify_grouped")


def linattn_verify_tree(desc: Desc, n, q, k, v, parent, conv_w, S, z, hist, accept, out, stream=None) -> None:
    st = load().linattn_verify_tree(ctypes.byref(desc), int(n), _ptr(q), _ptr(k), _ptr(v), _ptr(parent), _ptr(conv_w),
                                    _ptr(S), _ptr(z), _ptr(hist), _ptr(accept), _ptr(out), _stream(stream))
    _check(st, "linattn_verify_tree")


def linattn_decode(desc: Desc, q, k, v, conv_w, S, z, hist, out, stream=None) -> None:
    st = load().linattn_decode(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _ptr(conv_w),
                               _ptr(S), _ptr(z), _ptr(hist), _ptr(out), _stream(stream))
    _check(st, "linattn_decode")


def linattn_decay_workspace_bytes(desc: DecayDesc, L) -> int:
    return int(load().linattn_decay_workspace_bytes(ctypes.byref(desc), int(L)))


def linattn_decay_backward_workspace_bytes(desc: DecayDesc, L) -> int:
    return int(load().linattn_decay_backward_workspace_bytes(ctypes.byref(desc), int(L)))


def linattn_decay_prefill(desc: DecayDesc, L, q, k, v, log_decay, lens, S_in, out, S_out, workspace=None, workspace_bytes=None, stream=None) -> None:
    st = load().linattn_decay_prefill(ctypes.byref(desc), int(L), _ptr(q), _ptr(k), _ptr(v), _ptr(log_decay), _ptr(lens), _ptr(S_in), _ptr(out),
                                      _ptr(S_out), _ptr(workspace), _ws_bytes(workspace, workspace_bytes), _stream(stream))
    _check(st, "linattn_decay_prefill")


def linattn_decay_backward(desc: DecayDesc, L, q, k, v, log_decay, lens, dout, dq, dk, dv, workspace=None, workspace_bytes=None, stream=None) -> None:
    st = load().linattn_decay_backward(ctypes.byref(desc), int(L), _ptr(q), _ptr(k), _ptr(v), _ptr(log_decay), _ptr(lens), _ptr(dout), _ptr(dq),
                                       _ptr(dk), _ptr(dv), _ptr(workspace), _ws_bytes(workspace, workspace_bytes), _stream(stream))
    _check(st, "linattn_decay_backward")


def linattn_decay_step(desc: DecayDesc, kk, q, k, v, log_decay, S, n_commit, out, stream=None) -> None:
    st = load().linattn_decay_step(ctypes.byref(desc), int(kk), _ptr(q), _ptr(k), _ptr(v), _ptr(log_decay), _ptr(S), _ptr(n_commit), _ptr(out),
                                   _stream(stream))
    _check(st, "linattn_decay_step")


def linattn_window_prefill(desc: WindowDesc, L, q, k, v, lens, out, lse=None, kcache=None, vcache=None, pos=None, stream=None) -> None:
    st = load().linattn_window_prefill(ctypes.byref(desc), int(L), _ptr(q), _ptr(k), _ptr(v), _ptr(lens), _ptr(out), _ptr(lse), _ptr(kcache),
                                       _ptr(vcache), _ptr(pos), _stream(stream))
    _check(st, "linattn_window_prefill")


def linattn_window_backward_workspace_bytes(desc: WindowDesc, L) -> int:
    return int(load().linattn_window_backward_workspace_bytes(ctypes.byref(desc), int(L)))


def linattn_window_backward(desc: WindowDesc, L, q, k, v, lens, out, lse, dout, dq, dk, dv, workspace, workspace_bytes=None, stream=None) -> None:
    st = load().linattn_window_backward(ctypes.byref(desc), int(L), _ptr(q), _ptr(k), _ptr(v), _ptr(lens), _ptr(out), _ptr(lse), _ptr(dout), _ptr(dq),
                                        _ptr(dk), _ptr(dv), _ptr(workspace), _ws_bytes(workspace, workspace_bytes), _stream(stream))
    _check(st, "linattn_window_backward")


def linattn_window_step_workspace_bytes(desc: WindowDesc, kk) -> int:
    return int(load().linattn_window_step_workspace_bytes(ctypes.byref(desc), int(kk)))


def linattn_window_step(desc: WindowDesc, kk, q, k, v, kcache, vcache, pos, n_commit, out, workspace=None, workspace_bytes=None, stream=None) -> None:
    st = load().linattn_window_step(ctypes.byref(desc), int(kk), _ptr(q), _ptr(k), _ptr(v), _ptr(kcache), _ptr(vcache), _ptr(pos), _ptr(n_commit),
                                    _ptr(out), _ptr(workspace), _ws_bytes(workspace, workspace_bytes), _stream(stream))
    _check(st, "linattn_window_step")


# ---- conveniences that only allocate with torch and forward to the calls above ---------------
# ``stream``: None for the current one, or a torch stream or a raw handle on which the call is enqueued.  What the call reads has to
# be ready for that stream, and what it returns is ready when that stream is done, as usual between streams; no memory that
# the call works on is handed out again before it is done, whatever becomes of the tensors.
@contextlib.contextmanager
def _memory_for(stream, device, *given):
    """Marks the tensors that the call is given as in use by ``stream``.  What is allocated in here belongs to it: memory that earlier
    work of another stream may still use is not taken, and a workspace that is let go is handed out again only behind the call.  Yields
    what marks a tensor that is returned: the caller's current stream uses it too."""
    if stream is None:
        yield lambda t: t
        return
    caller = torch.cuda.current_stream(device)
    if not isinstance(stream, torch.cuda.Stream):
        handle = stream if isinstance(stream, int) else stream.cuda_stream
        # (0, and 1 by its other name: the default stream, which ExternalStream does not take)
        stream = torch.cuda.ExternalStream(handle, device=device) if handle not in (0, 1) else torch.cuda.default_stream(device)

    def returned(t):
        if t is not None:
            t.record_stream(caller)
        return t

    with torch.cuda.stream(stream):
        for t in given:
            if t is not None:
                t.record_stream(stream)
        yield returned


def prefill(q, k, v, conv_w, state=None, chunk=64, eps=0.0, want_state=True, stream=None, phi="elu1", grouped_alpha=None):
    """q, k: [B,H,L,d], v: [B,H,L,d_v] CUDA tensors (fp32 or bf16; d_v = d or a multiple of d), dense or any view
    with unit stride along the last axis (e.g. ``x.transpose(1, 2)`` of a token-major [B,L,H,d] tensor); q and k
    share their strides, and so does v when d_v = d; ``out`` gets v's shape and strides.  Returns out, (S, z, hist).
    grouped_alpha: None, or the weight of the grouped branch of the three-branch form (``linattn_prefill_grouped``)."""
    if stream is None:
        r = _native().prefill(q, k, v, conv_w, state, chunk, eps, want_state, phi, grouped_alpha)
        if r is not None:
            return _result(r, "linattn_prefill" if grouped_alpha is None else "linattn_prefill_grouped")
    B, H, L, d = q.shape
    d_v = v.shape[3]
    Kc = conv_w.shape[2]
    dense = q.is_contiguous() and k.is_contiguous() and v.is_contiguous()
    if not dense and (q.stride(3) != 1 or v.stride(3) != 1 or k.stride() != q.stride() or (d_v == d and v.stride() != q.stride())):
        raise ValueError("q, k (and v, when it has their width) must share their strides and be contiguous along d")
    sq = None if dense else q.stride()[:3]
    sv = None if dense else v.stride()[:3]
    if d_v == d:
        desc = make_desc(B, H, d, Kc, chunk, q.dtype, eps, strides=sq, L=L, phi=phi)
    else:
        desc = make_desc(B, H, d, Kc, chunk, q.dtype, eps, strides=sq, L=L, phi=phi, d_v=d_v, strides_v=sv)
    S_in, z_in, h_in = state if state is not None else (None, None, None)
    S = z = h = None
    with _memory_for(stream, q.device, q, k, v, conv_w, S_in, z_in, h_in) as returned:
        out = returned(torch.empty_like(v) if dense else torch.empty_strided(v.shape, v.stride(), dtype=v.dtype, device=v.device))
        if want_state:
            S = returned(torch.empty((B, H, d, d_v), dtype=torch.float32, device=q.device))
            z = returned(torch.empty((B, H, d), dtype=torch.float32, device=q.device))
            h = returned(torch.empty((B, H, max(Kc - 1, 0), d_v), dtype=q.dtype, device=q.device))
        nbytes = linattn_workspace_bytes(desc, L)
        ws = torch.empty(nbytes, dtype=torch.uint8, device=q.device) if nbytes else None
        if grouped_alpha is None:
            linattn_prefill(desc, L, q, k, v, conv_w, S_in, z_in, h_in, out, S, z, h, ws, nbytes, stream)
        else:
            linattn_prefill_grouped(desc, L, grouped_alpha, q, k, v, conv_w, S_in, z_in, h_in, out, S, z, h, ws, nbytes, stream)
    return out, (S, z, h)


def prefill_grouped(q, k, v, conv_w, alpha=1.0, state=None, eps=0.0, want_state=True, stream=None, phi="elu1", group=64):
    """The three-branch form (grouped linear attention, weight alpha + local softmax attention + masked conv)
    with groups of 64 or 256 tokens; arguments as for ``prefill``."""
    return prefill(q, k, v, conv_w, state, group, eps, want_state, stream, phi, grouped_alpha=alpha)


def prefill_grouped_backward(q, k, v, conv_w, dout, alpha=1.0, eps=0.0, stream=None, phi="elu1", group=256,
                             want_dw=True):
    """Gradient of ``prefill_grouped`` for a sequence that starts from nothing: q, k, v, dout bf16 [B,H,L,d] CUDA
    tensors, dense or views that share their strides and are contiguous along d.  Returns dq, dk, dv (same layout)
    and the gradient of the conv weights (fp32 [H,d,Kc], summed over the batch; None if not wanted)."""
    if stream is None:
        r = _native().prefill_grouped_backward(q, k, v, conv_w, dout, alpha, eps, phi, group, want_dw)
        if r is not None:
            return _result(r, "linattn_prefill_grouped_backward")
    B, H, L, d = q.shape
    Kc = conv_w.shape[2]
    dense = all(t.is_contiguous() for t in (q, k, v, dout))
    if not dense and (q.stride(3) != 1 or any(t.stride() != q.stride() for t in (k, v, dout))):
        raise ValueError("q, k, v and dout must share their strides and be contiguous along d")
    desc = make_desc(B, H, d, Kc, group, q.dtype, eps, strides=None if dense else q.stride()[:3], L=L, phi=phi)
    new = (lambda: torch.empty_like(q)) if dense else (lambda: torch.empty_strided(q.shape, q.stride(), dtype=q.dtype, device=q.device))
    with _memory_for(stream, q.device, q, k, v, conv_w, dout) as returned:
        dq, dk, dv = returned(new()), returned(new()), returned(new())
        dw = returned(torch.empty((H, d, Kc), dtype=torch.float32, device=q.device)) if want_dw else None
        nbytes = linattn_backward_workspace_bytes(desc, L)
        ws = torch.empty(max(nbytes, 16), dtype=torch.uint8, device=q.device)
        linattn_prefill_grouped_backward(desc, L, alpha, q, k, v, conv_w, dout, dq, dk, dv, dw, ws, nbytes, stream)
    return dq, dk, dv, dw


def verify(q, k, v, conv_w, state, n_commit=None, eps=0.0, stream=None, phi="elu1"):
    """q, k: dense [B,H,kk,d]; v: dense [B,H,kk,d_v].  ``state`` = (S, z, hist) is updated in place.  Returns out."""
    if stream is None:
        r = _native().verify(q, k, v, conv_w, state, n_commit, eps, phi)
        if r is not None:
            return _result(r, "linattn_verify")
    B, H, kk, d = q.shape
    desc = make_desc(B, H, d, conv_w.shape[2], 64, q.dtype, eps, L=kk, phi=phi, d_v=v.shape[-1])
    S, z, h = state
    with _memory_for(stream, q.device, q, k, v, conv_w, S, z, h, n_commit) as returned:
        out = returned(torch.empty_like(v))
        linattn_verify(desc, kk, q, k, v, conv_w, S, z, h, n_commit, out, stream)
    return out


def grouped_state(B, H, d, conv_k, dtype=torch.bfloat16, device="cuda", prefill_state=None):
    """State of the three-branch form for ``verify_grouped``: (S, z, hist, kwin, vwin, fill).  Zeros (start of a
    sequence), or the (S, z, hist) that ``prefill_grouped`` returned for a multiple of 64 tokens, with an empty
    open group."""
    if prefill_state is None:
        S = torch.zeros((B, H, d, d), dtype=torch.float32, device=device)
        z = torch.zeros((B, H, d), dtype=torch.float32, device=device)
        h = torch.zeros((B, H, max(conv_k - 1, 0), d), dtype=dtype, device=device)
    else:
        S, z, h = prefill_state
    kwin = torch.zeros((B, H, 64, d), dtype=dtype, device=device)
    vwin = torch.zeros((B, H, 64, d), dtype=dtype, device=device)
    fill = torch.zeros((B, H), dtype=torch.int32, device=device)
    return S, z, h, kwin, vwin, fill


def verify_grouped(q, k, v, conv_w, state, alpha=1.0, n_commit=None, eps=0.0, stream=None, phi="elu1"):
    """q, k, v: dense [B,H,kk,d].  ``state`` = (S, z, hist, kwin, vwin, fill) is updated in place.  Returns out."""
    if stream is None:
        r = _native().verify_grouped(q, k, v, conv_w, state, alpha, n_commit, eps, phi)
        if r is not None:
            return _result(r, "linattn_verify_grouped")
    B, H, kk, d = q.shape
    desc = make_desc(B, H, d, conv_w.shape[2], 64, q.dtype, eps, L=kk, phi=phi)
    S, z, h, kwin, vwin, fill = state
    with _memory_for(stream, q.device, q, k, v, conv_w, *state, n_commit) as returned:
        out = returned(torch.empty_like(q))
        linattn_verify_grouped(desc, kk, alpha, q, k, v, conv_w, S, z, h, kwin, vwin, fill, n_commit, out, stream)
    return out


def verify_tree(q, k, v, parent, conv_w, state, accept=None, eps=0.0, stream=None, phi="elu1"):
    """q, k, v: dense [B,H,n,d], bf16 or fp32; parent: int32 [n] on the GPU.  ``state`` is updated in place along the
    root path of candidate ``accept[b]`` (int32 [B] on the GPU; None accepts nothing).  Returns out."""
    if stream is None:
        r = _native().verify_tree(q, k, v, parent, conv_w, state, accept, eps, phi)
        if r is not None:
            return _result(r, "linattn_verify_tree")
    B, H, n, d = q.shape
    desc = make_desc(B, H, d, conv_w.shape[2], 64, q.dtype, eps, L=n, phi=phi)
    S, z, h = state
    with _memory_for(stream, q.device, q, k, v, parent, conv_w, S, z, h, accept) as returned:
        out = returned(torch.empty_like(q))
        linattn_verify_tree(desc, n, q, k, v, parent, conv_w, S, z, h, accept, out, stream)
    return out


def decode(q, k, v, conv_w, state, eps=0.0, stream=None, phi="elu1"):
    """q, k: dense [B,H,d] (or [B,H,1,d]); v: dense [B,H,d_v].  ``state`` is updated in place.  Returns out."""
    if stream is None:
        r = _native().decode(q, k, v, conv_w, state, eps, phi)
        if r is not None:
            return _result(r, "linattn_decode")
    B, H, d = q.shape[0], q.shape[1], q.shape[-1]
    desc = make_desc(B, H, d, conv_w.shape[2], 64, q.dtype, eps, L=1, phi=phi, d_v=v.shape[-1])
    S, z, h = state
    with _memory_for(stream, q.device, q, k, v, conv_w, S, z, h) as returned:
        out = returned(torch.empty_like(v))
        linattn_decode(desc, q, k, v, conv_w, S, z, h, out, stream)
    return out


# ---- attention whose memory per sequence is bounded ------------------------------------------
def _rows(where, q, **others):
    """Checks rows [B,heads,L,d] against q's type, device and last axis; the strides of those that lie in rows."""
    if q.dim() != 4 or q.dtype not in (torch.float32, torch.bfloat16):
        raise ValueError(f"{where}: q must be a [B,H,L,d] tensor in fp32 or bf16")
    for n, x in {"q": q, **others}.items():
        if x.dim() != 4 or x.dtype != q.dtype or x.device != q.device or x.shape[3] != q.shape[3]:
            raise ValueError(f"{where}: {n} must be a [B,heads,L,d] tensor of q's dtype and device")
        if x.shape[3] > 1 and x.stride(3) != 1:
            raise ValueError(f"{where}: {n} must be contiguous along d")


def _aux(where, name, x, dtype, shape, device):
    if x is not None and (x.dtype != dtype or tuple(x.shape) != tuple(shape) or x.device != device or not x.is_contiguous()):
        raise ValueError(f"{where}: {name} must be a dense {dtype} tensor of shape {tuple(shape)} on {device}")


def _st(x):
    """(b, h, t) strides; of an axis that holds one row or none they mean nothing."""
    return tuple(0 if n < 2 else s for n, s in zip(x.shape[:3], x.stride()))


def _like(x):
    """A tensor for rows laid out as x's are, dense where x is not (a slice, an expanded tensor)."""
    return torch.empty_like(x)


def _scratch(nbytes, device):
    return torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None


def _on(device):
    """The library works on the current device: make it the tensors'."""
    if device.type != "cuda":
        raise ValueError("the tensors must be on the GPU")
    return torch.cuda.device(device)


def decay_prefill(q, k, v, log_decay, scale=None, state=None, lens=None, want_state=True, stream=None):
    """Linear attention with a decay for each head: out_t = scale * q_t^T S_t, S_t = exp(log_decay) S_{t-1} + k_t v_t^T.

    q, k, v: [B,H,L,d] CUDA tensors, fp32 or bf16, contiguous along d and otherwise of any strides that are multiples of 8
    (slices of a packed projection, token-major views, broadcast heads), at multiples of 16 bytes.  log_decay: fp32 [H],
    each <= 0.  scale: None for d ** -0.5.  state: None or the fp32 [B,H,d,d] to go on from.  lens: None, or int32 [B],
    the tokens of each row; rows behind them are ignored and their outputs are zeros.  Returns out (q's layout where q is
    dense in some order of its axes) and the new state (None if not wanted)."""
    if stream is None:
        r = _native().decay_prefill(q, k, v, log_decay, scale, state, lens, want_state)
        if r is not None:
            return _result(r, "linattn_decay_prefill")
    _rows("decay_prefill", q, k=k, v=v)
    B, H, L, d = q.shape
    if k.shape != q.shape or v.shape != q.shape:
        raise ValueError("decay_prefill: q, k and v must have one shape")
    _aux("decay_prefill", "log_decay", log_decay, torch.float32, (H,), q.device)
    _aux("decay_prefill", "state", state, torch.float32, (B, H, d, d), q.device)
    _aux("decay_prefill", "lens", lens, torch.int32, (B,), q.device)
    with _on(q.device), _memory_for(stream, q.device, q, k, v, log_decay, state, lens) as returned:
        out = returned(_like(q))
        S = returned(torch.empty((B, H, d, d), dtype=torch.float32, device=q.device)) if want_state else None
        desc = make_decay_desc(B, H, d, q.dtype, d ** -0.5 if scale is None else scale, q=_st(q), k=_st(k), v=_st(v), out=_st(out))
        ws = _scratch(linattn_decay_workspace_bytes(desc, L), q.device)
        linattn_decay_prefill(desc, L, q, k, v, log_decay, lens, state, out, S, ws, None, stream)
    return out, S


def decay_backward(q, k, v, log_decay, dout, scale=None, lens=None, stream=None):
    """Gradient of ``decay_prefill`` (from no state) with respect to q, k and v; dout: [B,H,L,d], strides as
    there.  Returns dq, dk, dv."""
    if stream is None:
        r = _native().decay_backward(q, k, v, log_decay, dout, scale, lens)
        if r is not None:
            return _result(r, "linattn_decay_backward")
    _rows("decay_backward", q, k=k, v=v, dout=dout)
    B, H, L, d = q.shape
    if k.shape != q.shape or v.shape != q.shape or dout.shape != q.shape:
        raise ValueError("decay_backward: q, k, v and dout must have one shape")
    _aux("decay_backward", "log_decay", log_decay, torch.float32, (H,), q.device)
    _aux("decay_backward", "lens", lens, torch.int32, (B,), q.device)
    with _on(q.device), _memory_for(stream, q.device, q, k, v, log_decay, dout, lens) as returned:
        dq, dk, dv = (returned(_like(x)) for x in (q, k, v))
        desc = make_decay_desc(B, H, d, q.dtype, d ** -0.5 if scale is None else scale, q=_st(q), k=_st(k), v=_st(v),
                               dout=_st(dout), dq=_st(dq), dk=_st(dk), dv=_st(dv))
        ws = _scratch(linattn_decay_backward_workspace_bytes(desc, L), q.device)
        linattn_decay_backward(desc, L, q, k, v, log_decay, lens, dout, dq, dk, dv, ws, None, stream)
    return dq, dk, dv


def decay_step(q, k, v, log_decay, state, scale=None, n_commit=None, stream=None):
    """kk tokens (1..16) from a running state: q, k, v dense [B,H,kk,d]; ``state`` (fp32 [B,H,d,d]) advances in place over
    the first n_commit[b] (int32 [B]; None: all) of them.  Returns out."""
    if stream is None:
        r = _native().decay_step(q, k, v, log_decay, state, scale, n_commit)
        if r is not None:
            return _result(r, "linattn_decay_step")
    _rows("decay_step", q, k=k, v=v)
    B, H, kk, d = q.shape
    if k.shape != q.shape or v.shape != q.shape or not (q.is_contiguous() and k.is_contiguous() and v.is_contiguous()):
        raise ValueError("decay_step: q, k and v must be dense and of one shape")
    _aux("decay_step", "log_decay", log_decay, torch.float32, (H,), q.device)
    _aux("decay_step", "state", state, torch.float32, (B, H, d, d), q.device)
    _aux("decay_step", "n_commit", n_commit, torch.int32, (B,), q.device)
    with _on(q.device), _memory_for(stream, q.device, q, k, v, log_decay, state, n_commit) as returned:
        out = returned(torch.empty_like(q))
        desc = make_decay_desc(B, H, d, q.dtype, d ** -0.5 if scale is None else scale)
        linattn_decay_step(desc, kk, q, k, v, log_decay, state, n_commit, out, stream)
    return out


def _kv(where, q, k, v, window, sinks):
    """Key/value rows [B,H_kv,L,d] for queries [B,H,L,d]; the numbers."""
    _int32(f"{where}: window", window), _int32(f"{where}: sinks", sinks)
    if k.shape != v.shape or k.shape[0] != q.shape[0] or k.shape[2] != q.shape[2] or k.shape[1] < 1 or q.shape[1] % k.shape[1]:
        raise ValueError(f"{where}: k and v must have one shape, q's with a number of heads that divides q's")


def _new_cache(B, H_kv, d, window, sinks, dtype, device):
    """Memory alone: no kernel of torch's, which would run on the current stream whatever stream the call is for."""
    rows = [torch.empty((B, H_kv, sinks + window, d), dtype=dtype, device=device) for _ in range(2)]
    return (*rows, torch.empty((B, H_kv), dtype=torch.int32, device=device))


def window_cache(B, H_kv, d, window, sinks=0, dtype=torch.bfloat16, device="cuda"):
    """Cache of ``window_step`` for sequences that have not begun: (kcache, vcache, pos).  (pos is cleared on the current stream.)"""
    cache = _new_cache(B, H_kv, d, window, sinks, dtype, device)
    cache[2].zero_()
    return cache


def window_prefill(q, k, v, window, sinks=0, scale=None, lens=None, want_lse=False, want_cache=False, stream=None):
    """Softmax attention in which token t sees token s where s <= t and (s > t - window or s < sinks).

    q: [B,H,L,d], k, v: [B,H_kv,L,d] (H_kv divides H: query head h uses key/value head h // (H // H_kv)), fp32 or bf16,
    strides as for ``decay_prefill``.  scale: None for d ** -0.5.  lens: None, or int32 [B], the tokens of each row; rows behind them are ignored and their outputs are zeros.  sinks: at most 64.  Returns out, the logarithms of the
    softmax sums (fp32 [B,H,L], what ``window_backward`` takes; None if not wanted) and the cache for ``window_step``
    (kcache, vcache, pos; None if not wanted)."""
    if stream is None and not want_cache:
        r = _native().window_prefill(q, k, v, window, sinks, scale, lens, want_lse)
        if r is not None:
            return _result(r, "linattn_window_prefill")
    _rows("window_prefill", q, k=k, v=v)
    _kv("window_prefill", q, k, v, window, sinks)
    B, H, L, d = q.shape
    _aux("window_prefill", "lens", lens, torch.int32, (B,), q.device)
    with _on(q.device), _memory_for(stream, q.device, q, k, v, lens) as returned:
        out = returned(_like(q))
        lse = returned(torch.empty((B, H, L), dtype=torch.float32, device=q.device)) if want_lse else None
        cache = tuple(returned(x) for x in _new_cache(B, k.shape[1], d, window, sinks, q.dtype, q.device)) if want_cache else None   # (the call writes every pos)
        desc = make_window_desc(B, H, k.shape[1], d, window, sinks, q.dtype, d ** -0.5 if scale is None else scale, q=_st(q), k=_st(k), v=_st(v), out=_st(out))
        linattn_window_prefill(desc, L, q, k, v, lens, out, lse, *(cache or (None, None, None)), stream)
    return out, lse, cache


def window_backward(q, k, v, out, lse, dout, window, sinks=0, scale=None, lens=None, stream=None):
    """Gradient of ``window_prefill`` with respect to q, k and v: bf16 rows, out and lse as it returned them, dout [B,H,L,d].
    Returns dq, dk, dv (dk, dv summed over the query heads that share a key/value head)."""
    if stream is None:
        r = _native().window_backward(q, k, v, out, lse, dout, window, sinks, scale, lens)
        if r is not None:
            return _result(r, "linattn_window_backward")
    _rows("window_backward", q, k=k, v=v, out=out, dout=dout)
    _kv("window_backward", q, k, v, window, sinks)
    B, H, L, d = q.shape
    if out.shape != q.shape or dout.shape != q.shape:
        raise ValueError("window_backward: out and dout must have q's shape")
    if lse is None:
        raise ValueError("window_backward: lse is what window_prefill returns with want_lse=True")
    _aux("window_backward", "lse", lse, torch.float32, (B, H, L), q.device)
    _aux("window_backward", "lens", lens, torch.int32, (B,), q.device)
    with _on(q.device), _memory_for(stream, q.device, q, k, v, out, lse, dout, lens) as returned:
        dq, dk, dv = (returned(_like(x)) for x in (q, k, v))
        desc = make_window_desc(B, H, k.shape[1], d, window, sinks, q.dtype, d ** -0.5 if scale is None else scale, q=_st(q), k=_st(k), v=_st(v),
                                out=_st(out), dout=_st(dout), dq=_st(dq), dk=_st(dk), dv=_st(dv))
        ws = _scratch(linattn_window_backward_workspace_bytes(desc, L), q.device)
        linattn_window_backward(desc, L, q, k, v, lens, out, lse, dout, dq, dk, dv, ws, None, stream)
    return dq, dk, dv


def window_step(q, k, v, cache, window, sinks=0, scale=None, n_commit=None, stream=None):
    """kk tokens (1..16) behind a cache: q dense [B,H,kk,d], k, v dense [B,H_kv,kk,d]; ``cache`` (kcache, vcache, pos) of
    ``window_prefill`` or ``window_cache`` with the same window and sinks advances in place over the first n_commit[b]
    (int32 [B]; None: all) of them.  Returns out."""
    if stream is None:
        r = _native().window_step(q, k, v, cache, window, sinks, scale, n_commit)
        if r is not None:
            return _result(r, "linattn_window_step")
    _rows("window_step", q, k=k, v=v)
    _kv("window_step", q, k, v, window, sinks)
    B, H, kk, d = q.shape
    kcache, vcache, pos = cache
    for n, x in (("q", q), ("k", k), ("v", v)):
        if not x.is_contiguous():
            raise ValueError(f"window_step: {n} must be dense")
    for n, x in (("kcache", kcache), ("vcache", vcache)):
        _aux("window_step", n, x, q.dtype, (B, k.shape[1], sinks + window, d), q.device)
    _aux("window_step", "pos", pos, torch.int32, (B, k.shape[1]), q.device)
    _aux("window_step", "n_commit", n_commit, torch.int32, (B,), q.device)
    with _on(q.device), _memory_for(stream, q.device, q, k, v, kcache, vcache, pos, n_commit) as returned:
        out = returned(torch.empty_like(q))
        desc = make_window_desc(B, H, k.shape[1], d, window, sinks, q.dtype, d ** -0.5 if scale is None else scale)
        ws = _scratch(linattn_window_step_workspace_bytes(desc, kk), q.device)
        linattn_window_step(desc, kk, q, k, v, kcache, vcache, pos, n_commit, out, ws, None, stream)
    return out
