"""Python binding of the C ABI in include/exemcl.h (argument marshalling only).

Every function takes torch tensors that already live on the current HIP
device, passes their device pointers and the current torch stream (or the one
given as ``stream``) to libexemcl.so, and returns without synchronising.  On
a given stream the caller orders the call behind what writes its inputs, and
what reads its results behind the call; their memory may be freed at any time.
No computation happens here; when the library is missing every call raises.
"""
from __future__ import annotations

import ctypes
import os
from types import SimpleNamespace
from typing import Any, NamedTuple

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libexemcl.so")

EXEMCL_FP32, EXEMCL_FP16, EXEMCL_BF16 = 0, 1, 2
EXEMCL_MX_NONE, EXEMCL_MXFP4, EXEMCL_MXFP8 = 0, 4, 8
EXEMCL_SILU, EXEMCL_GELU, EXEMCL_GELU_TANH, EXEMCL_RELU = 0, 1, 2, 3
EXEMCL_OK, EXEMCL_EINVAL, EXEMCL_ENOMEM, EXEMCL_EDEVICE, EXEMCL_ESCRATCH = 0, 1, 2, 3, 4
EXEMCL_SCRATCH_BYTES = 64 << 20   # fixed scratch buffer of exemplar_eval_noalloc
PATH_NONE, PATH_VALU, PATH_MFMA = 0, 1, 2
PATH_NAMES = {PATH_NONE: "none", PATH_VALU: "valu", PATH_MFMA: "mfma"}

EXPORTED = ("exemplar_eval", "exemplar_eval_noalloc", "exemplar_eval_streamed", "exemplar_gain", "exemplar_greedy", "exemplar_sqnorm",
            "exemplar_plan", "exemplar_mx_layout", "exemplar_mx_quantize", "exemplar_mx_dequantize", "exemplar_rmsnorm",
            "exemplar_rmsnorm_backward", "exemplar_mx_product", "exemplar_mx_eval",
            "exemplar_glu", "exemplar_glu_backward", "exemplar_w4_layout", "exemplar_w4_quantize", "exemplar_w4_dequantize",
            "exemplar_w4_product", "exemplar_w4_glu",
            "exemplar_prof_enable", "exemplar_prof_read", "exemplar_strerror", "exemplar_version")


class ExemclError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {strerror(status)} (status {status})")


_LIB = None


def load(path: str | None = None) -> ctypes.CDLL:
    """Open libexemcl.so (once; EXEMCL_LIB overrides the path).  Raises if it
    has not been built."""
    global _LIB
    if _LIB is not None and path is None:
        return _LIB
    p = path or os.environ.get("EXEMCL_LIB") or LIB_PATH
    if not os.path.exists(p):
        raise ImportError(f"{p} is missing: build it with `python -m paper_2101_08763_amd.build` "
                          "(or __graft_entry__.build()); there is no fallback implementation")
    lib = ctypes.CDLL(p)
    vp, i64, ip = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int
    lib.exemplar_eval.argtypes = [vp, i64, i64, vp, i64, i64, ip, vp, vp]
    lib.exemplar_eval.restype = ip
    lib.exemplar_eval_noalloc.argtypes = [vp, i64, i64, vp, i64, i64, ip, vp, vp]
    lib.exemplar_eval_noalloc.restype = ip
    lib.exemplar_eval_streamed.argtypes = [vp, i64, i64, vp, i64, i64, ip, i64, vp, vp]
    lib.exemplar_eval_streamed.restype = ip
    lib.exemplar_gain.argtypes = [vp, i64, i64, vp, i64, vp, i64, vp, vp]
    lib.exemplar_gain.restype = ip
    lib.exemplar_greedy.argtypes = [vp, i64, i64, i64, vp, vp, vp]
    lib.exemplar_greedy.restype = ip
    lib.exemplar_sqnorm.argtypes = [vp, i64, i64, ip, vp, vp]
    lib.exemplar_sqnorm.restype = ip
    lib.exemplar_plan.argtypes = [i64, i64, i64, i64, ip, ctypes.POINTER(ctypes.c_int),
                                  ctypes.POINTER(ctypes.c_int64)]
    lib.exemplar_plan.restype = ip
    fl = ctypes.c_float
    lib.exemplar_mx_layout.argtypes = [i64, ip, ctypes.POINTER(ctypes.c_int64), ctypes.POINTER(ctypes.c_int64)]
    lib.exemplar_mx_layout.restype = ip
    lib.exemplar_mx_quantize.argtypes = [vp, i64, i64, ip, ip, vp, vp, vp]
    lib.exemplar_mx_quantize.restype = ip
    lib.exemplar_mx_dequantize.argtypes = [vp, vp, i64, i64, ip, ip, vp, vp]
    lib.exemplar_mx_dequantize.restype = ip
    lib.exemplar_rmsnorm.argtypes = [vp, vp, vp, i64, i64, ip, fl, ip, vp, vp, vp, vp, vp]
    lib.exemplar_rmsnorm.restype = ip
    lib.exemplar_rmsnorm_backward.argtypes = [vp, vp, vp, vp, vp, i64, i64, ip, vp, vp, vp]
    lib.exemplar_rmsnorm_backward.restype = ip
    lib.exemplar_mx_product.argtypes = [vp, vp, i64, ip, vp, vp, i64, i64, vp, ip, vp, vp]
    lib.exemplar_mx_product.restype = ip
    lib.exemplar_mx_eval.argtypes = [vp, vp, i64, i64, vp, i64, i64, vp, vp]
    lib.exemplar_mx_eval.restype = ip
    lib.exemplar_glu.argtypes = [vp, i64, i64, vp, vp, i64, vp, vp, ip, ip, vp, vp, vp, vp]
    lib.exemplar_glu.restype = ip
    lib.exemplar_glu_backward.argtypes = [vp, vp, vp, vp, vp, vp, i64, i64, i64, ip, ip, vp, vp, vp, vp, vp, vp]
    lib.exemplar_glu_backward.restype = ip
    lib.exemplar_w4_layout.argtypes = [i64, i64, ip, ctypes.POINTER(ctypes.c_int64), ctypes.POINTER(ctypes.c_int64)]
    lib.exemplar_w4_layout.restype = ip
    lib.exemplar_w4_quantize.argtypes = [vp, i64, i64, ip, ip, vp, vp, vp]
    lib.exemplar_w4_quantize.restype = ip
    lib.exemplar_w4_dequantize.argtypes = [vp, vp, i64, i64, ip, ip, vp, vp]
    lib.exemplar_w4_dequantize.restype = ip
    lib.exemplar_w4_product.argtypes = [vp, i64, i64, ip, vp, vp, i64, ip, vp, vp, vp]
    lib.exemplar_w4_product.restype = ip
    lib.exemplar_w4_glu.argtypes = [vp, i64, i64, ip, vp, vp, vp, vp, i64, ip, vp, vp, ip, vp, vp]
    lib.exemplar_w4_glu.restype = ip
    lib.exemplar_strerror.argtypes = [ip]
    lib.exemplar_strerror.restype = ctypes.c_char_p
    lib.exemplar_prof_enable.argtypes = [ip]
    lib.exemplar_prof_enable.restype = ip
    lib.exemplar_prof_read.argtypes = [ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int64)]
    lib.exemplar_prof_read.restype = ip
    lib.exemplar_version.argtypes = []
    lib.exemplar_version.restype = ip
    if path is None:
        _LIB = lib
    return lib


def strerror(status: int) -> str:
    try:
        return load().exemplar_strerror(int(status)).decode()
    except ImportError:
        return {0: "success", 1: "invalid argument", 2: "temporary device memory unavailable",
                3: "HIP runtime or kernel launch failure",
                4: "workspace needed exceeds the fixed no-allocation scratch buffer"}.get(int(status), "unknown status")


def precision_of(dtype) -> int:
    import torch
    table = {torch.float32: EXEMCL_FP32, torch.float16: EXEMCL_FP16, torch.bfloat16: EXEMCL_BF16}
    if dtype not in table:
        raise TypeError(f"V must be float32, float16 or bfloat16, not {dtype}")
    return table[dtype]


def _stream(stream):
    """The HIP stream handle of `stream`, or of the current stream of the
    current device (PyTorch's raw-stream query when it has one: it skips
    building a Stream object, a few microseconds per call)."""
    import torch
    if stream is not None:
        return ctypes.c_void_p(stream.cuda_stream)
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if raw is not None:
        return ctypes.c_void_p(raw(torch.cuda.current_device()))
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _torch_stream(stream):
    import torch
    return stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(stream.cuda_stream)


def _empty_on(stream):
    """torch.empty and empty_like for what a call on ``stream`` writes.  PyTorch's
    allocator hands out memory whose last use is still queued on the stream it
    belongs to, so a result of another stream comes from that one's memory, and is
    not reused there before the current stream, which gets it, is done with it."""
    import torch
    st = _torch_stream(stream)

    def empty(shape, dtype, device):
        if device.type != "cuda":
            return torch.empty(shape, dtype=dtype, device=device)
        with torch.cuda.stream(st):
            t = torch.empty(shape, dtype=dtype, device=device)
        t.record_stream(torch.cuda.current_stream(device))
        return t

    return empty, lambda t: empty(t.shape, t.dtype, t.device)


def _empty(stream):
    """torch.empty for results of a call on ``stream`` (None: the current one)."""
    import torch
    return torch.empty if stream is None else _empty_on(stream)[0]


def _used(stream, *tensors):
    """Keeps the memory of a call's tensors, when they are freed early, until
    the ``stream`` it was given is done with them."""
    if stream is None:
        return
    st = _torch_stream(stream)
    for t in tensors:
        if t is not None and t.is_cuda:
            t.record_stream(st)


def _check_device(*tensors):
    dev = None
    for t in tensors:
        if t is None:
            continue
        if not t.is_cuda:
            raise ValueError("all tensors must be on the GPU")
        if not t.is_contiguous():
            raise ValueError("tensors must be contiguous")
        if dev is None:
            dev = t.device
        elif t.device != dev:
            raise ValueError("tensors are on different devices")
    return dev


def _device_scope(dev):
    """Make `dev` current for the call; a no-op (no device switch) when it
    already is, which saves the switch and restore on every call."""
    import contextlib
    import torch
    if dev is None or dev.index == torch.cuda.current_device():
        return contextlib.nullcontext()
    return torch.cuda.device(dev)


def _ptr(t):
    return ctypes.c_void_p(t.data_ptr()) if t is not None and t.numel() > 0 else ctypes.c_void_p(0)


def exemplar_eval(V, sets, out=None, stream=None):
    """out[j] = f(S_j) for the l x k int32 index matrix ``sets`` (see exemplar_eval in exemcl.h)."""
    import torch
    if V.dim() != 2 or sets.dim() != 2:
        raise ValueError("V must be n x d and sets l x k")
    if sets.dtype != torch.int32:
        raise TypeError("sets must be int32")
    prec = precision_of(V.dtype)
    n, d = V.shape
    l, k = sets.shape
    if out is None:
        out = _empty(stream)(l, dtype=torch.float32, device=V.device)
    elif out.dtype != torch.float32 or out.numel() != l:
        raise ValueError("out must be float32 with l elements")
    with _device_scope(_check_device(V, sets, out)):
        rc = load().exemplar_eval(_ptr(V), n, d, _ptr(sets), l, k, prec, _ptr(out), _stream(stream))
    _used(stream, V, sets, out)
    if rc != EXEMCL_OK:
        raise ExemclError(rc, "exemplar_eval")
    return out


def exemplar_eval_noalloc(V, sets, out, stream=None):
    """exemplar_eval with every temporary in the library's fixed scratch
    buffer (see exemplar_eval_noalloc in exemcl.h); ``out`` (float32, l
    elements, on V's device) is required, so nothing is allocated here
    either."""
    import torch
    if V.dim() != 2 or sets.dim() != 2:
        raise ValueError("V must be n x d and sets l x k")
    if sets.dtype != torch.int32:
        raise TypeError("sets must be int32")
    prec = precision_of(V.dtype)
    n, d = V.shape
    l, k = sets.shape
    if out is None or out.dtype != torch.float32 or out.numel() != l:
        raise ValueError("out must be float32 with l elements")
    with _device_scope(_check_device(V, sets, out)):
        rc = load().exemplar_eval_noalloc(_ptr(V), n, d, _ptr(sets), l, k, prec, _ptr(out), _stream(stream))
    _used(stream, V, sets, out)
    if rc != EXEMCL_OK:
        raise ExemclError(rc, "exemplar_eval_noalloc")
    return out


def exemplar_eval_streamed(V, sets, rows_per_block=0, out=None, device=None, stream=None):
    """out[j] = f(S_j) for V and ``sets`` in host memory (CPU tensors), with V
    streamed through the GPU in row blocks (see exemplar_eval_streamed in
    exemcl.h).  Synchronous; returns a CPU float32 tensor.  ``device`` is the
    GPU to use (default: the current one)."""
    import torch
    if V.dim() != 2 or sets.dim() != 2:
        raise ValueError("V must be n x d and sets l x k")
    if V.is_cuda or sets.is_cuda:
        raise ValueError("V and sets must be in host memory")
    if not V.is_contiguous() or not sets.is_contiguous():
        raise ValueError("tensors must be contiguous")
    if sets.dtype != torch.int32:
        raise TypeError("sets must be int32")
    prec = precision_of(V.dtype)
    n, d = V.shape
    l, k = sets.shape
    if out is None:
        out = torch.empty(l, dtype=torch.float32)
    elif out.is_cuda or out.dtype != torch.float32 or out.numel() != l or not out.is_contiguous():
        raise ValueError("out must be a contiguous host float32 tensor with l elements")
    dev = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
    with torch.cuda.device(dev):
        rc = load().exemplar_eval_streamed(_ptr(V), n, d, _ptr(sets), l, k, prec, int(rows_per_block), _ptr(out),
                                           _stream(stream))
    if rc != EXEMCL_OK:
        raise ExemclError(rc, "exemplar_eval_streamed")
    return out


def exemplar_gain(V, S, cands, out=None, stream=None):
    """out[j] = f(S u {cands[j]}) for fp32 V (see exemplar_gain in exemcl.h)."""
    import torch
    if V.dtype != torch.float32:
        raise TypeError("exemplar_gain takes float32 V")
    if S.dtype != torch.int32 or cands.dtype != torch.int32:
        raise TypeError("S and cands must be int32")
    if V.dim() != 2:
        raise ValueError("V must be n x d")
    n, d = V.shape
    l = cands.numel()
    if out is None:
        out = _empty(stream)(l, dtype=torch.float32, device=V.device)
    elif out.dtype != torch.float32 or out.numel() != l:
        raise ValueError("out must be float32 with one element per candidate")
    with _device_scope(_check_device(V, S if S.numel() else None, cands, out)):
        rc = load().exemplar_gain(_ptr(V), n, d, _ptr(S), S.numel(), _ptr(cands), l, _ptr(out),
                                  _stream(stream))
    _used(stream, V, S, cands, out)
    if rc != EXEMCL_OK:
        raise ExemclError(rc, "exemplar_gain")
    return out


def exemplar_greedy(V, K, S_out=None, f_out=None, stream=None):
    """Algorithm 1 for K rounds on fp32 V: returns (S_out, f_out), the point
    added in each round and f of the solution after it (see exemplar_greedy
    in exemcl.h)."""
    import torch
    if V.dtype != torch.float32:
        raise TypeError("exemplar_greedy takes float32 V")
    if V.dim() != 2:
        raise ValueError("V must be n x d")
    n, d = V.shape
    K = int(K)
    if S_out is None:
        S_out = _empty(stream)(max(K, 0), dtype=torch.int32, device=V.device)
    if f_out is None:
        f_out = _empty(stream)(max(K, 0), dtype=torch.float32, device=V.device)
    if S_out.dtype != torch.int32 or f_out.dtype != torch.float32 or S_out.numel() < K or f_out.numel() < K:
        raise ValueError("S_out must be int32 and f_out float32, with K elements each")
    with _device_scope(_check_device(V, S_out if K > 0 else None, f_out if K > 0 else None)):
        rc = load().exemplar_greedy(_ptr(V), n, d, K, _ptr(S_out), _ptr(f_out), _stream(stream))
    _used(stream, V, S_out, f_out)
    if rc != EXEMCL_OK:
        raise ExemclError(rc, "exemplar_greedy")
    return S_out, f_out


def exemplar_sqnorm(V, out=None, stream=None):
    """q[i] = ||v_i||^2 in fp32."""
    import torch
    prec = precision_of(V.dtype)
    n, d = V.shape
    if out is None:
        out = _empty(stream)(n, dtype=torch.float32, device=V.device)
    elif out.dtype != torch.float32 or out.numel() != n:
        raise ValueError("out must be float32 with n elements")
    with _device_scope(_check_device(V, out)):
        rc = load().exemplar_sqnorm(_ptr(V), n, d, prec, _ptr(out), _stream(stream))
    _used(stream, V, out)
    if rc != EXEMCL_OK:
        raise ExemclError(rc, "exemplar_sqnorm")
    return out


class MxRows(NamedTuple):
    """Rows of ``d`` coordinates as 8- or 4-bit elements with a power-of-two
    scale per 32 of them (the layout is in exemcl.h): uint8 tensors ``codes``
    (n x row bytes) and ``scales`` (n x dp/32), and the format, EXEMCL_MXFP4 or
    EXEMCL_MXFP8."""
    codes: Any
    scales: Any
    d: int
    format: int


_PRECISIONS: dict = {}  # precision_of, filled as types come


def _precision(dtype) -> int:
    p = _PRECISIONS.get(dtype)
    if p is None:
        p = _PRECISIONS[dtype] = precision_of(dtype)
    return p


def _mx_row(d: int, format: int):
    """(code bytes, scale bytes) of one stored row."""
    if format != EXEMCL_MXFP4 and format != EXEMCL_MXFP8:
        raise ValueError("format must be EXEMCL_MXFP4 or EXEMCL_MXFP8")
    if not 1 <= d <= 1 << 22:
        raise ValueError("microscaled rows have 1 to 2^22 coordinates")
    groups = (d + 127) // 128
    return groups * 16 * format, groups * 4


def _mx_check(q, name):
    """The rows of q, after its tensors' types and shapes were checked."""
    import torch
    codes, scales, d, format = q
    rb, rs = _mx_row(d, format)
    if codes.dtype != torch.uint8 or scales.dtype != torch.uint8 or codes.dim() != 2 or scales.dim() != 2 \
            or codes.shape[1] != rb or scales.shape[1] != rs:
        raise ValueError(f"{name}: codes must be uint8 n x {rb} and scales uint8 n x {rs}")
    n = codes.shape[0]
    if n != scales.shape[0]:
        raise ValueError(f"{name}: codes and scales have different numbers of rows")
    return n


def _mx_empty(n, d, format, device, empty):
    import torch
    rb, rs = _mx_row(d, format)
    return MxRows(empty((n, rb), dtype=torch.uint8, device=device),
                  empty((n, rs), dtype=torch.uint8, device=device), d, format)


def _check_gradient(name, tensors):
    """Results carry no autograd graph and no tangent: a gradient that is asked for, or
    a forward-mode derivative (which torch.no_grad() does not switch off), would be lost
    without a word.  (Codes of rows have none to lose.)"""
    import torch
    if name in ("exemplar_mx_quantize", "exemplar_w4_quantize"):
        return
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors):
        raise ValueError(f"{name} records no gradient: call it under torch.no_grad() or on detached tensors "
                         "(exemplar_rmsnorm_backward computes the norm's, exemplar_glu_backward the gated block's)")
    unpack = torch.autograd.forward_ad.unpack_dual
    if any(t is not None and unpack(t).tangent is not None for t in tensors):
        raise ValueError(f"{name} records no forward-mode derivative: call it on the primals "
                         "(torch.autograd.forward_ad.unpack_dual)")


_QUERIES = None  # (current device, its current raw stream, forward_ad), where PyTorch has them


def _queries():
    global _QUERIES
    if _QUERIES is None:
        import torch
        from torch.autograd import forward_ad
        _QUERIES = (getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device),
                    getattr(torch._C, "_cuda_getCurrentRawStream",
                            lambda dev: torch.cuda.current_stream(dev).cuda_stream),
                    # (tangents are there only inside a level; without its number always looked for)
                    forward_ad if hasattr(forward_ad, "_current_level") else SimpleNamespace(_current_level=0))
    return _QUERIES


def _run(name, tensors, stream, *args):
    """Call ``name`` of the library on the device of ``tensors`` (the first
    one's; None: not given) with ``args`` and the stream, and raise its error.
    The checks and messages are _check_device's; the calls on rows can be a few
    microseconds each, so the common case takes the short way."""
    current_device, raw_stream, forward_ad = _QUERIES or _queries()
    if forward_ad._current_level >= 0:
        _check_gradient(name, tensors)
    dev = tensors[0].get_device()
    for t in tensors:
        if t is not None and (t.get_device() != dev or not t.is_contiguous() or t.requires_grad or dev < 0):
            _check_gradient(name, tensors)
            _check_device(*tensors)
    fn = getattr(_LIB or load(), name)
    if dev == current_device():
        rc = fn(*args, raw_stream(dev) if stream is None else _stream(stream))
    else:
        import torch
        with torch.cuda.device(dev):
            rc = fn(*args, _stream(stream))
    if stream is not None:
        _used(stream, *tensors)
    if rc != EXEMCL_OK:
        raise ExemclError(rc, name)


def _at(t):
    """A tensor's address, for an argument that may be None."""
    return None if t is None else t.data_ptr()


def exemplar_mx_layout(d: int, format: int):
    """(code bytes, scale bytes) of one row of d coordinates; host only."""
    rb, rs = ctypes.c_int64(-1), ctypes.c_int64(-1)
    rc = load().exemplar_mx_layout(d, format, ctypes.byref(rb), ctypes.byref(rs))
    if rc != EXEMCL_OK:
        raise ExemclError(rc, "exemplar_mx_layout")
    return int(rb.value), int(rs.value)


def exemplar_mx_quantize(x, format, out=None, stream=None):
    """The rows of x (n x d) rounded to MxRows of ``format`` (see
    exemplar_mx_quantize in exemcl.h)."""
    if x.dim() != 2:
        raise ValueError("x must be n x d")
    prec = _precision(x.dtype)
    n, d = x.shape
    if out is None:
        out = _mx_empty(n, d, format, x.device, _empty(stream))
    elif out.d != d or out.format != format or _mx_check(out, "out") != n:
        raise ValueError("out must be MxRows of x's shape and the format")
    codes, scales = out.codes, out.scales
    _run("exemplar_mx_quantize", (x, codes, scales), stream, x.data_ptr(), n, d, prec, format, codes.data_ptr(),
         scales.data_ptr())
    return out


def exemplar_mx_dequantize(q, dtype, out=None, stream=None):
    """The values of MxRows q as an n x d tensor of ``dtype`` (see
    exemplar_mx_dequantize in exemcl.h)."""
    prec = _precision(dtype)
    n = _mx_check(q, "q")
    codes, scales, d, format = q
    if out is None:
        out = _empty(stream)((n, d), dtype=dtype, device=codes.device)
    elif out.dtype != dtype or out.shape != (n, d):
        raise ValueError("out must be an n x d tensor of the dtype")
    _run("exemplar_mx_dequantize", (codes, scales, out), stream, codes.data_ptr(), scales.data_ptr(), n, d, format, prec,
         out.data_ptr())
    return out


def exemplar_rmsnorm(x, weight=None, residual=None, eps=1e-6, format=None, stream=None):
    """(y, h, rstd): v = x + residual, h = v in x's type (x itself without a
    residual), y = v * weight / sqrt(mean(v^2) + eps) as a tensor of x's type,
    or as MxRows of ``format``, and rstd = 1 / sqrt(...) in float32 (see
    exemplar_rmsnorm in exemcl.h).  No autograd graph is recorded, and tensors
    that require a gradient are refused outside torch.no_grad():
    exemplar_rmsnorm_backward is the gradient."""
    import torch
    if x.dim() != 2:
        raise ValueError("x must be n x d")
    dtype, device = x.dtype, x.device
    prec = _precision(dtype)
    n, d = x.shape
    if weight is not None and (weight.dtype != dtype or weight.shape != (d,)):
        raise ValueError("weight must have x's type and d elements")
    if residual is not None and (residual.dtype != dtype or residual.shape != x.shape):
        raise ValueError("residual must have x's type and shape")
    empty, like = (torch.empty, torch.empty_like) if stream is None else _empty_on(stream)
    rstd = empty(n, dtype=torch.float32, device=device)
    h = x if residual is None else like(residual)
    if format is None or format == EXEMCL_MX_NONE:
        y = codes = like(x)
        scales, format = None, EXEMCL_MX_NONE
    else:
        y = _mx_empty(n, d, format, device, empty)
        codes, scales = y.codes, y.scales
    _run("exemplar_rmsnorm", (x, residual, weight), stream, x.data_ptr(), _at(residual), _at(weight), n, d, prec, eps,
         format, None if residual is None else h.data_ptr(), codes.data_ptr(), _at(scales), rstd.data_ptr())
    return y, h, rstd


def exemplar_rmsnorm_backward(dy, h, weight, rstd, dh=None, stream=None):
    """(dx, dweight) of exemplar_rmsnorm from the gradient dy of y, the h and
    rstd it returned, and dh, the gradient that reaches h another way; dx is
    the gradient of x and of the residual, dweight is float32 (see
    exemplar_rmsnorm_backward in exemcl.h)."""
    import torch
    if h.dim() != 2:
        raise ValueError("h must be n x d")
    dtype = h.dtype
    prec = _precision(dtype)
    n, d = h.shape
    for t, name in ((dy, "dy"), (dh, "dh")):
        if t is not None and (t.dtype != dtype or t.shape != h.shape):
            raise ValueError(f"{name} must have h's type and shape")
    if weight is not None and (weight.dtype != dtype or weight.shape != (d,)):
        raise ValueError("weight must have h's type and d elements")
    if rstd.dtype != torch.float32 or rstd.shape != (n,):
        raise ValueError("rstd must be float32 with n elements")
    empty, like = (torch.empty, torch.empty_like) if stream is None else _empty_on(stream)
    dx = like(h)
    dw = empty(d, dtype=torch.float32, device=h.device)
    _run("exemplar_rmsnorm_backward", (h, dy, weight, rstd, dh), stream, dy.data_ptr(), h.data_ptr(), _at(weight),
         rstd.data_ptr(), _at(dh), n, d, prec, dx.data_ptr(), dw.data_ptr())
    return dx, dw


def exemplar_mx_product(A, B, bias=None, dtype=None, out=None, stream=None):
    """C[i][j] = <A_i, B_j> + bias[j] for MxRows A (m rows of 8 or 4 bits) and
    B (n rows of 4 bits), as an m x n tensor of ``dtype`` (default float32; see
    exemplar_mx_product in exemcl.h)."""
    import torch
    dtype = torch.float32 if dtype is None else dtype
    prec = _precision(dtype)
    m, n = _mx_check(A, "A"), _mx_check(B, "B")
    a, a_scales, d, format = A
    b, b_scales = B.codes, B.scales
    if d != B.d:
        raise ValueError("A and B must have the same number of coordinates")
    if B.format != EXEMCL_MXFP4:
        raise ValueError("B must be EXEMCL_MXFP4 rows")
    if bias is not None and (bias.dtype != torch.float32 or bias.shape != (n,)):
        raise ValueError("bias must be float32 with one element per row of B")
    if out is None:
        out = _empty(stream)((m, n), dtype=dtype, device=a.device)
    elif out.dtype != dtype or out.shape != (m, n):
        raise ValueError("out must be an m x n tensor of the dtype")
    _run("exemplar_mx_product", (a, a_scales, b, b_scales, bias, out), stream, a.data_ptr(), a_scales.data_ptr(), m, format,
         b.data_ptr(), b_scales.data_ptr(), n, d, _at(bias), prec, out.data_ptr())
    return out


def exemplar_mx_eval(V, sets, out=None, stream=None):
    """out[j] = f(S_j) for MxRows V of 4 bits and the l x k int32 index matrix
    ``sets`` (see exemplar_mx_eval in exemcl.h)."""
    import torch
    n = _mx_check(V, "V")
    codes, scales, d, format = V
    if format != EXEMCL_MXFP4:
        raise ValueError("V must be EXEMCL_MXFP4 rows")
    if sets.dim() != 2:
        raise ValueError("sets must be l x k")
    if sets.dtype != torch.int32:
        raise TypeError("sets must be int32")
    l, k = sets.shape
    if out is None:
        out = _empty(stream)(l, dtype=torch.float32, device=codes.device)
    elif out.dtype != torch.float32 or out.numel() != l:
        raise ValueError("out must be float32 with l elements")
    _run("exemplar_mx_eval", (codes, scales, sets, out), stream, codes.data_ptr(), scales.data_ptr(), n, d, sets.data_ptr(),
         l, k, out.data_ptr())
    return out


class W4Rows(NamedTuple):
    """Weights of ``n`` rows of ``d`` coordinates in 4 bits, with a scale and zero
    point for ``group`` (32, 64 or 128) of them (the layout is in exemcl.h): uint8
    ``codes`` (np/16 x dp/128 x 1024) and int32 ``words`` (np/16 x dp/group x 16), np
    and dp the multiples of 16 and 128 that hold n and d."""
    codes: Any
    words: Any
    n: int
    d: int
    group: int


def _w4_check(q, name):
    """Checks the tensors of W4Rows q and their sizes."""
    codes, words, n, d, group = q
    if group != 128 and group != 64 and group != 32:
        raise ValueError(f"{name}: groups have 32, 64 or 128 coordinates")
    if n < 0 or not 1 <= d <= 4194304:
        raise ValueError(f"{name}: rows have 1 to 2^22 coordinates, and there are not less than 0")
    tiles, blocks = n + 15 >> 4, d + 127 >> 7
    uint8, int32 = _W4_TYPES or _w4_types()
    if codes.dtype is not uint8 or words.dtype is not int32 or codes.shape != (tiles, blocks, 1024) \
            or words.shape != (tiles, blocks * 128 // group, 16):
        raise ValueError(f"{name}: codes must be uint8 {tiles} x {blocks} x 1024 and words int32 "
                         f"{tiles} x {blocks * 128 // group} x 16")


_W4_TYPES = None


def _w4_types():
    global _W4_TYPES
    import torch
    _W4_TYPES = (torch.uint8, torch.int32)
    return _W4_TYPES


def _bias_check(b, f, name):
    if b is None:
        return
    import torch
    if b.dtype != torch.float32 or b.shape != (f,):
        raise ValueError(f"{name} must be float32 with {f} elements")


def _out(out, shape, x, stream):
    """``out``, checked, or a new tensor, of x's type and device."""
    dtype = x.dtype
    if out is None:
        return x.new_empty(shape) if stream is None else _empty(stream)(shape, dtype=dtype, device=x.device)
    if out.dtype != dtype or out.shape != shape:
        raise ValueError(f"out must be a {shape[0]} x {shape[1]} tensor of {dtype}")
    return out


def exemplar_glu(x, Wg, Wu, bg=None, bu=None, activation=EXEMCL_SILU, save=False, out=None, stream=None):
    """(h, g, u): g = x Wg' + bg, u = x Wu' + bu, h = a(g) * u for x (n x d) and
    weights of its type (f x d), biases in float32; g and u are kept for
    exemplar_glu_backward where ``save``, else None (see exemplar_glu in
    exemcl.h).  No autograd graph is recorded, and tensors that require a gradient
    are refused outside torch.no_grad(), those with a tangent always."""
    if x.dim() != 2 or Wg.dim() != 2:
        raise ValueError("x must be n x d and Wg f x d")
    dtype = x.dtype
    prec = _precision(dtype)
    n, d = x.shape
    f = Wg.shape[0]
    if Wg.dtype is not dtype or Wu.dtype is not dtype or Wg.shape != (f, d) or Wu.shape != (f, d):
        raise ValueError("Wg and Wu must have x's type, one shape and x's number of columns")
    if bg is not None:
        _bias_check(bg, f, "bg")
    if bu is not None:
        _bias_check(bu, f, "bu")
    h = _out(out, (n, f), x, stream)
    g = u = None
    if save:
        g, u = _out(None, (n, f), x, stream), _out(None, (n, f), x, stream)
    _run("exemplar_glu", (x, Wg, Wu) if bg is None and bu is None and out is None else (x, Wg, Wu, bg, bu, out), stream,
         x.data_ptr(), n, d, Wg.data_ptr(), Wu.data_ptr(), f, None if bg is None else bg.data_ptr(),
         None if bu is None else bu.data_ptr(), prec, activation, h.data_ptr(), None if g is None else g.data_ptr(),
         None if u is None else u.data_ptr())
    return h, g, u


def exemplar_glu_backward(dh, x, Wg, Wu, g, u, activation=EXEMCL_SILU, bias=False, stream=None):
    """(dx, dWg, dWu, dbg, dbu) of exemplar_glu from the gradient dh of h and the g
    and u it returned: dx and the weights' in x's type, the biases' in float32, None
    unless ``bias`` (see exemplar_glu_backward in exemcl.h, where any may be left out:
    here the first three are always computed)."""
    import torch
    if x.dim() != 2 or Wg.dim() != 2:
        raise ValueError("x must be n x d and Wg f x d")
    dtype = x.dtype
    prec = _precision(dtype)
    n, d = x.shape
    f = Wg.shape[0]
    if Wg.dtype != dtype or Wu.dtype != dtype or Wg.shape[1] != d or Wu.shape != Wg.shape:
        raise ValueError("Wg and Wu must have x's type, one shape and x's number of columns")
    for t, name in ((dh, "dh"), (g, "g"), (u, "u")):
        if t.dtype != dtype or t.shape != (n, f):
            raise ValueError(f"{name} must have x's type and be n x f")
    empty, like = (torch.empty, torch.empty_like) if stream is None else _empty_on(stream)
    dx, dWg, dWu = like(x), like(Wg), like(Wu)
    dbg = dbu = None
    if bias:
        dbg, dbu = empty(f, dtype=torch.float32, device=x.device), empty(f, dtype=torch.float32, device=x.device)
    _run("exemplar_glu_backward", (x, dh, Wg, Wu, g, u), stream, dh.data_ptr(), x.data_ptr(), Wg.data_ptr(), Wu.data_ptr(),
         g.data_ptr(), u.data_ptr(), n, d, f, prec, activation, dx.data_ptr(), dWg.data_ptr(), dWu.data_ptr(), _at(dbg),
         _at(dbu))
    return dx, dWg, dWu, dbg, dbu


def exemplar_w4_layout(n: int, d: int, group: int):
    """(bytes of codes, number of words) of n rows of d coordinates; host only."""
    cb, w = ctypes.c_int64(-1), ctypes.c_int64(-1)
    rc = load().exemplar_w4_layout(n, d, group, ctypes.byref(cb), ctypes.byref(w))
    if rc != EXEMCL_OK:
        raise ExemclError(rc, "exemplar_w4_layout")
    return int(cb.value), int(w.value)


def exemplar_w4_quantize(w, group=128, stream=None):
    """The rows of w (n x d) rounded to W4Rows (see exemplar_w4_quantize in exemcl.h)."""
    import torch
    if w.dim() != 2:
        raise ValueError("w must be n x d")
    prec = _precision(w.dtype)
    n, d = w.shape
    if group not in (32, 64, 128) or not 1 <= d <= 1 << 22:
        raise ValueError("groups have 32, 64 or 128 coordinates, rows 1 to 2^22")
    tiles, blocks = (n + 15) // 16, (d + 127) // 128
    empty = _empty(stream)
    q = W4Rows(empty((tiles, blocks, 1024), dtype=torch.uint8, device=w.device),
               empty((tiles, blocks * 128 // group, 16), dtype=torch.int32, device=w.device), n, d, group)
    _run("exemplar_w4_quantize", (w, q.codes, q.words), stream, w.data_ptr(), n, d, prec, group, q.codes.data_ptr(),
         q.words.data_ptr())
    return q


def exemplar_w4_dequantize(q, dtype, out=None, stream=None):
    """The values of W4Rows q as an n x d tensor of ``dtype``."""
    prec = _precision(dtype)
    _w4_check(q, "q")
    if out is None:
        out = _empty(stream)((q.n, q.d), dtype=dtype, device=q.codes.device)
    elif out.dtype != dtype or out.shape != (q.n, q.d):
        raise ValueError(f"out must be a {q.n} x {q.d} tensor of {dtype}")
    _run("exemplar_w4_dequantize", (q.codes, q.words, out), stream, q.codes.data_ptr(), q.words.data_ptr(), q.n, q.d,
         q.group, prec, out.data_ptr())
    return out


def exemplar_w4_product(x, W, bias=None, out=None, stream=None):
    """x W' + bias for x (n x d) and W4Rows W (f rows), as an n x f tensor of x's
    type; the bias is float32 (see exemplar_w4_product in exemcl.h)."""
    if x.dim() != 2:
        raise ValueError("x must be n x d")
    dtype = x.dtype
    prec = _PRECISIONS.get(dtype)
    if prec is None:
        prec = _precision(dtype)
    n, d = x.shape
    _w4_check(W, "W")
    codes, words, f, wd, group = W
    if wd != d:
        raise ValueError("x and W must have the same number of coordinates")
    if bias is not None:
        _bias_check(bias, f, "bias")
    y = _out(out, (n, f), x, stream)
    _run("exemplar_w4_product", (x, codes, words) if bias is None and out is None else (x, codes, words, bias, out), stream,
         x.data_ptr(), n, d, prec, codes.data_ptr(), words.data_ptr(), f, group, None if bias is None else bias.data_ptr(),
         y.data_ptr())
    return y


def exemplar_w4_glu(x, Wg, Wu, bg=None, bu=None, activation=EXEMCL_SILU, out=None, stream=None):
    """a(x Wg' + bg) * (x Wu' + bu) for x (n x d) and W4Rows of f rows with one group
    size, as an n x f tensor of x's type (see exemplar_w4_glu in exemcl.h)."""
    if x.dim() != 2:
        raise ValueError("x must be n x d")
    dtype = x.dtype
    prec = _PRECISIONS.get(dtype)
    if prec is None:
        prec = _precision(dtype)
    n, d = x.shape
    _w4_check(Wg, "Wg")
    _w4_check(Wu, "Wu")
    gc, gw, f, gd, group = Wg
    uc, uw, uf, ud, ugroup = Wu
    if gd != d or ud != d or uf != f or ugroup != group:
        raise ValueError("Wg and Wu must have x's number of coordinates, one number of rows and one group size")
    if bg is not None:
        _bias_check(bg, f, "bg")
    if bu is not None:
        _bias_check(bu, f, "bu")
    h = _out(out, (n, f), x, stream)
    few = bg is None and bu is None and out is None
    _run("exemplar_w4_glu", (x, gc, gw, uc, uw) if few else (x, gc, gw, uc, uw, bg, bu, out), stream, x.data_ptr(), n, d, prec,
         gc.data_ptr(), gw.data_ptr(), uc.data_ptr(), uw.data_ptr(), f, group, None if bg is None else bg.data_ptr(),
         None if bu is None else bu.data_ptr(), activation, h.data_ptr())
    return h


def exemplar_plan(n: int, d: int, l: int, k: int, precision: int = EXEMCL_FP32):
    """(path name, workspace bytes) exemplar_eval would use; host only."""
    path = ctypes.c_int(-1)
    ws = ctypes.c_int64(-1)
    rc = load().exemplar_plan(n, d, l, k, precision, ctypes.byref(path), ctypes.byref(ws))
    if rc != EXEMCL_OK:
        raise ExemclError(rc, "exemplar_plan")
    return PATH_NAMES.get(path.value, str(path.value)), int(ws.value)


def exemplar_prof_enable(on=True) -> None:
    """Record HIP events around the dominant kernel of following calls:
    True or 1 = every call, an integer N > 1 = every N-th call (the first
    included), False or 0 = stop."""
    every = int(on) if not isinstance(on, bool) else (1 if on else 0)
    rc = load().exemplar_prof_enable(every)
    if rc != EXEMCL_OK:
        raise ExemclError(rc, "exemplar_prof_enable")


def exemplar_prof_read():
    """(summed kernel milliseconds, launches) recorded since the last read."""
    ms = ctypes.c_double(0.0)
    cnt = ctypes.c_int64(0)
    rc = load().exemplar_prof_read(ctypes.byref(ms), ctypes.byref(cnt))
    if rc != EXEMCL_OK:
        raise ExemclError(rc, "exemplar_prof_read")
    return float(ms.value), int(cnt.value)


def exemplar_version() -> int:
    return int(load().exemplar_version())
