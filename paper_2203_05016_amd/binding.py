"""Thin ctypes binding of the shflbw C ABI (see ``include/shflbw.h``).

Argument marshalling only: every step of the hot path runs inside the
library's kernels.  torch tensors are used for device memory and for the
stream handle; numpy arrays for host-side inputs of the compressor.

The library is required: if ``libshflbw.so`` has not been built this module
raises at first use.  There is no CPU fallback.
"""
import ctypes
import os

import numpy as np

F16, BF16, F32 = 0, 1, 2
NCHW, CHWN = 0, 1

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libshflbw.so")
CALLS_PATH = os.path.join(_HERE, "_torch_calls.so")
_lib = None
_calls = None   # native calls on torch tensors (csrc/torch_calls.cpp), loaded with the first use; False: none

EXPORTS = [
    "shflbw_compress", "shflbw_pattern_search", "shflbw_destroy", "shflbw_info", "shflbw_row_indices",
    "shflbw_group_columns", "shflbw_decompress", "shflbw_device_bytes", "shflbw_bind_device",
    "shflbw_set_tuning", "shflbw_device_status", "shflbw_set_wait_limit", "shflbw_spmm", "shflbw_spmm_unbound",
    "shflbw_conv2d",
    "shflbw_layernorm_transpose", "shflbw_kv_cache_bytes", "shflbw_kv_write", "shflbw_kv_read",
    "shflbw_kv_attention_workspace", "shflbw_kv_attention", "shflbw_window_attention", "shflbw_status_string", "shflbw_last_error", "shflbw_last_kernel",
]


class ShflbwError(RuntimeError):
    def __init__(self, status, text):
        super().__init__("shflbw status %d (%s): %s" % (status, status_string(status), text))
        self.status = status


class _Cache(ctypes.Structure):   # shflbw_kv_cache
    _fields_ = [("data", ctypes.c_void_p)] + [(name, ctypes.c_int32) for name in
                                              ("pages", "page_tokens", "heads", "head_dim", "dtype")]


class _Sequences(ctypes.Structure):   # shflbw_kv_sequences
    _fields_ = [(name, ctypes.c_int32) for name in ("q_heads", "batch", "max_queries", "table_pages", "window", "sinks")] + \
               [(name, ctypes.c_int64) for name in ("tokens", "max_length", "table_ld")] + \
               [(name, ctypes.c_void_p) for name in ("table", "lengths", "starts")]


def lib():
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("%s is missing: build it with `python -m paper_2203_05016_amd.build`"
                               % LIB_PATH)
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, i64 = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64
        L.shflbw_compress.restype = i32
        L.shflbw_compress.argtypes = [vp, i32, vp, vp, i32, i32, i32, i32, ctypes.POINTER(vp)]
        L.shflbw_destroy.restype = None
        L.shflbw_destroy.argtypes = [vp]
        L.shflbw_info.restype = i32
        L.shflbw_info.argtypes = [vp] + [ctypes.POINTER(i32)] * 4 + \
            [ctypes.POINTER(i64), ctypes.POINTER(ctypes.c_double)]
        L.shflbw_row_indices.restype = i32
        L.shflbw_row_indices.argtypes = [vp, vp]
        L.shflbw_group_columns.restype = i32
        L.shflbw_group_columns.argtypes = [vp, i32, vp, i32]
        L.shflbw_decompress.restype = i32
        L.shflbw_decompress.argtypes = [vp, vp, i32]
        L.shflbw_device_bytes.restype = ctypes.c_size_t
        L.shflbw_device_bytes.argtypes = [vp]
        L.shflbw_bind_device.restype = i32
        L.shflbw_bind_device.argtypes = [vp, vp, vp]
        L.shflbw_set_tuning.restype = i32
        L.shflbw_set_tuning.argtypes = [vp, i32, i32]
        L.shflbw_device_status.restype = i32
        L.shflbw_device_status.argtypes = [vp, vp]
        L.shflbw_set_wait_limit.restype = i32
        L.shflbw_set_wait_limit.argtypes = [vp, i32]
        L.shflbw_spmm.restype = i32
        L.shflbw_spmm.argtypes = [vp, vp, i64, vp, i64, i64, i32, vp]
        L.shflbw_spmm_unbound.restype = i32
        L.shflbw_spmm_unbound.argtypes = [vp, vp, i64, vp, i64, i64, i32, vp]
        L.shflbw_conv2d.restype = i32
        L.shflbw_conv2d.argtypes = [vp, vp, vp] + [i32] * 10 + [i32, i32, vp]
        L.shflbw_pattern_search.restype = i32
        L.shflbw_pattern_search.argtypes = [vp, i32, i32, i32, i32, ctypes.c_double, ctypes.c_double,
                                            i32, i32, vp, vp]
        L.shflbw_layernorm_transpose.restype = i32
        L.shflbw_layernorm_transpose.argtypes = [vp, i64, vp, vp, ctypes.c_float, i32, vp, i64, i64,
                                                 i32, i32, vp]
        L.shflbw_kv_cache_bytes.restype = ctypes.c_size_t
        L.shflbw_kv_cache_bytes.argtypes = [i32] * 4
        cache, sequences = ctypes.POINTER(_Cache), ctypes.POINTER(_Sequences)
        L.shflbw_kv_write.restype = i32
        L.shflbw_kv_write.argtypes = [cache, vp, i64, vp, i64, vp, i64, vp]
        L.shflbw_kv_read.restype = i32
        L.shflbw_kv_read.argtypes = [cache, vp, i64, vp, i64, vp, i64, vp]
        L.shflbw_kv_attention_workspace.restype = i64
        L.shflbw_kv_attention_workspace.argtypes = [cache, sequences]
        L.shflbw_kv_attention.restype = i32
        L.shflbw_kv_attention.argtypes = [cache, sequences, vp, i64, vp, i64, vp, i64, vp]
        L.shflbw_window_attention.restype = i32
        L.shflbw_window_attention.argtypes = [vp, i64] * 4 + [i32, i32, i32, i64, vp, i32, i64, i32, i32, i32, vp]
        L.shflbw_status_string.restype = ctypes.c_char_p
        L.shflbw_status_string.argtypes = [i32]
        L.shflbw_last_error.restype = ctypes.c_char_p
        L.shflbw_last_error.argtypes = []
        L.shflbw_last_kernel.restype = ctypes.c_char_p
        L.shflbw_last_kernel.argtypes = []
        _lib = L
    return _lib


def calls():
    """The native calls on plain torch tensors, connected to the library; False where there are none
    for this interpreter and this torch.  They make the same checks as the Python code below, faster; the
    library they call is the same."""
    global _calls
    if _calls is None:
        try:
            _calls = _load_calls()
        except ImportError as e:
            import warnings
            warnings.warn("native calls not in use (%s); build them with `python -m paper_2203_05016_amd.build`" % e)
            _calls = False
    return _calls


def _load_calls():
    import importlib.machinery
    import importlib.util
    import torch
    if not os.path.exists(CALLS_PATH):
        raise ImportError("%s is missing" % CALLS_PATH)
    loader = importlib.machinery.ExtensionFileLoader("_torch_calls", CALLS_PATH)
    m = importlib.util.module_from_spec(importlib.util.spec_from_loader("_torch_calls", loader))
    loader.exec_module(m)
    if m.TORCH_VERSION != str(torch.__version__):
        raise ImportError("built for torch %s, this is %s" % (m.TORCH_VERSION, torch.__version__))
    L = lib()
    address = lambda f: ctypes.cast(f, ctypes.c_void_p).value
    m.connect(address(L.shflbw_spmm), address(L.shflbw_conv2d), address(L.shflbw_layernorm_transpose),
              torch._C._cuda_getCurrentRawStream)
    m.connect_attention(address(L.shflbw_kv_write), address(L.shflbw_kv_read), address(L.shflbw_kv_attention_workspace),
                        address(L.shflbw_kv_attention), address(L.shflbw_window_attention))
    return m


def status_string(status):
    return lib().shflbw_status_string(int(status)).decode()


def last_error():
    return lib().shflbw_last_error().decode()


def last_kernel():
    """Name of the kernel this thread's last spmm / conv2d call launched."""
    return lib().shflbw_last_kernel().decode()


def _check(rc):
    if rc < 0:
        raise ShflbwError(rc, last_error())
    return rc


def _host_ptr(a):
    return None if a is None else ctypes.c_void_p(a.ctypes.data)


def _stream_ptr(stream):
    import torch
    s = torch.cuda.current_stream() if stream is None else stream
    return s.cuda_stream


def _empty(shape, dtype, device, stream):
    """Memory of the stream that the work runs on: what was there before it, and what comes after, is ordered with it."""
    import torch
    if stream is None or torch.device(device).type != "cuda":
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _result(shape, dtype, device, stream):
    """The same for what the caller gets, whose own (current) stream may still read it when it is let go."""
    import torch
    t = _empty(shape, dtype, device, stream)
    if stream is not None and t.is_cuda:
        t.record_stream(torch.cuda.current_stream(t.device))
    return t


_YDTYPE = None   # torch dtype -> shflbw_dtype, filled on first use (torch is imported lazily)


def _ydtype(t):
    global _YDTYPE
    if _YDTYPE is None:
        import torch
        _YDTYPE = {torch.float16: F16, torch.bfloat16: BF16, torch.float32: F32}
    try:
        return _YDTYPE[t.dtype]
    except KeyError:
        raise TypeError("output tensor must be float16, bfloat16 or float32") from None


class Matrix:
    """Owner of one ``shflbw_matrix`` handle and, once bound, of the device
    buffer (a torch uint8 tensor) that holds its packed arrays."""

    def __init__(self, handle, bf16=False):
        self._h = handle
        self._dev = None
        self._plan = None  # what the native calls need to know of the bound matrix
        self.bf16 = bf16   # operand format: bfloat16 instead of float16
        self._info = None  # what shflbw_info reports: fixed once the matrix is packed
        self._odt = None

    def _operand_dtype(self):
        if self._odt is None:
            import torch
            self._odt = torch.bfloat16 if self.bf16 else torch.float16
        return self._odt

    def __del__(self):
        h, self._h = getattr(self, "_h", None), None
        if h and _lib is not None:
            _lib.shflbw_destroy(h)

    # -- host side
    def info(self):
        if self._info is None:
            M, K, V, G = (ctypes.c_int() for _ in range(4))
            nnz, sp = ctypes.c_int64(), ctypes.c_double()
            _check(lib().shflbw_info(self._h, M, K, V, G, nnz, sp))
            self._info = dict(M=M.value, K=K.value, V=V.value, groups=G.value, nnz=nnz.value,
                              sparsity=sp.value)
        return dict(self._info)

    def row_indices(self):
        out = np.empty(self.info()["M"], dtype=np.int32)
        _check(lib().shflbw_row_indices(self._h, _host_ptr(out)))
        return out

    def group_columns(self, g):
        n = _check(lib().shflbw_group_columns(self._h, g, None, 0))
        out = np.empty(n, dtype=np.int32)
        if n:
            _check(lib().shflbw_group_columns(self._h, g, _host_ptr(out), n))
        return out

    def decompress(self, ldw=None):
        i = self.info()
        ldw = i["K"] if ldw is None else ldw
        out = np.zeros((i["M"], ldw), dtype=np.uint16 if self.bf16 else np.float16)
        _check(lib().shflbw_decompress(self._h, _host_ptr(out), ldw))
        return out

    def device_bytes(self):
        return int(lib().shflbw_device_bytes(self._h))

    def set_tuning(self, kernel=0, tile_n=0):
        _check(lib().shflbw_set_tuning(self._h, kernel, tile_n))

    def set_wait_limit(self, tries):
        _check(lib().shflbw_set_wait_limit(self._h, tries))

    def device_status(self, stream=None):
        """Waits for the stream; raises ShflbwError (status -10) if a bounded wait of
        the slab kernel ran out in a launch on this matrix since the last call."""
        _check(lib().shflbw_device_status(self._h, _stream_ptr(stream)))

    # -- device side
    def bind_device(self, device="cuda:0", stream=None):
        import torch
        buf = _result(self.device_bytes(), torch.uint8, device, stream)
        _check(lib().shflbw_bind_device(self._h, ctypes.c_void_p(buf.data_ptr()),
                                        _stream_ptr(stream)))
        self._dev = buf
        native, info = calls(), self.info()
        self._plan = native.plan(self._h.value, info["M"], info["K"], self.bf16, buf.device.index) if native else None
        return self

    def _require_on_bound_device(self, t, what):
        """The C ABI takes bare addresses: it cannot tell a host tensor, or one on
        another GPU, from device memory of the GPU the matrix is bound to."""
        if self._dev is None:
            raise RuntimeError("call bind_device before %s" % what)
        if not t.is_cuda or t.device != self._dev.device:
            raise ValueError("%s must live on %s, where the matrix is bound (got %s)"
                             % (what, self._dev.device, t.device))

    def spmm(self, X, Y=None, out_dtype=None, stream=None):
        """Y = (W . mask) X for a device tensor X of shape (K, N) in the
        matrix's operand format (float16, or bfloat16).  The C ABI has no K
        argument and sees only addresses, so shapes, strides and devices are
        checked here, before anything is enqueued."""
        if Y is not None and stream is None and self._plan is not None:
            rc = _calls.spmm(self._plan, X, Y)   # None: not the plain case, all checks below
            if rc is not None:
                if rc < 0:
                    _check(rc)
                return Y
        if X.dtype != self._operand_dtype() or X.dim() != 2 or X.stride(1) != 1 and X.shape[1] > 1:
            raise TypeError("X must be a 2-D %s tensor with unit column stride" % self._operand_dtype())
        info = self.info()
        K, N = X.shape
        if K != info["K"]:
            raise ValueError("X has %d rows, the packed matrix has K = %d columns" % (K, info["K"]))
        if K > 1 and X.stride(0) < N:
            raise ValueError("rows of X overlap (row stride %d < N = %d)" % (X.stride(0), N))
        if Y is not None:
            if Y.dim() != 2 or tuple(Y.shape) != (info["M"], N):
                raise ValueError("Y must have shape (%d, %d), got %r" % (info["M"], N, tuple(Y.shape)))
            if N > 1 and Y.stride(1) != 1:
                raise ValueError("Y must have unit column stride")
            if Y.shape[0] > 1 and Y.stride(0) < N:
                raise ValueError("rows of Y overlap (row stride %d < N = %d)" % (Y.stride(0), N))
            _ydtype(Y)
        self._require_on_bound_device(X, "X")
        if Y is None:
            Y = _result((info["M"], N), out_dtype or self._operand_dtype(), X.device, stream)
        else:
            self._require_on_bound_device(Y, "Y")
        ldx = X.stride(0) if K > 1 else max(N, 1)
        ldy = Y.stride(0) if Y.shape[0] > 1 else max(N, 1)
        rc = lib().shflbw_spmm(self._h, X.data_ptr(), ldx, Y.data_ptr(), ldy, N, _ydtype(Y),
                               _stream_ptr(stream))
        if rc < 0:
            _check(rc)
        return Y

    def conv2d(self, inp, R, S, stride=(1, 1), pad=(0, 0), layout="NCHW", out=None,
               out_dtype=None, stream=None):
        """Masked conv2d of a contiguous device tensor in the matrix's operand format."""
        if out is not None and stream is None and self._plan is not None and layout in ("NCHW", "CHWN"):
            rc = _calls.conv2d(self._plan, inp, R, S, stride, pad, layout == "CHWN", out)   # None: not the plain case
            if rc is not None:
                if rc < 0:
                    _check(rc)
                return out
        if inp.dtype != self._operand_dtype() or not inp.is_contiguous() or inp.dim() != 4:
            raise TypeError("input must be a contiguous 4-D %s tensor" % self._operand_dtype())
        if layout not in ("NCHW", "CHWN"):
            raise ValueError("layout must be 'NCHW' or 'CHWN'")
        if layout == "NCHW":
            B, C, H, W = inp.shape
        else:
            C, H, W, B = inp.shape
        info = self.info()
        if C * R * S != info["K"]:
            raise ValueError("C_in*R*S = %d does not match the packed matrix's K = %d" % (C * R * S, info["K"]))
        if min(stride) < 1 or min(pad) < 0 or H + 2 * pad[0] < R or W + 2 * pad[1] < S:
            raise ValueError("bad stride, padding or kernel size")
        Ho = (H + 2 * pad[0] - R) // stride[0] + 1
        Wo = (W + 2 * pad[1] - S) // stride[1] + 1
        Cout = info["M"]
        shape = (B, Cout, Ho, Wo) if layout == "NCHW" else (Cout, Ho, Wo, B)
        if out is not None:
            if tuple(out.shape) != shape or not out.is_contiguous():
                raise ValueError("out must be a contiguous tensor of shape %r, got %r" % (shape, tuple(out.shape)))
            _ydtype(out)
        self._require_on_bound_device(inp, "input")
        if out is None:
            out = _result(shape, out_dtype or self._operand_dtype(), inp.device, stream)
        else:
            self._require_on_bound_device(out, "out")
        _check(lib().shflbw_conv2d(self._h, inp.data_ptr(), out.data_ptr(), B, C, H, W, R, S,
                                   stride[0], stride[1], pad[0], pad[1],
                                   NCHW if layout == "NCHW" else CHWN, _ydtype(out),
                                   _stream_ptr(stream)))
        return out


def compress(W, mask, perm, V, K=None):
    """shflbw_compress on numpy arrays: W (M, ldw) float16, or uint16 holding
    bfloat16 bit patterns (numpy has no such dtype), of which the first K
    columns are the matrix (default: all), mask (M, K) uint8 or None, perm
    (M,) int32 or None."""
    if W.dtype not in (np.float16, np.uint16) or W.ndim != 2:
        raise TypeError("W must be a 2-D float16 array, or uint16 holding bfloat16 bits")
    bf16 = W.dtype == np.uint16
    W = np.ascontiguousarray(W)
    M, ldw = W.shape
    K = ldw if K is None else K
    m = None if mask is None else np.ascontiguousarray(mask, dtype=np.uint8)
    p = None if perm is None else np.ascontiguousarray(perm, dtype=np.int32)
    if m is not None and m.shape != (M, K):
        raise ValueError("mask shape")
    if p is not None and p.shape != (M,):
        raise ValueError("perm shape")
    h = ctypes.c_void_p()
    _check(lib().shflbw_compress(_host_ptr(W), ldw, _host_ptr(m), _host_ptr(p), M, K, V,
                                 BF16 if bf16 else F16, ctypes.byref(h)))
    return Matrix(h, bf16)


def layernorm_transpose(x, gamma=None, beta=None, eps=1e-5, normalize=True, out=None, stream=None):
    """shflbw_layernorm_transpose on device tensors: x (N tokens, K features)
    float16 or bfloat16 with unit feature stride; returns the (K, N) matrix
    shflbw_spmm takes as X."""
    if out is not None and stream is None and (_calls or calls()):
        rc = _calls.layernorm_transpose(x, gamma, beta, eps, normalize, out)   # None: not the plain case
        if rc is not None:
            if rc < 0:
                _check(rc)
            return out
    import torch
    if x.dtype not in (torch.float16, torch.bfloat16) or x.dim() != 2 or x.stride(1) != 1:
        raise TypeError("x must be a 2-D float16 or bfloat16 tensor with unit feature stride")
    N, K = x.shape
    for t in (gamma, beta):
        if t is not None and (t.dtype != x.dtype or t.shape != (K,) or not t.is_contiguous()):
            raise TypeError("gamma and beta must be contiguous (K,) tensors of x's dtype")
    if out is not None and (out.dtype != x.dtype or out.shape != (K, N) or out.stride(1) != 1):
        raise TypeError("out must be a (K, N) tensor of x's dtype with unit token stride")
    for t in (x, out, gamma, beta):
        if t is not None and (not t.is_cuda or t.device != x.device):
            raise ValueError("x, gamma, beta and out must live on one GPU")
    if out is None:
        out = _result((K, N), x.dtype, x.device, stream)
    if (N > 1 and x.stride(0) < K) or (K > 1 and out.stride(0) < N):
        raise ValueError("rows of x or out overlap")
    ptr = lambda t: ctypes.c_void_p(None if t is None else t.data_ptr())
    _check(lib().shflbw_layernorm_transpose(ptr(x), x.stride(0) if N > 1 else K, ptr(gamma), ptr(beta),
                                            float(eps), 1 if normalize else 0, ptr(out),
                                            out.stride(0) if K > 1 else N, N, K,
                                            BF16 if x.dtype == torch.bfloat16 else F16,
                                            _stream_ptr(stream)))
    return out


def _columns(t, name, rows, dtype, tokens=None):
    """Checks a (rows, tokens) activation matrix; returns its leading dimension."""
    if t.dtype != dtype or t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise TypeError("%s must be a 2-D %s tensor with unit token stride" % (name, dtype))
    if t.shape[0] != rows or (tokens is not None and t.shape[1] != tokens):
        raise ValueError("%s must have shape (%d, %s), got %r" % (name, rows, "tokens" if tokens is None else tokens, tuple(t.shape)))
    n = t.shape[1]
    if rows > 1 and t.stride(0) < n:
        raise ValueError("rows of %s overlap (row stride %d < %d tokens)" % (name, t.stride(0), n))
    return t.stride(0) if rows > 1 else max(n, 1)


def _indices(t, name, size):
    import torch
    if t.dtype != torch.int32 or t.dim() != 1 or not t.is_contiguous():
        raise TypeError("%s must be a contiguous 1-D int32 tensor" % name)
    if t.shape[0] != size:
        raise ValueError("%s must have %d entries, got %d" % (name, size, t.shape[0]))


def _on(device, **tensors):
    for name, t in tensors.items():
        if t is not None and (not t.is_cuda or t.device != device):
            raise ValueError("%s must live on %s (got %s)" % (name, device, t.device))


def _natural(**numbers):
    for name, n in numbers.items():
        if isinstance(n, bool) or int(n) != n or not 0 <= n < 2 ** 31:
            raise ValueError("%s must be a whole number from 0 to 2^31 - 1, got %r" % (name, n))


class KVCache:
    """Keys and values of many sequences in 4 bits, in pages on a GPU (the format is shflbw_kv_cache's).

    Activations are (heads * head_dim, tokens) as ``Matrix.spmm`` takes and leaves them.  Slot
    ``page * page_tokens + place`` holds one token; which pages a sequence has is the caller's bookkeeping.
    The memory is this object's: one torch uint8 tensor, zeros at first."""

    _plan = None   # what the native calls need to know of the cache

    def __init__(self, pages, page_tokens, heads, head_dim, dtype, device="cuda:0"):
        import torch
        if dtype not in (torch.float16, torch.bfloat16):
            raise TypeError("dtype must be float16 or bfloat16")
        _natural(pages=pages, page_tokens=page_tokens, heads=heads, head_dim=head_dim)
        size = int(lib().shflbw_kv_cache_bytes(pages, page_tokens, heads, head_dim))
        if size == 0:
            raise ValueError("%s (got %d pages of %d, %d heads of %d)" % (last_error(), pages, page_tokens, heads, head_dim))
        self.pages, self.page_tokens, self.heads, self.head_dim, self.dtype = pages, page_tokens, heads, head_dim, dtype
        self._dev = torch.zeros(size, dtype=torch.uint8, device=device)
        bf16 = dtype == torch.bfloat16
        self._c = _Cache(self._dev.data_ptr(), pages, page_tokens, heads, head_dim, BF16 if bf16 else F16)
        native = calls()
        if native and self._dev.is_cuda:
            self._plan = native.cache_plan(self._dev.data_ptr(), pages, page_tokens, heads, head_dim, bf16, self._dev.device.index)

    @property
    def device(self):
        return self._dev.device

    def device_bytes(self):
        return self._dev.numel()

    def write(self, k, v, slots, stream=None):
        """Quantises column t of k and v into slot ``slots[t]`` (int32, on the GPU); slots outside the cache are skipped."""
        if stream is None and self._plan is not None:
            rc = _calls.kv_write(self._plan, k, v, slots)   # None: not the plain case, all checks below
            if rc is not None:
                _check(rc)
                return
        rows = self.heads * self.head_dim
        ldk = _columns(k, "k", rows, self.dtype)
        ldv = _columns(v, "v", rows, self.dtype, k.shape[1])
        _indices(slots, "slots", k.shape[1])
        _on(self.device, k=k, v=v, slots=slots)
        _check(lib().shflbw_kv_write(self._c, k.data_ptr(), ldk, v.data_ptr(), ldv, slots.data_ptr(), k.shape[1],
                                     _stream_ptr(stream)))

    def read(self, slots, k=None, v=None, stream=None):
        """(k, v) of the slots, (heads * head_dim, len(slots)) each; NaN for slots outside the cache."""
        if k is None and v is None and stream is None and self._plan is not None:
            both = _calls.kv_read(self._plan, slots)
            if both is not None:
                if type(both) is int:
                    _check(both)
                return both
        n, rows = slots.shape[0] if slots.dim() else 0, self.heads * self.head_dim
        _indices(slots, "slots", n)
        _on(self.device, slots=slots, k=k, v=v)
        k, v = (_result((rows, n), self.dtype, self.device, stream) if t is None else t for t in (k, v))
        ldk, ldv = _columns(k, "k", rows, self.dtype, n), _columns(v, "v", rows, self.dtype, n)
        _check(lib().shflbw_kv_read(self._c, slots.data_ptr(), n, k.data_ptr(), ldk, v.data_ptr(), ldv, _stream_ptr(stream)))
        return k, v

    def attention(self, q, table, lengths, starts=None, max_queries=1, max_length=None, window=0, sinks=0, out=None, stream=None):
        """Attention of the last tokens of every sequence over the cache, their own keys and values in it already.

        q (q_heads * head_dim, tokens): sequence b's queries are columns ``starts[b]`` to ``starts[b + 1] - 1``; without
        starts every sequence has one, column b.  table (batch, pages) int32: the sequence's pages in order.
        lengths (batch,) int32: its tokens in the cache.  max_queries: at least what any sequence has.  max_length: of the longest
        (all of the table's pages by default); it decides how the work is cut, and sequences past it only take longer.  window 0 is none; the first ``sinks`` tokens stay visible
        past it.  What is on the GPU is not looked at by the host: see shflbw_kv_sequences for what bad entries do."""
        if stream is None and self._plan is not None:
            r = _calls.kv_attention(self._plan, q, table, lengths, starts, max_queries, max_length, window, sinks, out)
            if r is not None:
                if type(r) is int:
                    _check(r)
                return r if out is None else out
        import torch
        if q.dtype != self.dtype or q.dim() != 2 or q.shape[0] == 0 or q.shape[0] % (self.heads * self.head_dim):
            raise TypeError("q must be a 2-D %s tensor with a multiple of %d rows" % (self.dtype, self.heads * self.head_dim))
        rows, tokens = q.shape
        ldq = _columns(q, "q", rows, self.dtype)
        if table.dtype != torch.int32 or table.dim() != 2 or (table.shape[1] > 1 and table.stride(1) != 1) or table.shape[1] < 1:
            raise TypeError("table must be a 2-D int32 tensor with unit page stride and a page or more")
        batch, width = table.shape
        if batch > 1 and table.stride(0) < width:
            raise ValueError("rows of table overlap")
        _indices(lengths, "lengths", batch)
        if starts is not None:
            _indices(starts, "starts", batch + 1)
        elif tokens != batch or max_queries != 1:
            raise ValueError("without starts every sequence has one query: q must have %d columns, max_queries be 1" % batch)
        max_length = width * self.page_tokens if max_length is None else max_length
        _natural(max_queries=max_queries, max_length=max_length, window=window, sinks=sinks)
        _on(self.device, q=q, table=table, lengths=lengths, starts=starts, out=out)
        if out is None:
            out = _result((rows, tokens), self.dtype, self.device, stream)
        ldo = _columns(out, "out", rows, self.dtype, tokens)
        s = _Sequences(rows // self.head_dim, batch, max_queries, width, window, sinks, tokens, max_length,
                       table.stride(0) if batch > 1 else width, table.data_ptr(), lengths.data_ptr(),
                       None if starts is None else starts.data_ptr())
        size = _check(lib().shflbw_kv_attention_workspace(self._c, s))
        work = _empty(size, torch.uint8, self.device, stream) if size else None
        _check(lib().shflbw_kv_attention(self._c, s, q.data_ptr(), ldq, out.data_ptr(), ldo, work.data_ptr() if size else None, size,
                                         _stream_ptr(stream)))
        return out


def window_attention(q, k, v, head_dim, starts=None, max_tokens=None, window=0, sinks=0, out=None, stream=None):
    """Causal attention of prompts to themselves: q (q_heads * head_dim, tokens), k and v (heads * head_dim, tokens).

    Sequence b is columns ``starts[b]`` to ``starts[b + 1] - 1`` (int32, on the GPU); without starts all columns are one.
    max_tokens: at least the longest sequence's tokens (all of them by default; workgroups are laid out for that many of every
    sequence, so name it where there are many).  A key at j is visible from p if
    j <= p and (window 0, or p - j < window, or j < sinks)."""
    if stream is None and (_calls or calls()):
        r = _calls.window_attention(q, k, v, head_dim, starts, max_tokens, window, sinks, out)   # None: not the plain case
        if r is not None:
            if type(r) is int:
                _check(r)
            return r if out is None else out
    import torch
    if q.dtype not in (torch.float16, torch.bfloat16) or q.dim() != 2 or k.dim() != 2:
        raise TypeError("q, k and v must be 2-D float16 or bfloat16 tensors")
    _natural(head_dim=head_dim, window=window, sinks=sinks)
    rows, tokens = q.shape
    if head_dim == 0 or rows == 0 or k.shape[0] == 0 or k.shape[0] % head_dim or rows % k.shape[0]:
        raise ValueError("q's rows must be a multiple of k's, and those of head_dim = %d (got %d and %d)" % (head_dim, rows, k.shape[0]))
    ldq = _columns(q, "q", rows, q.dtype)
    ldk, ldv = _columns(k, "k", k.shape[0], q.dtype, tokens), _columns(v, "v", k.shape[0], q.dtype, tokens)
    sequences = 1
    if starts is not None:
        sequences = starts.shape[0] - 1 if starts.dim() == 1 and starts.shape[0] else 0
        _indices(starts, "starts", sequences + 1)
    max_tokens = tokens if max_tokens is None else max_tokens
    _natural(max_tokens=max_tokens)
    _on(q.device, q=q, k=k, v=v, starts=starts, out=out)
    if out is None:
        out = _result((rows, tokens), q.dtype, q.device, stream)
    ldo = _columns(out, "out", rows, q.dtype, tokens)
    _check(lib().shflbw_window_attention(q.data_ptr(), ldq, k.data_ptr(), ldk, v.data_ptr(), ldv, out.data_ptr(), ldo,
                                         rows // head_dim, k.shape[0] // head_dim, head_dim, tokens,
                                         None if starts is None else starts.data_ptr(), sequences, max_tokens, window, sinks,
                                         BF16 if q.dtype == torch.bfloat16 else F16, _stream_ptr(stream)))
    return out


def pattern_search(W, V, alpha, beta=None, iterations=10):
    """shflbw_pattern_search on a numpy matrix (float16, or uint16 holding
    bfloat16 bit patterns): returns (perm, mask) ready for ``compress``.
    beta None = the paper's 2*alpha."""
    if W.dtype not in (np.float16, np.uint16) or W.ndim != 2:
        raise TypeError("W must be a 2-D float16 array, or uint16 holding bfloat16 bits")
    W = np.ascontiguousarray(W)
    M, K = W.shape
    perm = np.empty(M, dtype=np.int32)
    mask = np.empty((M, K), dtype=np.uint8)
    _check(lib().shflbw_pattern_search(_host_ptr(W), K, M, K, V, float(alpha),
                                       -1.0 if beta is None else float(beta), int(iterations),
                                       BF16 if W.dtype == np.uint16 else F16,
                                       _host_ptr(perm), _host_ptr(mask)))
    return perm, mask
