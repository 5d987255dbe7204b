"""Python binding of libelbow_moe (ctypes): argument marshalling only.

Every function has the name of the C entry point it calls (include/elbow_moe.h) and takes
torch tensors that live on the GPU; torch provides device memory and the current stream,
every step of the computation runs in the library's HIP kernels.  There is no fallback:
if the library is missing or a call fails, an exception is raised.

The calls are outside autograd: they read tensors that require gradients like any other, record
nothing, and their results never require gradients.  Where elb_ffn_forward is trained through,
elb_ffn_backward gives its gradients (an autograd.Function of the two is a user's few lines).
"""
from __future__ import annotations

import ctypes as C
import functools
import os
import threading
from typing import Optional

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libelbow_moe.so")

ELB_F32, ELB_BF16 = 0, 1
MODE_ELBOW, MODE_TOPK = 0, 1
MAX_EXPERTS, MAX_K = 64, 64

_lib = None


class ElbError(RuntimeError):
    def __init__(self, fn: str, status: int, msg: str):
        super().__init__("%s failed: %s (%s)" % (fn, _status_str(status), msg))
        self.status = status


class RouteParams(C.Structure):
    _fields_ = [("K", C.c_int32), ("eps", C.c_float), ("mode", C.c_int32),
                ("renormalize", C.c_int32)]


def lib():
    """Load libelbow_moe.so (built by paper_2608_04401_amd.build); raise if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError("libelbow_moe.so is not built (%s); run "
                           "`python -m paper_2608_04401_amd.build`" % LIB_PATH)
    L = C.CDLL(LIB_PATH)
    P, I32, I64, SZ = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
    sig = {
        "elb_abi_version": ([], C.c_int),
        "elb_status_str": ([C.c_int], C.c_char_p),
        "elb_last_error": ([], C.c_char_p),
        "elb_router_logits": ([P, P, I64, I32, I32, I32, P, P], C.c_int),
        "elb_route": ([P, I64, I32, C.POINTER(RouteParams), P, P, P, P], C.c_int),
        "elb_router_route": ([P, P, I64, I32, I32, I32, C.POINTER(RouteParams), P, P, P, P, P],
                             C.c_int),
        "elb_route_tail_random": ([P, P, I64, I32, C.POINTER(RouteParams), P, P, P, P],
                                  C.c_int),
        "elb_elbow_angle": ([P, I64, I32, C.c_float, P, P, P], C.c_int),
        "elb_dispatch_workspace_bytes": ([I64, I32], SZ),
        "elb_dispatch": ([P, P, I64, I32, I32, P, P, P, P, P, SZ, P], C.c_int),
        "elb_moe_workspace_bytes": ([I64, I32, I32, I32, I32, I32], SZ),
        "elb_moe_experts": ([P, P, P, P, P, P, P, I64, I32, I32, I32, I32, I32, P, P, SZ, P],
                            C.c_int),
        "elb_moe_forward": ([P, P, P, P, P, I64, I32, I32, I32, I32, C.POINTER(RouteParams), P,
                             P, SZ, P, P, P, P, P, P], C.c_int),
        "elb_packed_expert_bytes": ([I32, I32, I32], SZ),
        "elb_pack_expert_weights": ([P, P, I32, I32, I32, I32, P, P], C.c_int),
        "elb_moe_experts_packed": ([P, P, P, P, P, P, P, P, I64, I32, I32, I32, I32, I32, P, P,
                                    SZ, P], C.c_int),
        "elb_moe_forward_packed": ([P, P, P, P, P, P, I64, I32, I32, I32, I32,
                                    C.POINTER(RouteParams), P, P, SZ, P, P, P, P, P, P],
                                   C.c_int),
        "elb_moe_forward_noalloc": ([P, P, P, P, P, I64, I32, I32, I32, I32,
                                     C.POINTER(RouteParams), P, P, P, P, P, P, P], C.c_int),
        "elb_ffn_workspace_bytes": ([I64, I32, I32, I32], SZ),
        "elb_ffn_forward": ([P, P, P, P, I64, I32, I32, I32, P, P, P, SZ, P], C.c_int),
        "elb_ffn_backward_workspace_bytes": ([I64, I32, I32, I32], SZ),
        "elb_ffn_backward": ([P, P, P, P, P, I64, I32, I32, I32, P, P, P, P, SZ, P], C.c_int),
        "elb_quantize_rows": ([P, I64, I32, I32, P, P, P], C.c_int),
        "elb_gemm_i8": ([P, P, P, P, P, I64, I32, I32, I32, P, P], C.c_int),
        "elb_linear_i8_workspace_bytes": ([I64, I32, I32], SZ),
        "elb_linear_i8": ([P, P, P, P, I64, I32, I32, I32, P, P, SZ, P], C.c_int),
        "elb_ffn_i8_workspace_bytes": ([I64, I32, I32], SZ),
        "elb_ffn_forward_i8": ([P, P, P, P, P, P, I64, I32, I32, I32, P, P, SZ, P], C.c_int),
        "elb_calibrate_mfma_bf16": ([I32, I32, P, P], C.c_int64),
        "elb_calibrate_read_stream": ([P, I64, I32, P, P], C.c_int),
        "elb_profile_enable": ([C.c_int], C.c_int),
        "elb_profile_read": ([C.POINTER(C.c_char_p), C.POINTER(C.c_double),
                              C.POINTER(C.c_int64), C.c_int], C.c_int),
    }
    for name, (args, res) in sig.items():
        f = getattr(L, name)
        f.argtypes = args
        f.restype = res
    _lib = L
    return L


def _status_str(s: int) -> str:
    return lib().elb_status_str(s).decode()


def _check(fn: str, status: int):
    if status != 0:
        raise ElbError(fn, status, lib().elb_last_error().decode())


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _stream():
    """The current stream's handle.  (torch.cuda.current_stream() builds a Stream object first:
    2.8 us of a call's 10 to 19.)"""
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return ELB_F32
    if t.dtype == torch.bfloat16:
        return ELB_BF16
    raise TypeError("unsupported dtype %s (float32 or bfloat16)" % t.dtype)


def _dev(*ts):
    for t in ts:
        if t is None:
            continue
        if not t.is_cuda:
            raise ValueError("tensors must be on the GPU")
        if not t.is_contiguous():
            raise ValueError("tensors must be contiguous")


_ws = threading.local()  # .pool: {(device index, stream handle): buffer}
_WS_STREAMS = 8          # buffers a thread keeps


def workspace(nbytes: int, device, stream: Optional[int] = None) -> torch.Tensor:
    """Scratch of at least nbytes for one call on `stream` (None: the current one).

    A thread keeps one uint8 buffer per device and stream (the last _WS_STREAMS of them, until
    the thread ends): calls in order on one stream may share scratch, calls that can overlap, on
    other streams or from other threads, must not.  A buffer is allocated and used on one stream
    only, so one that is dropped (replaced by a larger one, or the oldest of too many) is safe
    with the allocator, which hands it on in that stream's order.  Under graph capture nothing
    is kept: the scratch then comes from the graph's own memory pool, which no call outside the
    graph uses and which lasts as long as the graph can be replayed."""
    nbytes = max(int(nbytes), 1)
    if torch._C._cuda_isCurrentStreamCapturing():
        return torch.empty(nbytes, dtype=torch.uint8, device=device)
    try:
        pool = _ws.pool
    except AttributeError:
        pool = _ws.pool = {}
    index = device.index if isinstance(device, torch.device) else torch.device(device).index
    key = (index, _stream() if stream is None else stream)
    buf = pool.get(key)
    if buf is None or buf.numel() < nbytes:
        pool.pop(key, None)
        if len(pool) >= _WS_STREAMS:
            del pool[next(iter(pool))]
        buf = pool[key] = torch.empty(nbytes, dtype=torch.uint8, device=device)
    return buf


def elb_abi_version() -> int:
    return lib().elb_abi_version()


def elb_router_logits(x: torch.Tensor, W_router: torch.Tensor) -> torch.Tensor:
    _dev(x, W_router)
    T, d = x.shape
    N = W_router.shape[0]
    logits = torch.empty((T, N), dtype=torch.float32, device=x.device)
    _check("elb_router_logits", lib().elb_router_logits(
        _ptr(x), _ptr(W_router), T, d, N, _dtype_code(x), _ptr(logits), _stream()))
    return logits


def elb_route(logits: torch.Tensor, K: int, eps: float = 1e-8, mode: int = MODE_ELBOW,
              renormalize: bool = False):
    """-> (k [T] int32, ids [T, K] int32, w [T, K] float32)"""
    _dev(logits)
    if logits.dtype != torch.float32:
        raise TypeError("logits must be float32")
    T, N = logits.shape
    k = torch.empty(T, dtype=torch.int32, device=logits.device)
    ids = torch.empty((T, K), dtype=torch.int32, device=logits.device)
    w = torch.empty((T, K), dtype=torch.float32, device=logits.device)
    p = RouteParams(K, eps, mode, int(renormalize))
    _check("elb_route", lib().elb_route(_ptr(logits), T, N, C.byref(p), _ptr(k), _ptr(ids),
                                        _ptr(w), _stream()))
    return k, ids, w


def elb_router_route(x: torch.Tensor, W_router: torch.Tensor, K: int, eps: float = 1e-8,
                     mode: int = MODE_ELBOW, renormalize: bool = False,
                     with_logits: bool = False):
    """-> (k [T], ids [T, K], w [T, K], logits [T, N] or None)"""
    _dev(x, W_router)
    T, d = x.shape
    N = W_router.shape[0]
    dev = x.device
    k = torch.empty(T, dtype=torch.int32, device=dev)
    ids = torch.empty((T, K), dtype=torch.int32, device=dev)
    w = torch.empty((T, K), dtype=torch.float32, device=dev)
    logits = torch.empty((T, N), dtype=torch.float32, device=dev) if with_logits else None
    p = RouteParams(K, eps, mode, int(renormalize))
    _check("elb_router_route", lib().elb_router_route(
        _ptr(x), _ptr(W_router), T, d, N, _dtype_code(x), C.byref(p), _ptr(logits), _ptr(k),
        _ptr(ids), _ptr(w), _stream()))
    return k, ids, w, logits


def elb_route_tail_random(logits: torch.Tensor, rand: torch.Tensor, K: int, eps: float = 1e-8,
                          mode: int = MODE_ELBOW, renormalize: bool = False):
    """-> (k_elbow [T] int32, ids [T, K] int32, w [T, K] float32); rand [T, N] float32"""
    _dev(logits, rand)
    if logits.dtype != torch.float32 or rand.dtype != torch.float32:
        raise TypeError("logits and rand must be float32")
    if rand.shape != logits.shape:
        raise ValueError("rand must have the shape of logits")
    T, N = logits.shape
    k = torch.empty(T, dtype=torch.int32, device=logits.device)
    ids = torch.empty((T, K), dtype=torch.int32, device=logits.device)
    w = torch.empty((T, K), dtype=torch.float32, device=logits.device)
    p = RouteParams(K, eps, mode, int(renormalize))
    _check("elb_route_tail_random", lib().elb_route_tail_random(
        _ptr(logits), _ptr(rand), T, N, C.byref(p), _ptr(k), _ptr(ids), _ptr(w), _stream()))
    return k, ids, w


def elb_elbow_angle(logits: torch.Tensor, eps: float = 1e-8):
    """-> (e [T] int32, theta [T] float32 degrees)"""
    _dev(logits)
    if logits.dtype != torch.float32:
        raise TypeError("logits must be float32")
    T, N = logits.shape
    e = torch.empty(T, dtype=torch.int32, device=logits.device)
    theta = torch.empty(T, dtype=torch.float32, device=logits.device)
    _check("elb_elbow_angle", lib().elb_elbow_angle(_ptr(logits), T, N, eps, _ptr(e),
                                                    _ptr(theta), _stream()))
    return e, theta


@functools.lru_cache(maxsize=256)
def elb_dispatch_workspace_bytes(T: int, N: int) -> int:
    return int(lib().elb_dispatch_workspace_bytes(T, N))


def elb_dispatch(k: torch.Tensor, ids: torch.Tensor, N: int):
    """-> (counts [N], offsets [N+1], row_token [T*K], inv [T, K]) int32"""
    _dev(k, ids)
    T, K = ids.shape
    dev = ids.device
    counts = torch.empty(N, dtype=torch.int32, device=dev)
    offsets = torch.empty(N + 1, dtype=torch.int32, device=dev)
    row_token = torch.full((T * K,), -1, dtype=torch.int32, device=dev)
    inv = torch.empty((T, K), dtype=torch.int32, device=dev)
    stream = _stream()
    ws = workspace(elb_dispatch_workspace_bytes(T, N), dev, stream)
    _check("elb_dispatch", lib().elb_dispatch(_ptr(k), _ptr(ids), T, N, K, _ptr(counts),
                                              _ptr(offsets), _ptr(row_token), _ptr(inv),
                                              _ptr(ws), ws.numel(), stream))
    return counts, offsets, row_token, inv


@functools.lru_cache(maxsize=256)
def elb_moe_workspace_bytes(T: int, d: int, N: int, m: int, K: int, dtype: int) -> int:
    return int(lib().elb_moe_workspace_bytes(T, d, N, m, K, dtype))


def elb_pack_expert_weights(W_gate_up: torch.Tensor, W_down: torch.Tensor) -> torch.Tensor:
    """The packed copy of bf16 expert weights (uint8 tensor), in the order the header gives.  No
    kernel of the library reads it any more: a program needs it only for code of its own."""
    _dev(W_gate_up, W_down)
    N, m2, d = W_gate_up.shape
    m = m2 // 2
    packed = torch.empty(int(lib().elb_packed_expert_bytes(N, d, m)), dtype=torch.uint8,
                         device=W_gate_up.device)
    _check("elb_pack_expert_weights", lib().elb_pack_expert_weights(
        _ptr(W_gate_up), _ptr(W_down), N, d, m, _dtype_code(W_gate_up), _ptr(packed),
        _stream()))
    return packed


def elb_moe_experts(x, W_gate_up, W_down, k, ids, w, residual=None, out=None,
                    packed=None) -> torch.Tensor:
    """packed: optional packed weights (elb_pack_expert_weights), kept for compatibility: not
    read, the same bits without."""
    _dev(x, W_gate_up, W_down, k, ids, w, residual, out, packed)
    T, d = x.shape
    N, m2, _ = W_gate_up.shape
    m = m2 // 2
    K = ids.shape[1]
    dt = _dtype_code(x)
    y = torch.empty_like(x) if out is None else out
    nb = elb_moe_workspace_bytes(T, d, N, m, K, dt)
    stream = _stream()
    ws = workspace(nb, x.device, stream)
    if packed is None:
        _check("elb_moe_experts", lib().elb_moe_experts(
            _ptr(x), _ptr(W_gate_up), _ptr(W_down), _ptr(k), _ptr(ids), _ptr(w),
            _ptr(residual), T, d, N, m, K, dt, _ptr(y), _ptr(ws), ws.numel(), stream))
    else:
        _check("elb_moe_experts_packed", lib().elb_moe_experts_packed(
            _ptr(x), _ptr(W_gate_up), _ptr(W_down), _ptr(packed), _ptr(k), _ptr(ids), _ptr(w),
            _ptr(residual), T, d, N, m, K, dt, _ptr(y), _ptr(ws), ws.numel(), stream))
    return y


def elb_moe_forward(x, W_router, W_gate_up, W_down, K: int = 8, eps: float = 1e-8,
                    mode: int = MODE_ELBOW, renormalize: bool = False, residual=None,
                    out=None, debug: bool = False, packed=None):
    """The whole layer.  Returns y, or (y, dict of intermediates) when debug=True.
    packed: optional packed weights (elb_pack_expert_weights), kept for compatibility: not read,
    the same bits without."""
    _dev(x, W_router, W_gate_up, W_down, residual, out, packed)
    T, d = x.shape
    N = W_router.shape[0]
    m = W_down.shape[2]
    dt = _dtype_code(x)
    dev = x.device
    y = torch.empty_like(x) if out is None else out
    nb = elb_moe_workspace_bytes(T, d, N, m, K, dt)
    stream = _stream()
    ws = workspace(nb, dev, stream)
    dbg = {}
    if debug:
        dbg = {"logits": torch.empty((T, N), dtype=torch.float32, device=dev),
               "k": torch.empty(T, dtype=torch.int32, device=dev),
               "ids": torch.empty((T, K), dtype=torch.int32, device=dev),
               "w": torch.empty((T, K), dtype=torch.float32, device=dev),
               "counts": torch.empty(N, dtype=torch.int32, device=dev)}
    p = RouteParams(K, eps, mode, int(renormalize))
    tail = (_ptr(dbg.get("logits")), _ptr(dbg.get("k")), _ptr(dbg.get("ids")),
            _ptr(dbg.get("w")), _ptr(dbg.get("counts")), stream)
    if packed is None:
        _check("elb_moe_forward", lib().elb_moe_forward(
            _ptr(x), _ptr(W_router), _ptr(W_gate_up), _ptr(W_down), _ptr(residual), T, d, N, m,
            dt, C.byref(p), _ptr(y), _ptr(ws), ws.numel(), *tail))
    else:
        _check("elb_moe_forward_packed", lib().elb_moe_forward_packed(
            _ptr(x), _ptr(W_router), _ptr(W_gate_up), _ptr(W_down), _ptr(packed),
            _ptr(residual), T, d, N, m, dt, C.byref(p), _ptr(y), _ptr(ws), ws.numel(), *tail))
    return (y, dbg) if debug else y


NOALLOC_SCRATCH_BYTES = 256 << 20


def elb_moe_forward_noalloc(x, W_router, W_gate_up, W_down, K: int = 8, eps: float = 1e-8,
                            mode: int = MODE_ELBOW, renormalize: bool = False, residual=None,
                            out=None, debug: bool = False):
    """The whole layer through the allocation-free entry point (the library's static scratch,
    no workspace).  Returns y, or (y, dict of intermediates) when debug=True."""
    _dev(x, W_router, W_gate_up, W_down, residual, out)
    T, d = x.shape
    N = W_router.shape[0]
    m = W_down.shape[2]
    dev = x.device
    y = torch.empty_like(x) if out is None else out
    dbg = {}
    if debug:
        dbg = {"logits": torch.empty((T, N), dtype=torch.float32, device=dev),
               "k": torch.empty(T, dtype=torch.int32, device=dev),
               "ids": torch.empty((T, K), dtype=torch.int32, device=dev),
               "w": torch.empty((T, K), dtype=torch.float32, device=dev),
               "counts": torch.empty(N, dtype=torch.int32, device=dev)}
    p = RouteParams(K, eps, mode, int(renormalize))
    _check("elb_moe_forward_noalloc", lib().elb_moe_forward_noalloc(
        _ptr(x), _ptr(W_router), _ptr(W_gate_up), _ptr(W_down), _ptr(residual), T, d, N, m,
        _dtype_code(x), C.byref(p), _ptr(y), _ptr(dbg.get("logits")), _ptr(dbg.get("k")),
        _ptr(dbg.get("ids")), _ptr(dbg.get("w")), _ptr(dbg.get("counts")), _stream()))
    return (y, dbg) if debug else y


def elb_moe_forward_prepared(x, W_router, W_gate_up, W_down, K: int = 8, eps: float = 1e-8,
                             mode: int = MODE_ELBOW, renormalize: bool = False, residual=None,
                             out=None, packed=None):
    """elb_moe_forward with its arguments marshalled once: returns (call, y), where call() enqueues
    the layer on the stream that was current here and raises on a failed status.  For timing
    loops, where the per-call argument checks would otherwise add host time.  call() uses the
    scratch of this thread and stream, so it is for the thread that prepared it."""
    _dev(x, W_router, W_gate_up, W_down, residual, out, packed)
    T, d = x.shape
    N = W_router.shape[0]
    m = W_down.shape[2]
    dt = _dtype_code(x)
    y = torch.empty_like(x) if out is None else out
    ws = workspace(elb_moe_workspace_bytes(T, d, N, m, K, dt), x.device)
    p = RouteParams(K, eps, mode, int(renormalize))
    L = lib()
    if packed is None:
        fn, name = L.elb_moe_forward, "elb_moe_forward"
        args = (_ptr(x), _ptr(W_router), _ptr(W_gate_up), _ptr(W_down), _ptr(residual), T, d, N,
                m, dt, C.byref(p), _ptr(y), _ptr(ws), ws.numel(), None, None, None, None, None,
                _stream())
    else:
        fn, name = L.elb_moe_forward_packed, "elb_moe_forward_packed"
        args = (_ptr(x), _ptr(W_router), _ptr(W_gate_up), _ptr(W_down), _ptr(packed),
                _ptr(residual), T, d, N, m, dt, C.byref(p), _ptr(y), _ptr(ws), ws.numel(), None,
                None, None, None, None, _stream())
    keep = (p, ws, y)  # referenced by the closure: the parameter block and buffers stay alive

    def call():
        rc = fn(*args)
        if rc != 0:
            _check(name, rc)
        return keep
    return call, y


def _want(name: str, t: Optional[torch.Tensor], shape, dtype: torch.dtype, device: int):
    """t: None, or a contiguous tensor of that shape and type on the current device (_device())."""
    if t is None or (t.dtype is dtype and t.shape == shape and t.is_contiguous()
                     and t.get_device() == device):
        return
    if t.get_device() != device:
        raise ValueError("%s must be on the current GPU" % name)
    if t.dtype != dtype:
        raise TypeError("%s must be %s, not %s" % (name, dtype, t.dtype))
    if t.shape != shape:
        raise ValueError("%s must have shape %s, not %s" % (name, tuple(shape), tuple(t.shape)))
    raise ValueError("%s must be contiguous" % name)


def _device(*ts) -> int:
    """The current device's index (tensors on the CPU are refused before it is asked for)."""
    for t in ts:
        if not t.is_cuda:
            raise ValueError("tensors must be on the GPU")
    return torch._C._cuda_getDevice()


def _matrix(name: str, t: torch.Tensor):
    if t.dim() != 2:
        raise ValueError("%s must have two dimensions, not %d" % (name, t.dim()))
    return t.shape


def _ffn_dims(x, W_gate_up, W_down):
    """(T, d, m, dtype code, device) of the dense block; its operands checked."""
    T, d = _matrix("x", x)
    m = _matrix("W_down", W_down)[1]
    dt = _dtype_code(x)
    dev = _device(x)
    _want("x", x, (T, d), x.dtype, dev)
    _want("W_gate_up", W_gate_up, (2 * m, d), x.dtype, dev)
    _want("W_down", W_down, (d, m), x.dtype, dev)
    return T, d, m, dt, dev


@functools.lru_cache(maxsize=256)
def elb_ffn_workspace_bytes(T: int, d: int, m: int, dtype: int) -> int:
    return int(lib().elb_ffn_workspace_bytes(T, d, m, dtype))


def elb_ffn_forward(x, W_gate_up, W_down, residual=None, out=None, keep: bool = False):
    """The dense gated feed-forward block.  -> y, or with keep=True (y, gate_up): gate_up
    [T, 2m] float32 is what elb_ffn_backward needs of the forward pass.  out may be residual or x.
    Outside autograd: y never requires a gradient."""
    T, d, m, dt, dev = _ffn_dims(x, W_gate_up, W_down)
    _want("residual", residual, (T, d), x.dtype, dev)
    _want("out", out, (T, d), x.dtype, dev)
    y = torch.empty_like(x) if out is None else out
    gate_up = torch.empty((T, 2 * m), dtype=torch.float32, device=x.device) if keep else None
    stream = _stream()
    ws = workspace(elb_ffn_workspace_bytes(T, d, m, dt), x.device, stream)
    _check("elb_ffn_forward", lib().elb_ffn_forward(
        _ptr(x), _ptr(W_gate_up), _ptr(W_down), _ptr(residual), T, d, m, dt, _ptr(y),
        _ptr(gate_up), _ptr(ws), ws.numel(), stream))
    return (y, gate_up) if keep else y


@functools.lru_cache(maxsize=256)
def elb_ffn_backward_workspace_bytes(T: int, d: int, m: int, dtype: int) -> int:
    return int(lib().elb_ffn_backward_workspace_bytes(T, d, m, dtype))


def elb_ffn_backward(dy, x, W_gate_up, W_down, gate_up, need=(True, True, True)):
    """-> (dx, dW_gate_up, dW_down), None where need is false; gate_up from
    elb_ffn_forward(..., keep=True)."""
    T, d, m, dt, dev = _ffn_dims(x, W_gate_up, W_down)
    _want("dy", dy, (T, d), x.dtype, dev)
    _want("gate_up", gate_up, (T, 2 * m), torch.float32, dev)
    dx, dWgu, dWd = (torch.empty_like(t) if n else None
                     for t, n in zip((x, W_gate_up, W_down), need))
    stream = _stream()
    ws = workspace(elb_ffn_backward_workspace_bytes(T, d, m, dt), x.device, stream)
    _check("elb_ffn_backward", lib().elb_ffn_backward(
        _ptr(dy), _ptr(x), _ptr(W_gate_up), _ptr(W_down), _ptr(gate_up), T, d, m, dt, _ptr(dx),
        _ptr(dWgu), _ptr(dWd), _ptr(ws), ws.numel(), stream))
    return dx, dWgu, dWd


def elb_quantize_rows(x: torch.Tensor):
    """-> (q [T, d] int8, scale [T] float32): q scale[:, None] stands for x"""
    T, d = _matrix("x", x)
    dt = _dtype_code(x)
    _want("x", x, (T, d), x.dtype, _device(x))
    q = torch.empty((T, d), dtype=torch.int8, device=x.device)
    scale = torch.empty(T, dtype=torch.float32, device=x.device)
    _check("elb_quantize_rows", lib().elb_quantize_rows(_ptr(x), T, d, dt, _ptr(q), _ptr(scale),
                                                        _stream()))
    return q, scale


def elb_gemm_i8(q, scale, W, W_scale, dtype: torch.dtype = torch.bfloat16, residual=None,
                out=None) -> torch.Tensor:
    """y [T, n] of dtype (bfloat16 or float32) from q [T, k] int8 and W [n, k] int8.  out may be
    residual."""
    T, k = _matrix("q", q)
    n = _matrix("W", W)[0]
    dev = _device(q)
    _want("q", q, (T, k), torch.int8, dev)
    _want("scale", scale, (T,), torch.float32, dev)
    _want("W", W, (n, k), torch.int8, dev)
    _want("W_scale", W_scale, (n,), torch.float32, dev)
    _want("residual", residual, (T, n), dtype, dev)
    _want("out", out, (T, n), dtype, dev)
    y = torch.empty((T, n), dtype=dtype, device=q.device) if out is None else out
    _check("elb_gemm_i8", lib().elb_gemm_i8(
        _ptr(q), _ptr(scale), _ptr(W), _ptr(W_scale), _ptr(residual), T, n, k, _dtype_code(y),
        _ptr(y), _stream()))
    return y


@functools.lru_cache(maxsize=256)
def elb_linear_i8_workspace_bytes(T: int, n: int, k: int) -> int:
    return int(lib().elb_linear_i8_workspace_bytes(T, n, k))


def elb_linear_i8(x, W, W_scale, residual=None, out=None) -> torch.Tensor:
    """y [T, n] = x [T, k], quantised by rows on the way, times W [n, k] int8.  out may be residual,
    not x."""
    T, k = _matrix("x", x)
    n = _matrix("W", W)[0]
    dt = _dtype_code(x)
    dev = _device(x)
    _want("x", x, (T, k), x.dtype, dev)
    _want("W", W, (n, k), torch.int8, dev)
    _want("W_scale", W_scale, (n,), torch.float32, dev)
    _want("residual", residual, (T, n), x.dtype, dev)
    _want("out", out, (T, n), x.dtype, dev)
    y = torch.empty((T, n), dtype=x.dtype, device=x.device) if out is None else out
    stream = _stream()
    ws = workspace(elb_linear_i8_workspace_bytes(T, n, k), x.device, stream)
    _check("elb_linear_i8", lib().elb_linear_i8(
        _ptr(x), _ptr(W), _ptr(W_scale), _ptr(residual), T, n, k, dt, _ptr(y), _ptr(ws),
        ws.numel(), stream))
    return y


@functools.lru_cache(maxsize=256)
def elb_ffn_i8_workspace_bytes(T: int, d: int, m: int) -> int:
    return int(lib().elb_ffn_i8_workspace_bytes(T, d, m))


def elb_ffn_forward_i8(x, W_gate_up, gate_up_scale, W_down, down_scale, residual=None,
                       out=None) -> torch.Tensor:
    """The dense gated feed-forward block with int8 weights (elb_quantize_rows of the float
    ones): W_gate_up [2m, d], gate_up_scale [2m], W_down [d, m], down_scale [d].  out may be
    residual or x."""
    T, d = _matrix("x", x)
    m = _matrix("W_down", W_down)[1]
    dt = _dtype_code(x)
    dev = _device(x)
    _want("x", x, (T, d), x.dtype, dev)
    _want("W_gate_up", W_gate_up, (2 * m, d), torch.int8, dev)
    _want("gate_up_scale", gate_up_scale, (2 * m,), torch.float32, dev)
    _want("W_down", W_down, (d, m), torch.int8, dev)
    _want("down_scale", down_scale, (d,), torch.float32, dev)
    _want("residual", residual, (T, d), x.dtype, dev)
    _want("out", out, (T, d), x.dtype, dev)
    y = torch.empty_like(x) if out is None else out
    stream = _stream()
    ws = workspace(elb_ffn_i8_workspace_bytes(T, d, m), x.device, stream)
    _check("elb_ffn_forward_i8", lib().elb_ffn_forward_i8(
        _ptr(x), _ptr(W_gate_up), _ptr(gate_up_scale), _ptr(W_down), _ptr(down_scale),
        _ptr(residual), T, d, m, dt, _ptr(y), _ptr(ws), ws.numel(), stream))
    return y


def elb_calibrate_read_stream(buf: torch.Tensor, blocks: int, out: torch.Tensor) -> None:
    """Enqueue the read-only stream over the bytes of buf (out: blocks * 4 int32 words)."""
    _dev(buf, out)
    _check("elb_calibrate_read_stream", lib().elb_calibrate_read_stream(
        _ptr(buf), buf.numel() * buf.element_size(), blocks, _ptr(out), _stream()))


def elb_calibrate_mfma_bf16(blocks: int, iters: int) -> int:
    """Enqueue the back-to-back MFMA calibration kernel; returns the MFMA instruction count
    (each v_mfma_f32_32x32x16_bf16 is 32 * 32 * 16 * 2 FLOPs)."""
    out = torch.empty(blocks * 4, dtype=torch.float32, device="cuda")
    n = lib().elb_calibrate_mfma_bf16(blocks, iters, _ptr(out), _stream())
    if n < 0:
        _check("elb_calibrate_mfma_bf16", -n)
    return int(n)


def elb_profile_enable(on=True) -> None:
    """on: False/0 off, True/1 every launch, 2 the grouped expert GEMMs only."""
    _check("elb_profile_enable", lib().elb_profile_enable(int(on)))


def elb_profile_read() -> dict:
    """{kernel name: (total ms, launches)} since the last read; clears the records."""
    cap = 64
    names = (C.c_char_p * cap)()
    ms = (C.c_double * cap)()
    n_l = (C.c_int64 * cap)()
    n = lib().elb_profile_read(names, ms, n_l, cap)
    if n < 0:
        _check("elb_profile_read", -n)
    return {names[i].decode(): (ms[i], int(n_l[i])) for i in range(min(n, cap))}
