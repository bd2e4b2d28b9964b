"""ctypes binding of libturbomuon.so: argument marshalling only.

Every step of the orthogonalization runs in the library's HIP kernels; this
module checks tensor metadata, passes raw device pointers, the coefficient
table and the current HIP stream, and turns status codes into exceptions.
It never computes anything itself and has no fallback: a missing library is
an error.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libturbomuon.so")

TM_OK = 0
TM_ERR_INVALID_ARG = -1
TM_ERR_UNSUPPORTED = -2
TM_ERR_NO_MEMORY = -3
TM_ERR_HIP = -4

PRECOND = {"none": 0, "frobenius": 1, "frob": 1, "aol": 2, "schatten4": 3, "s4": 3}
PHASES = {"transpose_in": 0, "frob": 1, "gram": 2, "aol_vector": 3, "poly": 4, "update": 5,
          "apply_scale": 6, "copy_out": 7, "load_in": 8, "scale_a": 9, "opt_momentum": 10,
          "opt_apply": 11, "fused": 12, "layer_norm": 13, "layer_norm_backward": 14,
          "expert_matmul": 15, "expert_wgrad": 16, "policy_loss": 17, "policy_loss_backward": 18}
DTYPE_BF16, DTYPE_F32 = 0, 1
TM_MAX_DIM = 65536
TM_MAX_ITERS = 64

_c_i64p = ctypes.POINTER(ctypes.c_int64)
_c_fp = ctypes.POINTER(ctypes.c_float)
_vp, _i64, _f32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_float

_SIGNATURES = {
    "tm_orthogonalize": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64,
                                        ctypes.c_int64, ctypes.c_int, _c_fp, ctypes.c_int,
                                        ctypes.c_void_p]),
    "tm_orthogonalize_f32": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64,
                                            ctypes.c_int64, ctypes.c_int, _c_fp, ctypes.c_int,
                                            ctypes.c_void_p]),
    "tm_orthogonalize_grouped": (ctypes.c_int, [ctypes.POINTER(ctypes.c_void_p), _c_i64p, _c_i64p,
                                                ctypes.c_int64, ctypes.c_int, _c_fp, ctypes.c_int,
                                                ctypes.c_void_p]),
    "tm_orthogonalize_grouped_f32": (ctypes.c_int, [ctypes.POINTER(ctypes.c_void_p), _c_i64p,
                                                    _c_i64p, ctypes.c_int64, ctypes.c_int, _c_fp,
                                                    ctypes.c_int, ctypes.c_void_p]),
    "tm_muon_step_grouped": (ctypes.c_int, [ctypes.POINTER(ctypes.c_void_p),
                                            ctypes.POINTER(ctypes.c_void_p),
                                            ctypes.POINTER(ctypes.c_void_p), _c_i64p, _c_i64p,
                                            ctypes.c_int64, ctypes.c_float, ctypes.c_float,
                                            ctypes.c_int, ctypes.c_float, ctypes.c_int,
                                            ctypes.c_int, _c_fp, ctypes.c_int, ctypes.c_void_p]),
    "tm_orthogonalize_noalloc": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64,
                                                ctypes.c_int64, ctypes.c_int, _c_fp, ctypes.c_int,
                                                ctypes.c_void_p]),
    "tm_layer_norm": (ctypes.c_int, [_vp, _i64, _vp, _vp, _vp, _i64, _vp, _vp, _i64, _i64, _f32,
                                     ctypes.c_int, _vp]),
    "tm_layer_norm_backward": (ctypes.c_int, [_vp, _i64, _vp, _i64, _vp, _vp, _vp, _vp, _i64, _vp,
                                              _vp, _i64, _i64, ctypes.c_int, _vp]),
    "tm_expert_matmul": (ctypes.c_int, [_vp, _i64, _vp, _i64, _i64, _vp, _vp, _i64, _i64, _i64, _i64,
                                        _i64, ctypes.c_int, ctypes.c_int, _vp]),
    "tm_expert_wgrad": (ctypes.c_int, [_vp, _i64, _vp, _i64, _vp, _vp, _i64, _i64, _i64, _i64, _i64,
                                       _i64, ctypes.c_int, ctypes.c_int, _vp]),
    "tm_policy_loss": (ctypes.c_int, [_vp, _i64, _vp, _vp, _vp, _vp, _vp, _f32, _f32, _f32, _f32,
                                      _vp, _vp, _vp, _vp, _vp, _i64, _i64, _i64, ctypes.c_int, _vp]),
    "tm_policy_loss_backward": (ctypes.c_int, [_vp, _i64, _vp, _vp, _vp, _vp, _f32, _vp, _i64, _i64,
                                               _i64, ctypes.c_int, _vp]),
    "tm_schedule_tail": (_c_fp, [_c_fp, ctypes.c_int, ctypes.c_int]),
    "tm_workspace_bytes": (ctypes.c_uint64, [_c_i64p, _c_i64p, ctypes.c_int64, ctypes.c_int]),
    "tm_release_workspaces": (ctypes.c_int, []),
    "tm_timing_enable": (ctypes.c_int, [ctypes.c_int]),
    "tm_timing_read": (ctypes.c_int, [ctypes.c_int, ctypes.POINTER(ctypes.c_double),
                                      ctypes.POINTER(ctypes.c_int64)]),
    "tm_timing_reset": (ctypes.c_int, []),
    "tm_status_string": (ctypes.c_char_p, [ctypes.c_int]),
    "tm_last_error": (ctypes.c_char_p, []),
    "tm_version": (ctypes.c_char_p, []),
}

_lib = None


class TurboMuonError(RuntimeError):
    def __init__(self, fn: str, status: int, detail: str):
        self.status = status
        super().__init__(f"{fn} failed: {status_string(status)}: {detail}")


def lib() -> ctypes.CDLL:
    """Load libturbomuon.so (built in-tree by paper_2512_04632_amd.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing; build it with "
                               "`python -m paper_2512_04632_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            f = getattr(L, name)
            f.restype = res
            f.argtypes = args
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().tm_status_string(status).decode()


def last_error() -> str:
    return lib().tm_last_error().decode()


def version() -> str:
    return lib().tm_version().decode()


def _check(fn: str, status: int) -> None:
    if status != TM_OK:
        raise TurboMuonError(fn, status, last_error())


def _coeff_array(iters: int, coeffs):
    if coeffs is None:
        return None
    flat = [float(v) for row in coeffs for v in row]
    if len(flat) != 3 * iters:
        raise ValueError("coeffs must hold one (a, b, c) triple per iteration")
    return (ctypes.c_float * len(flat))(*flat)


def _precond(p) -> int:
    if isinstance(p, int):
        return p
    return PRECOND[p]


def _stream_handle(t, stream) -> int:
    import torch
    if stream is None:
        stream = torch.cuda.current_stream(t.device)
    return int(stream.cuda_stream)


def orthogonalize(x, iters: int = 4, coeffs: Optional[Sequence] = None, precond="aol",
                  stream=None):
    """Orthogonalize x in place: (m, n) or (batch, m, n), contiguous, bf16 or fp32, on a GPU.

    iters Newton-Schulz iterations after the pre-conditioning ("aol",
    "frobenius", "schatten4" or "none"); coeffs is an optional list of (a, b, c) per
    iteration.  Work is enqueued on `stream` (default: the current stream).
    Returns x.
    """
    import torch
    if not x.is_cuda:
        raise ValueError("x must be a device tensor")
    if not x.is_contiguous():
        raise ValueError("x must be contiguous")
    if x.dim() not in (2, 3):
        raise ValueError("x must be (m, n) or (batch, m, n)")
    if x.dtype == torch.bfloat16:
        fn = "tm_orthogonalize"
    elif x.dtype == torch.float32:
        fn = "tm_orthogonalize_f32"
    else:
        raise ValueError("x must be bfloat16 or float32")
    m, n = int(x.shape[-2]), int(x.shape[-1])
    batch = int(x.shape[0]) if x.dim() == 3 else 1
    carr = _coeff_array(iters, coeffs)
    with torch.cuda.device(x.device):
        st = getattr(lib(), fn)(ctypes.c_void_p(x.data_ptr()), m, n, batch, int(iters),
                                carr, _precond(precond), ctypes.c_void_p(_stream_handle(x, stream)))
    _check(fn, st)
    return x


TM_NOALLOC_SCRATCH_BYTES = 64 << 20


def orthogonalize_noalloc(x, iters: int = 4, coeffs: Optional[Sequence] = None, precond="aol",
                          stream=None):
    """tm_orthogonalize_noalloc: as orthogonalize for a bf16 (m, n) or (batch, m, n)
    tensor, with the workspace in the library's static per-GPU scratch array instead
    of an allocated one (raises TurboMuonError if the call needs more).  Returns x."""
    import torch
    if not x.is_cuda or not x.is_contiguous() or x.dim() not in (2, 3):
        raise ValueError("x must be a contiguous (m, n) or (batch, m, n) device tensor")
    if x.dtype != torch.bfloat16:
        raise ValueError("x must be bfloat16")
    m, n = int(x.shape[-2]), int(x.shape[-1])
    batch = int(x.shape[0]) if x.dim() == 3 else 1
    carr = _coeff_array(iters, coeffs)
    with torch.cuda.device(x.device):
        st = lib().tm_orthogonalize_noalloc(ctypes.c_void_p(x.data_ptr()), m, n, batch,
                                            int(iters), carr, _precond(precond),
                                            ctypes.c_void_p(_stream_handle(x, stream)))
    _check("tm_orthogonalize_noalloc", st)
    return x


def orthogonalize_grouped(xs: Sequence, iters: int = 4, coeffs: Optional[Sequence] = None,
                          precond="aol", stream=None):
    """Orthogonalize a list of 2-D tensors (any shapes, one dtype, one device) in place."""
    import torch
    xs = list(xs)
    if not xs:
        return xs
    dt, dev = xs[0].dtype, xs[0].device
    for t in xs:
        if not t.is_cuda or t.dim() != 2 or not t.is_contiguous():
            raise ValueError("grouped inputs must be contiguous 2-D device tensors")
        if t.dtype != dt or t.device != dev:
            raise ValueError("grouped inputs must share dtype and device")
    if dt == torch.bfloat16:
        fn = "tm_orthogonalize_grouped"
    elif dt == torch.float32:
        fn = "tm_orthogonalize_grouped_f32"
    else:
        raise ValueError("inputs must be bfloat16 or float32")
    cnt = len(xs)
    ptrs = (ctypes.c_void_p * cnt)(*[t.data_ptr() for t in xs])
    ms = (ctypes.c_int64 * cnt)(*[int(t.shape[0]) for t in xs])
    ns = (ctypes.c_int64 * cnt)(*[int(t.shape[1]) for t in xs])
    carr = _coeff_array(iters, coeffs)
    with torch.cuda.device(dev):
        st = getattr(lib(), fn)(ptrs, ms, ns, cnt, int(iters), carr, _precond(precond),
                                ctypes.c_void_p(_stream_handle(xs[0], stream)))
    _check(fn, st)
    return xs


def muon_step_grouped(params: Sequence, grads: Sequence, bufs: Sequence, lr: float,
                      momentum: float = 0.95, nesterov: bool = True, weight_decay: float = 0.0,
                      shape_scale: bool = True, iters: int = 4, coeffs: Optional[Sequence] = None,
                      precond="aol", stream=None):
    """One optimizer step (tm_muon_step_grouped) over lists of 2-D fp32 device tensors.

    params and bufs (momentum buffers) are updated in place; grads are read.
    """
    import torch
    params, grads, bufs = list(params), list(grads), list(bufs)
    if not (len(params) == len(grads) == len(bufs)):
        raise ValueError("params, grads and bufs must have the same length")
    if not params:
        return
    dev = params[0].device
    for w, g, m in zip(params, grads, bufs):
        for t in (w, g, m):
            if (not t.is_cuda or t.dtype != torch.float32 or t.dim() != 2 or
                    not t.is_contiguous() or t.device != dev):
                raise ValueError("optimizer tensors must be contiguous 2-D fp32 tensors on one device")
        if g.shape != w.shape or m.shape != w.shape:
            raise ValueError("gradient and momentum buffer must match the parameter's shape")
    cnt = len(params)
    W = (ctypes.c_void_p * cnt)(*[t.data_ptr() for t in params])
    G = (ctypes.c_void_p * cnt)(*[t.data_ptr() for t in grads])
    M = (ctypes.c_void_p * cnt)(*[t.data_ptr() for t in bufs])
    ms = (ctypes.c_int64 * cnt)(*[int(t.shape[0]) for t in params])
    ns = (ctypes.c_int64 * cnt)(*[int(t.shape[1]) for t in params])
    carr = _coeff_array(iters, coeffs)
    with torch.cuda.device(dev):
        st = lib().tm_muon_step_grouped(W, G, M, ms, ns, cnt, float(lr), float(momentum),
                                        1 if nesterov else 0, float(weight_decay),
                                        1 if shape_scale else 0, int(iters), carr,
                                        _precond(precond),
                                        ctypes.c_void_p(_stream_handle(params[0], stream)))
    _check("tm_muon_step_grouped", st)


# ------------------------------------------------------------------ operators

def _dtype_code(t, name: str) -> int:
    import torch
    if t.dtype is torch.bfloat16:
        return DTYPE_BF16
    if t.dtype is torch.float32:
        return DTYPE_F32
    raise ValueError(f"{name} must be bfloat16 or float32")


def _rows(t, name: str):
    """t as (tensor, rows, width, row stride): any leading dimensions that lie at one stride
    (others are copied), the last one contiguous."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dim() < 1:
        raise ValueError(f"{name} must have at least one dimension")
    d = t.shape[-1]
    if t.dim() != 2:
        t = t.reshape(-1, d) if d else t.reshape(t.shape[:-1].numel(), 0)
    rows = t.shape[0]
    ld = t.stride(0)
    if (d > 1 and t.stride(1) != 1) or (rows > 1 and ld < d):
        t = t.contiguous()
        ld = d
    return t, rows, d, max(ld, d)


def _same(t, like, name: str, shape, dtype=None):
    """Checks a companion tensor: device, shape, and type where one is asked for."""
    if t.device != like.device:
        raise ValueError(f"{name} must be on the same device")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, not {tuple(t.shape)}")
    if dtype is not None and t.dtype is not dtype:
        raise ValueError(f"{name} must be {dtype}")


def _vector(t, like, name: str, n: int, dtype):
    _same(t, like, name, (n,), dtype)
    return t if t.is_contiguous() else t.contiguous()


def _ptr(t):
    return None if t is None else t.data_ptr()


def _call(fn: str, device, stream, *args) -> None:
    """An operator's entry point on `device`, its last argument the stream."""
    import torch
    f = getattr(lib(), fn)
    if device.index == torch.cuda.current_device():
        if stream is None:
            handle = torch._C._cuda_getCurrentRawStream(device.index)
        else:
            handle = stream.cuda_stream
        st = f(*args, handle)
    else:
        with torch.cuda.device(device):
            if stream is None:
                stream = torch.cuda.current_stream(device)
            st = f(*args, stream.cuda_stream)
    if st != TM_OK:
        raise TurboMuonError(fn, st, last_error())


def layer_norm(x, weight=None, bias=None, eps: float = 1e-5, stream=None):
    """Layer norm over the last dimension of x (bf16 or fp32, any strides between rows).

    weight and bias are fp32 vectors or None.  Returns (y, mean, rstd): y of x's shape and
    type, mean and rstd fp32, one per row.
    """
    import torch
    code = _dtype_code(x, "x")
    rows_of, rows, d, ld = _rows(x, "x")
    f32 = torch.float32
    if weight is not None:
        weight = _vector(weight, x, "weight", d, f32)
    if bias is not None:
        bias = _vector(bias, x, "bias", d, f32)
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    mean, rstd = torch.empty((2, rows), dtype=f32, device=x.device).unbind(0)
    _call("tm_layer_norm", x.device, stream, rows_of.data_ptr(), ld, _ptr(weight), _ptr(bias), y.data_ptr(), d,
          mean.data_ptr(), rstd.data_ptr(), rows, d, eps, code)
    return y, mean, rstd


def layer_norm_backward(dy, x, mean, rstd, weight=None, param_grads: bool = True, stream=None):
    """Gradients of layer_norm: (dx, dweight, dbias), the last two fp32, or None without
    param_grads.  mean and rstd are layer_norm's; dy has x's shape and type."""
    import torch
    code = _dtype_code(x, "x")
    _same(dy, x, "dy", x.shape, x.dtype)
    x2, rows, d, ldx = _rows(x, "x")
    dy2, _, _, lddy = _rows(dy, "dy")
    f32 = torch.float32
    mean, rstd = _vector(mean, x, "mean", rows, f32), _vector(rstd, x, "rstd", rows, f32)
    if weight is not None:
        weight = _vector(weight, x, "weight", d, f32)
    dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    dweight = dbias = None
    if param_grads:
        dweight, dbias = torch.empty((2, d), dtype=f32, device=x.device).unbind(0)
    _call("tm_layer_norm_backward", x.device, stream, dy2.data_ptr(), lddy, x2.data_ptr(), ldx, _ptr(weight),
          mean.data_ptr(), rstd.data_ptr(), dx.data_ptr(), d, _ptr(dweight), _ptr(dbias), rows, d, code)
    return dx, dweight, dbias


def _matrices(w, like, name: str):
    """Stacked matrices as (tensor, row stride, matrix stride), the last dimension contiguous."""
    if w.dim() != 3:
        raise ValueError(f"{name} must be (experts, rows, columns)")
    if w.device != like.device or w.dtype is not like.dtype:
        raise ValueError(f"{name} must have x's type and device")
    e, r, c = w.shape
    if (c > 1 and w.stride(2) != 1) or (r > 1 and w.stride(1) < c) or \
            (e > 1 and w.stride(0) < (r - 1) * w.stride(1) + c):
        w = w.contiguous()
    return w, max(w.stride(1), c), w.stride(0) if e > 1 else 0


def _ends(ends, like):
    import torch
    if ends.dim() != 1 or ends.dtype is not torch.int32 or ends.device != like.device:
        raise ValueError("ends must be an int32 vector on x's device")
    return ends if ends.is_contiguous() else ends.contiguous()


def expert_matmul(x, w, ends, transposed: bool = False, stream=None):
    """y[i] = x[i] @ w[e] for the rows of each expert e (w[e].T with transposed).

    x is (rows, k), bf16 or fp32, rows sorted by expert; w is (experts, k, n), or (experts, n, k)
    with transposed; ends is an int32 device vector, ends[e] the number of rows up to expert e's
    last.  Rows after ends[-1] come out as zeros.  Nothing is synchronised.
    """
    import torch
    code = _dtype_code(x, "x")
    if x.dim() != 2:
        raise ValueError("x must be (rows, k)")
    x, rows, k, ldx = _rows(x, "x")
    w, ldw, stride_w = _matrices(w, x, "w")
    experts, n = w.shape[0], w.shape[1 if transposed else 2]
    if w.shape[2 if transposed else 1] != k:
        raise ValueError(f"w's matrices of {tuple(w.shape[1:])} do not fit rows of {k}")
    ends = _ends(ends, x)
    if ends.shape[0] != experts:
        raise ValueError("ends must hold one entry per expert")
    y = torch.empty((rows, n), dtype=x.dtype, device=x.device)
    _call("tm_expert_matmul", x.device, stream, x.data_ptr(), ldx, w.data_ptr(), ldw, stride_w, ends.data_ptr(),
          y.data_ptr(), n, rows, experts, k, n, 1 if transposed else 0, code)
    return y


def expert_wgrad(x, dy, ends, dtype=None, stream=None):
    """dw[e] = x_e.T @ dy_e for the rows of each expert: (experts, k, n), fp32 unless dtype says
    bf16 (for bf16 rows).  Experts without rows get zeros."""
    import torch
    code = _dtype_code(x, "x")
    if x.dim() != 2 or dy.dim() != 2:
        raise ValueError("x and dy must be (rows, k) and (rows, n)")
    _same(dy, x, "dy", (x.shape[0], dy.shape[1]), x.dtype)
    x, rows, k, ldx = _rows(x, "x")
    dy, _, n, lddy = _rows(dy, "dy")
    ends = _ends(ends, x)
    experts = ends.shape[0]
    dw = torch.empty((experts, k, n), dtype=dtype or torch.float32, device=x.device)
    _call("tm_expert_wgrad", x.device, stream, x.data_ptr(), ldx, dy.data_ptr(), lddy, ends.data_ptr(), dw.data_ptr(),
          n, k * n if experts > 1 else 0, rows, experts, k, n, code, _dtype_code(dw, "dtype"))
    return dw


def _policy_loss(logits, targets, old_logp, advantages, weights, ref_logp, clip_low, clip_high, kl, temperature,
                 stream, grad: bool, keep: bool):
    import torch
    code = _dtype_code(logits, "logits")
    if logits.dim() != 2:
        raise ValueError("logits must be (rows, vocabulary)")
    logits, rows, vocab, ld = _rows(logits, "logits")
    f32 = torch.float32
    targets = _vector(targets, logits, "targets", rows, torch.int64)
    old_logp = _vector(old_logp, logits, "old_logp", rows, f32)
    advantages = _vector(advantages, logits, "advantages", rows, f32)
    weights = _vector(weights, logits, "weights", rows, f32)
    if ref_logp is not None:
        ref_logp = _vector(ref_logp, logits, "ref_logp", rows, f32)
    loss = torch.empty((), dtype=f32, device=logits.device)
    dlogits = torch.empty((rows, vocab), dtype=logits.dtype, device=logits.device) if grad else None
    if keep:
        logp, lse, slope = torch.empty((3, rows), dtype=f32, device=logits.device).unbind(0)
    else:
        logp, lse, slope = torch.empty(rows, dtype=f32, device=logits.device), None, None
    _call("tm_policy_loss", logits.device, stream, logits.data_ptr(), ld, targets.data_ptr(), old_logp.data_ptr(),
          advantages.data_ptr(), weights.data_ptr(), _ptr(ref_logp), clip_low, clip_high, kl, temperature,
          loss.data_ptr(), logp.data_ptr(), _ptr(lse), _ptr(slope), _ptr(dlogits), vocab, rows, vocab, code)
    return loss, logp, lse, slope, dlogits


def policy_loss(logits, targets, old_logp, advantages, weights, ref_logp=None, clip_low: float = 0.2,
                clip_high: float = 0.2, kl: float = 0.0, temperature: float = 1.0, stream=None):
    """Clipped policy loss with a KL term over (rows, vocabulary) logits, bf16 or fp32:

        sum weight (-min(r A, clip(r, 1 - clip_low, 1 + clip_high) A) + kl (q - log q - 1)),
        r = exp(logp - old_logp), q = exp(ref_logp - logp)

    with logp the log probability of each row's int64 target at the temperature.  The other
    vectors are fp32, one entry per row; ref_logp None leaves the KL term out.  Rows of weight 0
    or with a negative target take no part.  Returns (loss, logp, lse, slope): the last two are
    what policy_loss_backward takes.
    """
    return _policy_loss(logits, targets, old_logp, advantages, weights, ref_logp, clip_low, clip_high, kl,
                        temperature, stream, False, True)[:4]


def policy_loss_with_grad(logits, targets, old_logp, advantages, weights, ref_logp=None, clip_low: float = 0.2,
                          clip_high: float = 0.2, kl: float = 0.0, temperature: float = 1.0, stream=None):
    """policy_loss and its gradient in one pass: (loss, logp, dlogits)."""
    loss, logp, _, _, dlogits = _policy_loss(logits, targets, old_logp, advantages, weights, ref_logp, clip_low,
                                             clip_high, kl, temperature, stream, True, False)
    return loss, logp, dlogits


def policy_loss_backward(logits, targets, lse, slope, grad=None, temperature: float = 1.0, stream=None):
    """Gradient by the logits from policy_loss's lse and slope, times grad (an fp32 scalar on the
    device; None: 1)."""
    import torch
    code = _dtype_code(logits, "logits")
    if logits.dim() != 2:
        raise ValueError("logits must be (rows, vocabulary)")
    logits, rows, vocab, ld = _rows(logits, "logits")
    targets = _vector(targets, logits, "targets", rows, torch.int64)
    lse = _vector(lse, logits, "lse", rows, torch.float32)
    slope = _vector(slope, logits, "slope", rows, torch.float32)
    if grad is not None:
        _same(grad, logits, "grad", (), torch.float32)
    dlogits = torch.empty((rows, vocab), dtype=logits.dtype, device=logits.device)
    _call("tm_policy_loss_backward", logits.device, stream, logits.data_ptr(), ld, targets.data_ptr(),
          lse.data_ptr(), slope.data_ptr(), _ptr(grad), temperature, dlogits.data_ptr(), vocab, rows, vocab, code)
    return dlogits


def schedule_tail(schedule: Sequence, iters: int) -> list:
    """The rows of a coefficient schedule that a call with `iters` iterations runs
    (tm_schedule_tail: the last `iters` rows)."""
    flat = [float(v) for row in schedule for v in row]
    rows = len(flat) // 3
    if rows * 3 != len(flat):
        raise ValueError("a schedule holds (a, b, c) triples")
    arr = (ctypes.c_float * max(len(flat), 1))(*flat)
    p = lib().tm_schedule_tail(arr, rows, int(iters))
    if not p:
        raise TurboMuonError("tm_schedule_tail", TM_ERR_INVALID_ARG, last_error())
    return [(p[3 * i], p[3 * i + 1], p[3 * i + 2]) for i in range(int(iters))]


def workspace_bytes(shapes: Sequence, dtype_bytes: int) -> int:
    cnt = len(shapes)
    ms = (ctypes.c_int64 * max(cnt, 1))(*[int(s[0]) for s in shapes])
    ns = (ctypes.c_int64 * max(cnt, 1))(*[int(s[1]) for s in shapes])
    return int(lib().tm_workspace_bytes(ms, ns, cnt, dtype_bytes))


def release_workspaces() -> None:
    _check("tm_release_workspaces", lib().tm_release_workspaces())


def timing_enable(on: bool = True) -> None:
    _check("tm_timing_enable", lib().tm_timing_enable(1 if on else 0))


def timing_reset() -> None:
    _check("tm_timing_reset", lib().tm_timing_reset())


def timing_read(phase: str):
    """(summed event milliseconds, launches) of one phase since the last reset."""
    ms = ctypes.c_double(0.0)
    n = ctypes.c_int64(0)
    _check("tm_timing_read", lib().tm_timing_read(PHASES[phase], ctypes.byref(ms), ctypes.byref(n)))
    return ms.value, n.value
