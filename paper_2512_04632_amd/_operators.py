"""ctypes binding of the operators around the optimizer: argument marshalling only.

Called as attributes of ``_lib``.  Each function checks its tensors' metadata,
allocates its results, and passes raw device pointers and the current stream
(``stream=`` makes another one current for the call; as everywhere, a tensor made
on one stream is used on another only after an event or a wait);
all arithmetic runs in the library's kernels.  A small call is bound by its
host time, so the common case (contiguous tensors on the current device) takes
few steps.
"""
from __future__ import annotations

import torch

from . import _lib

_BF16, _F32, _I32, _I64 = torch.bfloat16, torch.float32, torch.int32, torch.int64
_CODE = {_BF16: _lib.DTYPE_BF16, _F32: _lib.DTYPE_F32}


def _code(t, name: str) -> int:
    code = _CODE.get(t.dtype)
    if code is None:
        raise ValueError(f"{name} must be bfloat16 or float32")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    return code


def _rows(t):
    """t as (tensor, rows, width, row stride): any leading dimensions, the last one contiguous
    and rows at one stride that is no less than the width (anything else is copied)."""
    if t.dim() != 2:
        if t.dim() < 1:
            raise ValueError("a tensor with rows is needed, not a scalar")
        t = t.reshape(t.shape[:-1].numel(), t.shape[-1])
    rows, d = t.shape
    ld, along = t.stride()
    if (d > 1 and along != 1) or (rows > 1 and ld < d):
        return t.contiguous(), rows, d, d
    return t, rows, d, ld if ld > d else d


def _vector(t, index: int, name: str, n: int, dtype):
    """A companion vector of n entries on device `index`, contiguous."""
    if t.dtype is not dtype or t.get_device() != index or t.shape != (n,):
        raise ValueError(f"{name} must be a {dtype} vector of {n} entries on cuda:{index}, not a {t.dtype} "
                         f"tensor of shape {tuple(t.shape)} on {t.device}")
    return t if t.is_contiguous() else t.contiguous()


def _empty_like(t):
    """A contiguous tensor of t's shape and type (for a contiguous t the cheaper call)."""
    return torch.empty_like(t) if t.is_contiguous() else torch.empty_like(t, memory_format=torch.contiguous_format)


def _ptr(t):
    return None if t is None else t.data_ptr()


_current_stream, _current_device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice


def _call(fn: str, index: int, *args) -> None:
    """An operator's entry point on device `index`, its current stream the last argument."""
    f = getattr(_lib._lib or _lib.lib(), fn)
    if index == _current_device():
        st = f(*args, _current_stream(index))
    else:
        with torch.cuda.device(index):
            st = f(*args, _current_stream(index))
    if st != _lib.TM_OK:
        raise _lib.TurboMuonError(fn, st, _lib.last_error())


def _on(stream, like, op, *args):
    """op(*args) with `stream`, one of like's device, current: the copies and the results of the
    call belong to that stream as the kernels do."""
    if stream.device != like.device:
        raise ValueError(f"the stream is one of {stream.device}, the tensors are on {like.device}")
    with torch.cuda.stream(stream):
        return op(*args)


def layer_norm(x, weight=None, bias=None, eps: float = 1e-5, stream=None):
    """Layer norm over the last dimension of x (bf16 or fp32, any strides between rows).

    weight and bias are fp32 vectors or None.  Returns (y, mean, rstd): y of x's shape and
    type, mean and rstd fp32, one per row.
    """
    if stream is not None:
        return _on(stream, x, layer_norm, x, weight, bias, eps)
    code, index = _code(x, "x"), x.get_device()
    x2, rows, d, ld = _rows(x)
    if weight is not None:
        weight = _vector(weight, index, "weight", d, _F32)
    if bias is not None:
        bias = _vector(bias, index, "bias", d, _F32)
    y = _empty_like(x)
    mean = x.new_empty_strided((rows,), (1,), dtype=_F32)
    rstd = torch.empty_like(mean)
    _call("tm_layer_norm", index, x2.data_ptr(), ld, _ptr(weight), _ptr(bias), y.data_ptr(), d,
          mean.data_ptr(), rstd.data_ptr(), rows, d, eps, code)
    return y, mean, rstd


def layer_norm_backward(dy, x, mean, rstd, weight=None, param_grads: bool = True, stream=None):
    """Gradients of layer_norm: (dx, dweight, dbias), the last two fp32, or None without
    param_grads.  mean and rstd are layer_norm's; dy has x's shape and type."""
    if stream is not None:
        return _on(stream, x, layer_norm_backward, dy, x, mean, rstd, weight, param_grads)
    code, index = _code(x, "x"), x.get_device()
    if dy.shape != x.shape or dy.dtype is not x.dtype or dy.get_device() != index:
        raise ValueError("dy must have x's shape, type and device")
    x2, rows, d, ldx = _rows(x)
    dy2, _, _, lddy = _rows(dy)
    mean, rstd = _vector(mean, index, "mean", rows, _F32), _vector(rstd, index, "rstd", rows, _F32)
    if weight is not None:
        weight = _vector(weight, index, "weight", d, _F32)
    dx = _empty_like(x)
    dweight = dbias = None
    if param_grads:
        dweight = x.new_empty_strided((d,), (1,), dtype=_F32)
        dbias = torch.empty_like(dweight)
    _call("tm_layer_norm_backward", index, dy2.data_ptr(), lddy, x2.data_ptr(), ldx, _ptr(weight),
          mean.data_ptr(), rstd.data_ptr(), dx.data_ptr(), d, _ptr(dweight), _ptr(dbias), rows, d, code)
    return dx, dweight, dbias


def _matrices(w, x, index: int):
    """Stacked matrices as (tensor, row stride, matrix stride), their last dimension contiguous."""
    if w.dim() != 3:
        raise ValueError("w must be (experts, rows, columns)")
    if w.get_device() != index or w.dtype is not x.dtype:
        raise ValueError("w must have x's type and device")
    e, r, c = w.shape
    apart, ld, along = w.stride()
    if (c > 1 and along != 1) or (r > 1 and ld < c) or (e > 1 and apart < (r - 1) * max(ld, c) + c):
        return w.contiguous(), c, r * c
    return w, ld if ld > c else c, apart if e > 1 else 0


def _ends(ends, index: int):
    if ends.dim() != 1 or ends.dtype is not _I32 or ends.get_device() != index:
        raise ValueError("ends must be an int32 vector on x's device")
    return ends if ends.is_contiguous() else ends.contiguous()


def expert_matmul(x, w, ends, transposed: bool = False, stream=None):
    """y[i] = x[i] @ w[e] for the rows of each expert e (w[e].T with transposed).

    x is (rows, k), bf16 or fp32, rows sorted by expert; w is (experts, k, n), or (experts, n, k)
    with transposed; ends is an int32 device vector, ends[e] the number of rows up to expert e's
    last.  Rows after ends[-1] come out as zeros.  Nothing is synchronised.
    """
    if stream is not None:
        return _on(stream, x, expert_matmul, x, w, ends, transposed)
    code, index = _code(x, "x"), x.get_device()
    if x.dim() != 2:
        raise ValueError("x must be (rows, k)")
    x2, rows, k, ldx = _rows(x)
    w, ldw, stride_w = _matrices(w, x, index)
    experts, kw, n = w.shape
    if transposed:
        kw, n = n, kw
    if kw != k:
        raise ValueError(f"w's matrices of {tuple(w.shape[1:])} do not fit rows of {k}")
    ends = _ends(ends, index)
    if ends.shape[0] != experts:
        raise ValueError("ends must hold one entry per expert")
    y = x.new_empty_strided((rows, n), (n, 1))
    _call("tm_expert_matmul", index, x2.data_ptr(), ldx, w.data_ptr(), ldw, stride_w, ends.data_ptr(),
          y.data_ptr(), n, rows, experts, k, n, 1 if transposed else 0, code)
    return y


def expert_wgrad(x, dy, ends, dtype=None, stream=None):
    """dw[e] = x_e.T @ dy_e for the rows of each expert: (experts, k, n), fp32 unless dtype says
    bf16 (for bf16 rows).  Experts without rows get zeros."""
    if stream is not None:
        return _on(stream, x, expert_wgrad, x, dy, ends, dtype)
    code, index = _code(x, "x"), x.get_device()
    if x.dim() != 2 or dy.dim() != 2 or dy.shape[0] != x.shape[0]:
        raise ValueError("x and dy must be (rows, k) and (rows, n)")
    if dy.dtype is not x.dtype or dy.get_device() != index:
        raise ValueError("dy must have x's type and device")
    x2, rows, k, ldx = _rows(x)
    dy2, _, n, lddy = _rows(dy)
    ends = _ends(ends, index)
    experts = ends.shape[0]
    dw = x.new_empty_strided((experts, k, n), (k * n, n, 1), dtype=dtype or _F32)
    _call("tm_expert_wgrad", index, x2.data_ptr(), ldx, dy2.data_ptr(), lddy, ends.data_ptr(),
          dw.data_ptr(), n, k * n if experts > 1 else 0, rows, experts, k, n, code, _code(dw, "dtype"))
    return dw


def _policy_loss(logits, targets, old_logp, advantages, weights, ref_logp, clip_low, clip_high, kl, temperature,
                 stream, grad: bool, keep: bool):
    if stream is not None:
        return _on(stream, logits, _policy_loss, logits, targets, old_logp, advantages, weights, ref_logp, clip_low,
                   clip_high, kl, temperature, None, grad, keep)
    code, index = _code(logits, "logits"), logits.get_device()
    if logits.dim() != 2:
        raise ValueError("logits must be (rows, vocabulary)")
    l2, rows, vocab, ld = _rows(logits)
    targets = _vector(targets, index, "targets", rows, _I64)
    old_logp = _vector(old_logp, index, "old_logp", rows, _F32)
    advantages = _vector(advantages, index, "advantages", rows, _F32)
    weights = _vector(weights, index, "weights", rows, _F32)
    if ref_logp is not None:
        ref_logp = _vector(ref_logp, index, "ref_logp", rows, _F32)
    loss = logits.new_empty_strided((), (), dtype=_F32)
    logp = torch.empty_like(weights)
    lse = slope = dlogits = None
    if grad:
        dlogits = _empty_like(logits)
    if keep:
        lse, slope = torch.empty_like(weights), torch.empty_like(weights)
    _call("tm_policy_loss", index, l2.data_ptr(), ld, targets.data_ptr(), old_logp.data_ptr(),
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
    if stream is not None:
        return _on(stream, logits, policy_loss_backward, logits, targets, lse, slope, grad, temperature)
    code, index = _code(logits, "logits"), logits.get_device()
    if logits.dim() != 2:
        raise ValueError("logits must be (rows, vocabulary)")
    l2, rows, vocab, ld = _rows(logits)
    targets = _vector(targets, index, "targets", rows, _I64)
    lse = _vector(lse, index, "lse", rows, _F32)
    slope = _vector(slope, index, "slope", rows, _F32)
    if grad is not None and (grad.dim() != 0 or grad.dtype is not _F32 or grad.get_device() != index):
        raise ValueError("grad must be an fp32 scalar on the logits' device")
    dlogits = _empty_like(logits)
    _call("tm_policy_loss_backward", index, l2.data_ptr(), ld, targets.data_ptr(),
          lse.data_ptr(), slope.data_ptr(), _ptr(grad), temperature, dlogits.data_ptr(), vocab, rows, vocab, code)
    return dlogits
