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

_BF16, _F32, _I32, _I64, _BOOL = torch.bfloat16, torch.float32, torch.int32, torch.int64, torch.bool
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


def _like(t, like, name: str):
    """t checked to be of like's shape, type and device."""
    if t.shape != like.shape or t.dtype is not like.dtype or t.get_device() != like.get_device():
        raise ValueError(f"{name} must have the shape {tuple(like.shape)}, the type {like.dtype} and the device of "
                         f"what it goes with, not {tuple(t.shape)}, {t.dtype}, {t.device}")
    return t


def rms_norm(x, weight=None, residual=None, eps: float = 1e-5, stream=None):
    """Root-mean-square norm over the last dimension of s = x + residual (bf16 or fp32).

    weight is an fp32 vector or None; residual has x's shape and type, or is None.  Returns
    (y, s, rstd): y and s of x's shape and type (s is x itself without a residual, else rounded
    to the type before it is normalised), rstd fp32, one per row.
    """
    if stream is not None:
        return _on(stream, x, rms_norm, x, weight, residual, eps)
    code, index = _code(x, "x"), x.get_device()
    x2, rows, d, ld = _rows(x)
    if weight is not None:
        weight = _vector(weight, index, "weight", d, _F32)
    s, ldr, r2 = x, d, None
    if residual is not None:
        r2, _, _, ldr = _rows(_like(residual, x, "residual"))
        s = _empty_like(x)
    y = _empty_like(x)
    rstd = x.new_empty_strided((rows,), (1,), dtype=_F32)
    _call("tm_rms_norm", index, x2.data_ptr(), ld, _ptr(r2), ldr, _ptr(weight), None if r2 is None else s.data_ptr(), d,
          y.data_ptr(), d, rstd.data_ptr(), rows, d, eps, code)
    return y, s, rstd


def rms_norm_backward(dy, s, rstd, weight=None, dsum=None, param_grads: bool = True, stream=None):
    """Gradients of rms_norm: (ds, dweight).  s and rstd are rms_norm's; dy and dsum (the gradient that
    reaches s by another way, or None) have s's shape and type.  ds is the gradient of x and of the
    residual; dweight is fp32, or None without param_grads."""
    if stream is not None:
        return _on(stream, s, rms_norm_backward, dy, s, rstd, weight, dsum, param_grads)
    code, index = _code(s, "s"), s.get_device()
    s2, rows, d, lds = _rows(s)
    dy2, _, _, lddy = _rows(_like(dy, s, "dy"))
    a2, lda = None, d
    if dsum is not None:
        a2, _, _, lda = _rows(_like(dsum, s, "dsum"))
    rstd = _vector(rstd, index, "rstd", rows, _F32)
    if weight is not None:
        weight = _vector(weight, index, "weight", d, _F32)
    ds = _empty_like(s)
    dweight = s.new_empty_strided((d,), (1,), dtype=_F32) if param_grads else None
    _call("tm_rms_norm_backward", index, dy2.data_ptr(), lddy, s2.data_ptr(), lds, _ptr(weight), rstd.data_ptr(),
          _ptr(a2), lda, ds.data_ptr(), d, _ptr(dweight), rows, d, code)
    return ds, dweight


def _table(t, index: int, name: str, rows, top, dtype):
    """A companion of `top` entries per row on device `index`, contiguous."""
    if t.dim() != 2 or t.dtype is not dtype or t.get_device() != index or t.shape[0] != rows or \
            (top is not None and t.shape[1] != top):
        raise ValueError(f"{name} must be a {dtype} matrix of {rows} rows of {'the choices' if top is None else top} on "
                         f"cuda:{index}, not a {t.dtype} tensor of shape {tuple(t.shape)} on {t.device}")
    return t if t.is_contiguous() else t.contiguous()


def expert_route(logits, top: int, active=None, renormalize: bool = True, scale: float = 1.0, stream=None):
    """The `top` experts of each row of (rows, experts) scores, bf16 or fp32.

    Returns (chosen, weights, slots, ends, balance): the experts (int32, most likely first, of equal
    scores the lowest), their weights (fp32: scale times the softmax, over the sum of the chosen ones
    with renormalize), where each choice stands among the rows sorted by expert (int32), the int32
    ends that expert_matmul takes, and the balance loss (an fp32 scalar, 1 where all experts are
    used alike).  Rows where the bool vector `active` is False take no part: their choices and slots
    are -1, their weights 0.
    """
    if stream is not None:
        return _on(stream, logits, expert_route, logits, top, active, renormalize, scale)
    code, index = _code(logits, "logits"), logits.get_device()
    if logits.dim() != 2:
        raise ValueError("logits must be (rows, experts)")
    l2, rows, experts, ld = _rows(logits)
    if active is not None:
        active = _vector(active, index, "active", rows, _BOOL)
    held = min(max(top, 0), _lib.TM_MAX_TOP)   # any other is refused below
    chosen = logits.new_empty_strided((rows, held), (held, 1), dtype=_I32)
    slots = torch.empty_like(chosen)
    weights = logits.new_empty_strided(chosen.shape, chosen.stride(), dtype=_F32)
    ends = logits.new_empty_strided((experts,), (1,), dtype=_I32)
    balance = logits.new_empty_strided((), (), dtype=_F32)
    _call("tm_expert_route", index, l2.data_ptr(), ld, _ptr(active), 1 if renormalize else 0, scale, chosen.data_ptr(),
          weights.data_ptr(), slots.data_ptr(), ends.data_ptr(), balance.data_ptr(), rows, experts, top, code)
    return chosen, weights, slots, ends, balance


def expert_route_backward(logits, chosen, ends, dweights=None, dbalance=None, renormalize: bool = True,
                          scale: float = 1.0, stream=None):
    """Gradient by the logits from those of expert_route's weights (fp32, of chosen's shape, or None)
    and of its balance loss (an fp32 scalar on the device, or None).  chosen and ends are expert_route's."""
    if stream is not None:
        return _on(stream, logits, expert_route_backward, logits, chosen, ends, dweights, dbalance, renormalize, scale)
    code, index = _code(logits, "logits"), logits.get_device()
    if logits.dim() != 2:
        raise ValueError("logits must be (rows, experts)")
    l2, rows, experts, ld = _rows(logits)
    chosen = _table(chosen, index, "chosen", rows, None, _I32)
    ends = _vector(ends, index, "ends", experts, _I32)
    if dweights is not None:
        dweights = _table(dweights, index, "dweights", rows, chosen.shape[1], _F32)
    if dbalance is not None and (dbalance.dim() != 0 or dbalance.dtype is not _F32 or dbalance.get_device() != index):
        raise ValueError("dbalance must be an fp32 scalar on the logits' device")
    dlogits = _empty_like(logits)
    _call("tm_expert_route_backward", index, l2.data_ptr(), ld, chosen.data_ptr(), ends.data_ptr(), _ptr(dweights),
          _ptr(dbalance), 1 if renormalize else 0, scale, dlogits.data_ptr(), experts, rows, experts, chosen.shape[1],
          code)
    return dlogits


def _filled(ends, index: int):
    """ends checked, or None; the address of its last entry, how many rows are filled."""
    if ends is None:
        return None, None
    ends = _ends(ends, index)
    if ends.shape[0] < 1:
        raise ValueError("ends must hold one entry per expert")
    return ends, ends.data_ptr() + 4 * (ends.shape[0] - 1)


def _matrix(t, name: str):
    if t.dim() != 2:
        raise ValueError(f"{name} must be a matrix of rows")
    return _rows(t)


def _by_slot(like, count: int, d: int, ends):
    """A matrix of `count` rows that go to their slots.  Which of them have one is known on the device alone: with `ends`
    the library writes every row, those that it finds filled and zeros behind them; without, those that no slot names
    would be what the memory held before, so they are zeros to begin with."""
    return like.new_zeros((count, d)) if ends is None else like.new_empty_strided((count, d), (d, 1))


def expert_gather(x, slots, ends=None, stream=None):
    """The rows of x (rows, d) in the experts' order: out[slots[i, j]] = x[i], of rows times top rows.

    slots and ends are expert_route's: every row below ends[-1] has its slot, slots that are negative,
    or not below ends[-1], are none, and the rows from ends[-1] on come out as zeros.  For other slots
    (choices taken out, gaps) leave `ends` out: rows that no slot names are zeros then, which
    takes another pass over the result.
    """
    if stream is not None:
        return _on(stream, x, expert_gather, x, slots, ends)
    code, index = _code(x, "x"), x.get_device()
    x2, rows, d, ldx = _matrix(x, "x")
    slots = _table(slots, index, "slots", rows, None, _I32)
    ends, used = _filled(ends, index)
    top = slots.shape[1]
    out = _by_slot(x, rows * top, d, ends)
    _call("tm_expert_gather", index, x2.data_ptr(), ldx, slots.data_ptr(), used, out.data_ptr(), d, rows * top, rows,
          top, d, code)
    return out


def expert_combine(y, slots, weights=None, residual=None, ends=None, stream=None):
    """out[i] = residual[i] + sum over j of weights[i, j] y[slots[i, j]], summed in fp32.

    y is (count, d), bf16 or fp32; slots int32 and weights fp32 (None: ones) are (rows, top);
    residual is (rows, d) of y's type, or None.  Slots that are negative, or not
    below ends[-1] (ends None: past y), are left out.
    """
    if stream is not None:
        return _on(stream, y, expert_combine, y, slots, weights, residual, ends)
    code, index = _code(y, "y"), y.get_device()
    y2, count, d, ldy = _matrix(y, "y")
    if slots.dim() != 2:
        raise ValueError("slots must be (rows, top)")
    rows, top = slots.shape
    slots = _table(slots, index, "slots", rows, top, _I32)
    if weights is not None:
        weights = _table(weights, index, "weights", rows, top, _F32)
    r2, ldr = None, d
    if residual is not None:
        if residual.shape != (rows, d) or residual.dtype is not y.dtype or residual.get_device() != index:
            raise ValueError(f"residual must be ({rows}, {d}) of y's type and device")
        r2, _, _, ldr = _rows(residual)
    ends, used = _filled(ends, index)
    out = y.new_empty_strided((rows, d), (d, 1))
    _call("tm_expert_combine", index, y2.data_ptr(), ldy, slots.data_ptr(), used, _ptr(weights), _ptr(r2), ldr,
          out.data_ptr(), d, count, rows, top, d, code)
    return out


def expert_combine_backward(dout, y, slots, ends=None, weights=None, weight_grads: bool = True, stream=None):
    """Gradients of expert_combine by y and the weights: (dy, dweights), the second None without
    weight_grads.  dout is (rows, d) of y's type; ends as for expert_gather: with it every row of y below
    ends[-1] has to be in a slot, without it rows in no slot have a gradient of zero.  (The residual's is dout.)"""
    if stream is not None:
        return _on(stream, y, expert_combine_backward, dout, y, slots, ends, weights, weight_grads)
    code, index = _code(y, "y"), y.get_device()
    y2, count, d, ldy = _matrix(y, "y")
    g2, rows, dg, ldg = _matrix(dout, "dout")
    if dg != d or dout.dtype is not y.dtype or dout.get_device() != index:
        raise ValueError("dout must have y's width, type and device")
    slots = _table(slots, index, "slots", rows, None, _I32)
    top = slots.shape[1]
    if weights is not None:
        weights = _table(weights, index, "weights", rows, top, _F32)
    ends, used = _filled(ends, index)
    dy = _by_slot(y, count, d, ends)
    dweights = y.new_empty_strided((rows, top), (top, 1), dtype=_F32) if weight_grads else None
    _call("tm_expert_combine_backward", index, g2.data_ptr(), ldg, y2.data_ptr(), ldy, slots.data_ptr(),
          used, _ptr(weights), dy.data_ptr(), d, _ptr(dweights), count, rows, top, d, code)
    return dy, dweights


def token_logp(logits, targets, top: int = 0, temperature: float = 1.0, stream=None):
    """Log probabilities of int64 targets under (rows, vocabulary) logits, bf16 or fp32, at the temperature.

    Returns (logp, entropy, stats, top_logp, top_ids): per row the target's log probability, the
    entropy, the largest logit with the sum of exponentials about it (what token_logp_backward takes),
    and the `top` most likely tokens, fp32 log probabilities and int64 places, of equal logits the
    lowest (None with top 0).  Rows with a negative target take no part: zeros, places of -1.
    """
    if stream is not None:
        return _on(stream, logits, token_logp, logits, targets, top, temperature)
    code, index = _code(logits, "logits"), logits.get_device()
    if logits.dim() != 2:
        raise ValueError("logits must be (rows, vocabulary)")
    l2, rows, vocab, ld = _rows(logits)
    targets = _vector(targets, index, "targets", rows, _I64)
    logp = logits.new_empty_strided((rows,), (1,), dtype=_F32)
    entropy = torch.empty_like(logp)
    stats = logits.new_empty_strided((rows, 2), (2, 1), dtype=_F32)
    top_logp = top_ids = None
    if top > 0:
        held = min(top, _lib.TM_MAX_TOP)   # more are refused below
        top_logp = logits.new_empty_strided((rows, held), (held, 1), dtype=_F32)
        top_ids = targets.new_empty_strided((rows, held), (held, 1))
    _call("tm_token_logp", index, l2.data_ptr(), ld, targets.data_ptr(), temperature, logp.data_ptr(),
          entropy.data_ptr(), stats.data_ptr(), top, _ptr(top_logp), _ptr(top_ids), rows, vocab, code)
    return logp, entropy, stats, top_logp, top_ids


def token_logp_backward(logits, targets, stats, entropy, dlogp=None, dentropy=None, temperature: float = 1.0,
                        stream=None):
    """Gradient by the logits from those of token_logp's logp and entropy (fp32 per row, None: zeros);
    stats and entropy are token_logp's."""
    if stream is not None:
        return _on(stream, logits, token_logp_backward, logits, targets, stats, entropy, dlogp, dentropy, temperature)
    code, index = _code(logits, "logits"), logits.get_device()
    if logits.dim() != 2:
        raise ValueError("logits must be (rows, vocabulary)")
    l2, rows, vocab, ld = _rows(logits)
    targets = _vector(targets, index, "targets", rows, _I64)
    stats = _table(stats, index, "stats", rows, 2, _F32)
    entropy = _vector(entropy, index, "entropy", rows, _F32)
    if dlogp is not None:
        dlogp = _vector(dlogp, index, "dlogp", rows, _F32)
    if dentropy is not None:
        dentropy = _vector(dentropy, index, "dentropy", rows, _F32)
    dlogits = _empty_like(logits)
    _call("tm_token_logp_backward", index, l2.data_ptr(), ld, targets.data_ptr(), stats.data_ptr(), entropy.data_ptr(),
          _ptr(dlogp), _ptr(dentropy), temperature, dlogits.data_ptr(), vocab, rows, vocab, code)
    return dlogits
