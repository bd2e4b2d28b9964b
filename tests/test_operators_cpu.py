"""The operators' entry points without a GPU: what they refuse before the HIP runtime is touched."""
import ctypes

import pytest

from paper_2512_04632_amd import _lib as tm

P = 0x1000   # never dereferenced: every call here is refused, or has nothing to do


def _norm(x=P, ldx=8, w=P, b=P, y=P, ldy=8, mean=P, rstd=P, rows=4, d=8, eps=1e-5, dtype=1):
    return tm.lib().tm_layer_norm(x, ldx, w, b, y, ldy, mean, rstd, rows, d, eps, dtype, None)


def _norm_back(dy=P, lddy=8, x=P, ldx=8, w=P, mean=P, rstd=P, dx=P, lddx=8, dw=P, db=P, rows=4, d=8, dtype=1):
    return tm.lib().tm_layer_norm_backward(dy, lddy, x, ldx, w, mean, rstd, dx, lddx, dw, db, rows, d, dtype, None)


def _matmul(x=P, ldx=8, w=P, ldw=16, sw=128, ends=P, y=P, ldy=16, rows=4, experts=2, k=8, n=16, t=0, dtype=0):
    return tm.lib().tm_expert_matmul(x, ldx, w, ldw, sw, ends, y, ldy, rows, experts, k, n, t, dtype, None)


def _wgrad(x=P, ldx=8, dy=P, lddy=16, ends=P, dw=P, lddw=16, sdw=128, rows=4, experts=2, k=8, n=16, dtype=0, out=1):
    return tm.lib().tm_expert_wgrad(x, ldx, dy, lddy, ends, dw, lddw, sdw, rows, experts, k, n, dtype, out, None)


def _loss(logits=P, ld=64, targets=P, old=P, adv=P, weights=P, ref=None, low=0.2, high=0.2, kl=0.0, temp=1.0, loss=P,
          logp=P, lse=None, slope=None, dlogits=None, ldd=64, rows=4, vocab=64, dtype=0):
    return tm.lib().tm_policy_loss(logits, ld, targets, old, adv, weights, ref, low, high, kl, temp, loss, logp, lse,
                                   slope, dlogits, ldd, rows, vocab, dtype, None)


def _loss_back(logits=P, ld=64, targets=P, lse=P, slope=P, grad=None, temp=1.0, dlogits=P, ldd=64, rows=4, vocab=64,
               dtype=0):
    return tm.lib().tm_policy_loss_backward(logits, ld, targets, lse, slope, grad, temp, dlogits, ldd, rows, vocab,
                                            dtype, None)


INVALID, UNSUPPORTED = tm.TM_ERR_INVALID_ARG, tm.TM_ERR_UNSUPPORTED
BIG = 1 << 32


@pytest.mark.parametrize("call,bad,code", [
    (_norm, dict(rows=-1), INVALID), (_norm, dict(rows=BIG), INVALID), (_norm, dict(d=0), INVALID),
    (_norm, dict(d=65537), INVALID), (_norm, dict(dtype=2), INVALID), (_norm, dict(eps=-1.0), INVALID),
    (_norm, dict(eps=float("nan")), INVALID), (_norm, dict(ldx=7), INVALID), (_norm, dict(ldy=7), INVALID),
    (_norm, dict(ldx=1 << 41), INVALID), (_norm, dict(x=None), INVALID), (_norm, dict(mean=None), INVALID),
    (_norm, dict(x=0x1002), UNSUPPORTED), (_norm, dict(w=0x1002), UNSUPPORTED),
    (_norm_back, dict(dy=None), INVALID), (_norm_back, dict(dx=None), INVALID), (_norm_back, dict(rstd=None), INVALID),
    (_norm_back, dict(lddx=7), INVALID), (_norm_back, dict(dw=0x1001), UNSUPPORTED), (_norm_back, dict(d=0), INVALID),
    (_matmul, dict(experts=0), INVALID), (_matmul, dict(experts=8193), INVALID), (_matmul, dict(k=0), INVALID),
    (_matmul, dict(n=65537), INVALID), (_matmul, dict(ldw=15), INVALID), (_matmul, dict(sw=127), INVALID),
    (_matmul, dict(sw=-1, experts=1), INVALID), (_matmul, dict(ends=None), INVALID),
    (_matmul, dict(ends=0x1002), UNSUPPORTED), (_matmul, dict(x=0x1001), UNSUPPORTED),
    (_matmul, dict(t=1, ldw=7), INVALID), (_matmul, dict(dtype=-1), INVALID), (_matmul, dict(ldy=15), INVALID),
    (_wgrad, dict(dtype=1, out=0), UNSUPPORTED), (_wgrad, dict(out=3), INVALID), (_wgrad, dict(lddw=15), INVALID),
    (_wgrad, dict(sdw=100), INVALID), (_wgrad, dict(dw=None), INVALID), (_wgrad, dict(dw=0x1002), UNSUPPORTED),
    (_wgrad, dict(rows=0, ends=None), INVALID),
    (_loss, dict(vocab=0), INVALID), (_loss, dict(vocab=(1 << 30) + 1), INVALID), (_loss, dict(ld=63), INVALID),
    (_loss, dict(temp=0.0), INVALID), (_loss, dict(temp=-1.0), INVALID), (_loss, dict(temp=1e-39), INVALID),
    (_loss, dict(low=1.1), INVALID), (_loss, dict(high=-0.1), INVALID), (_loss, dict(kl=-0.1), INVALID),
    (_loss, dict(loss=None), INVALID), (_loss, dict(targets=0x1004), UNSUPPORTED),
    (_loss, dict(dlogits=P, ldd=63), INVALID), (_loss, dict(rows=0, loss=None), INVALID),
    (_loss_back, dict(dlogits=None), INVALID), (_loss_back, dict(lse=None), INVALID),
    (_loss_back, dict(temp=float("nan")), INVALID), (_loss_back, dict(grad=0x1002), UNSUPPORTED),
    (_loss_back, dict(rows=1 << 30, vocab=1 << 20, ld=1 << 20, ldd=1 << 20), UNSUPPORTED),
])
def test_refused(call, bad, code):
    assert call(**bad) == code
    assert tm.last_error() != ""


def test_nothing_to_do():
    assert _norm(rows=0, x=None, y=None, mean=None, rstd=None) == tm.TM_OK
    assert _norm_back(rows=0, dw=None, db=None) == tm.TM_OK
    assert _matmul(rows=0, x=None, y=None) == tm.TM_OK
    assert _loss_back(rows=0) == tm.TM_OK


def test_python_checks_come_before_the_library():
    torch = pytest.importorskip("torch")
    x = torch.zeros((2, 4))
    ends = torch.tensor([2], dtype=torch.int32)
    for call in (lambda: tm.layer_norm(x), lambda: tm.layer_norm(x.double()),
                 lambda: tm.expert_matmul(x, torch.zeros((1, 4, 4)), ends),
                 lambda: tm.expert_wgrad(x, x, ends), lambda: tm.policy_loss(x, ends, x[0], x[0], x[0])):
        with pytest.raises(ValueError):
            call()


def test_dtype_codes_match_the_header():
    import os
    import re
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = open(os.path.join(root, "include", "turbomuon.h")).read()
    d = {k: int(v) for k, v in re.findall(r"#define\s+(TM_DTYPE_\w+)\s+(\d+)", text)}
    assert d == {"TM_DTYPE_BF16": tm.DTYPE_BF16, "TM_DTYPE_F32": tm.DTYPE_F32}
    assert ctypes.sizeof(ctypes.c_void_p) == 8


@pytest.mark.parametrize("call,size", [
    (_loss, dict(rows=1 << 26, vocab=2000, ld=2000)), (_loss, dict(rows=1 << 24, vocab=8000, ld=8000)),
    (_loss, dict(rows=1 << 22, vocab=100000, ld=100000)), (_loss_back, dict(rows=1 << 24, vocab=64)),
])
def test_launches_past_32_bits_of_threads_are_refused(call, size):
    """A dispatch counts its threads in 32 bits: more would wrap."""
    assert call(**size) == UNSUPPORTED
    assert "too many blocks" in tm.last_error()


@pytest.mark.parametrize("rows", [(1 << 26) - 3, (1 << 26) - 2, (1 << 26) - 1])
@pytest.mark.parametrize("vocab,dtype", [(2, 0), (2048, 0), (2, 1), (1024, 1)])
def test_four_rows_a_workgroup_count_as_one_that_is_full(rows, vocab, dtype):
    """Short rows go four to a workgroup of 256: 2^24 workgroups are one thread too many for a launch."""
    assert _loss(rows=rows, vocab=vocab, ld=vocab, ldd=vocab, dtype=dtype) == UNSUPPORTED
    assert "too many blocks" in tm.last_error()
