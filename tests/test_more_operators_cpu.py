"""The norm, routing, row and log probability entry points without a GPU: what they refuse before the HIP runtime is touched."""
import os
import re

import pytest

from paper_2512_04632_amd import _lib as tm

P = 0x1000   # never dereferenced: every call here is refused, or has nothing to do
Q = 0x2000


def _rms(x=P, ldx=8, r=P, ldr=8, w=P, s=Q, lds=8, y=P, ldy=8, rstd=P, rows=4, d=8, eps=1e-5, dtype=1):
    return tm.lib().tm_rms_norm(x, ldx, r, ldr, w, s, lds, y, ldy, rstd, rows, d, eps, dtype, None)


def _rms_back(dy=P, lddy=8, s=P, lds=8, w=P, rstd=P, dsum=P, lddsum=8, ds=P, ldds=8, dw=P, rows=4, d=8, dtype=1):
    return tm.lib().tm_rms_norm_backward(dy, lddy, s, lds, w, rstd, dsum, lddsum, ds, ldds, dw, rows, d, dtype, None)


def _route(logits=P, ld=8, active=None, renorm=1, scale=1.0, chosen=P, weights=P, slots=P, ends=P, balance=P, rows=4,
           experts=8, top=2, dtype=1):
    return tm.lib().tm_expert_route(logits, ld, active, renorm, scale, chosen, weights, slots, ends, balance, rows, experts,
                                    top, dtype, None)


def _route_back(logits=P, ld=8, chosen=P, ends=P, dw=P, db=P, renorm=1, scale=1.0, dl=P, ldd=8, rows=4, experts=8, top=2,
                dtype=1):
    return tm.lib().tm_expert_route_backward(logits, ld, chosen, ends, dw, db, renorm, scale, dl, ldd, rows, experts, top,
                                             dtype, None)


def _gather(x=P, ldx=8, slots=P, used=P, out=P, ldo=8, count=8, rows=4, top=2, d=8, dtype=1):
    return tm.lib().tm_expert_gather(x, ldx, slots, used, out, ldo, count, rows, top, d, dtype, None)


def _combine(y=P, ldy=8, slots=P, used=P, w=P, r=P, ldr=8, out=P, ldo=8, count=8, rows=4, top=2, d=8, dtype=1):
    return tm.lib().tm_expert_combine(y, ldy, slots, used, w, r, ldr, out, ldo, count, rows, top, d, dtype, None)


def _combine_back(g=P, ldg=8, y=P, ldy=8, slots=P, used=P, w=P, dy=P, lddy=8, dw=P, count=8, rows=4, top=2, d=8, dtype=1):
    return tm.lib().tm_expert_combine_backward(g, ldg, y, ldy, slots, used, w, dy, lddy, dw, count, rows, top, d, dtype, None)


def _logp(logits=P, ld=64, targets=P, temp=1.0, logp=P, entropy=P, stats=P, top=2, tl=P, ti=P, rows=4, vocab=64, dtype=1):
    return tm.lib().tm_token_logp(logits, ld, targets, temp, logp, entropy, stats, top, tl, ti, rows, vocab, dtype, None)


def _logp_back(logits=P, ld=64, targets=P, stats=P, entropy=P, g=P, h=P, temp=1.0, dl=P, ldd=64, rows=4, vocab=64, dtype=1):
    return tm.lib().tm_token_logp_backward(logits, ld, targets, stats, entropy, g, h, temp, dl, ldd, rows, vocab, dtype, None)


INVALID, UNSUPPORTED = tm.TM_ERR_INVALID_ARG, tm.TM_ERR_UNSUPPORTED
BIG = 1 << 32
NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("call,bad,code", [
    (_rms, dict(rows=-1), INVALID), (_rms, dict(rows=BIG), INVALID), (_rms, dict(d=0), INVALID), (_rms, dict(d=65537), INVALID),
    (_rms, dict(dtype=2), INVALID), (_rms, dict(eps=-1.0), INVALID), (_rms, dict(eps=NAN), INVALID), (_rms, dict(ldx=7), INVALID),
    (_rms, dict(ldr=7), INVALID), (_rms, dict(lds=7), INVALID), (_rms, dict(ldy=7), INVALID), (_rms, dict(ldx=1 << 41), INVALID),
    (_rms, dict(x=None), INVALID), (_rms, dict(s=None), INVALID), (_rms, dict(s=P), INVALID), (_rms, dict(rstd=None), INVALID),
    (_rms, dict(x=0x1002), UNSUPPORTED), (_rms, dict(r=0x1002), UNSUPPORTED), (_rms, dict(w=0x1001), UNSUPPORTED),
    (_rms_back, dict(dy=None), INVALID), (_rms_back, dict(s=None), INVALID), (_rms_back, dict(ds=None), INVALID),
    (_rms_back, dict(rstd=None), INVALID), (_rms_back, dict(lddsum=7), INVALID), (_rms_back, dict(ldds=7), INVALID),
    (_rms_back, dict(dw=0x1002), UNSUPPORTED), (_rms_back, dict(d=0), INVALID), (_rms_back, dict(dtype=-1), INVALID),
    (_route, dict(rows=-1), INVALID), (_route, dict(experts=0), INVALID), (_route, dict(experts=8193, ld=8193), INVALID),
    (_route, dict(top=0), INVALID), (_route, dict(top=9), INVALID), (_route, dict(experts=100, ld=100, top=65), INVALID),
    (_route, dict(rows=1 << 30, top=2), INVALID), (_route, dict(scale=NAN), INVALID), (_route, dict(scale=INF), INVALID),
    (_route, dict(ld=7), INVALID), (_route, dict(logits=None), INVALID), (_route, dict(chosen=None), INVALID),
    (_route, dict(slots=0x1002), UNSUPPORTED), (_route, dict(ends=None), INVALID), (_route, dict(balance=None), INVALID),
    (_route, dict(rows=0, ends=None), INVALID), (_route, dict(dtype=7), INVALID),
    (_route_back, dict(logits=None), INVALID), (_route_back, dict(ends=None), INVALID), (_route_back, dict(dl=None), INVALID),
    (_route_back, dict(ldd=7), INVALID), (_route_back, dict(dw=0x1002), UNSUPPORTED), (_route_back, dict(scale=-INF), INVALID),
    (_route_back, dict(top=9), INVALID), (_route_back, dict(db=0x1002), UNSUPPORTED),
    (_gather, dict(count=-1), INVALID), (_gather, dict(count=BIG), INVALID), (_gather, dict(rows=-1), INVALID),
    (_gather, dict(top=0), INVALID), (_gather, dict(top=65), INVALID), (_gather, dict(d=0), INVALID), (_gather, dict(d=65537), INVALID),
    (_gather, dict(ldx=7), INVALID), (_gather, dict(ldo=7), INVALID), (_gather, dict(x=None), INVALID),
    (_gather, dict(slots=None), INVALID), (_gather, dict(out=None), INVALID), (_gather, dict(used=0x1002), UNSUPPORTED),
    (_combine, dict(y=None), INVALID), (_combine, dict(out=None), INVALID), (_combine, dict(slots=None), INVALID),
    (_combine, dict(ldr=7), INVALID), (_combine, dict(ldy=7), INVALID), (_combine, dict(w=0x1002), UNSUPPORTED),
    (_combine, dict(dtype=3), INVALID), (_combine, dict(top=65), INVALID),
    (_combine_back, dict(g=None), INVALID), (_combine_back, dict(y=None), INVALID), (_combine_back, dict(dy=None), INVALID),
    (_combine_back, dict(ldg=7), INVALID), (_combine_back, dict(lddy=7), INVALID), (_combine_back, dict(dw=0x1001), UNSUPPORTED),
    (_combine_back, dict(slots=None), INVALID),
    (_logp, dict(vocab=0), INVALID), (_logp, dict(vocab=(1 << 30) + 1), INVALID), (_logp, dict(ld=63), INVALID),
    (_logp, dict(top=-1), INVALID), (_logp, dict(top=65), INVALID), (_logp, dict(vocab=1, top=2), INVALID),
    (_logp, dict(temp=0.0), INVALID), (_logp, dict(temp=NAN), INVALID), (_logp, dict(logp=None), INVALID),
    (_logp, dict(stats=None), INVALID), (_logp, dict(stats=0x1004), UNSUPPORTED), (_logp, dict(tl=None), INVALID),
    (_logp, dict(ti=None), INVALID), (_logp, dict(ti=0x1004), UNSUPPORTED), (_logp, dict(targets=0x1004), UNSUPPORTED),
    (_logp_back, dict(dl=None), INVALID), (_logp_back, dict(stats=None), INVALID), (_logp_back, dict(entropy=None), INVALID),
    (_logp_back, dict(ldd=63), INVALID), (_logp_back, dict(temp=-1.0), INVALID), (_logp_back, dict(g=0x1002), UNSUPPORTED),
])
def test_refused(call, bad, code):
    assert call(**bad) == code
    assert tm.last_error() != ""


def test_nothing_to_do():
    assert _rms(rows=0, x=None, s=None, y=None, rstd=None) == tm.TM_OK
    assert _rms_back(rows=0, dw=None) == tm.TM_OK
    assert _route_back(rows=0, logits=None) == tm.TM_OK
    assert _gather(count=0, out=None) == tm.TM_OK and _combine(rows=0, out=None) == tm.TM_OK
    assert _combine_back(count=0, rows=0) == tm.TM_OK and _combine_back(count=0, dw=None) == tm.TM_OK
    assert _logp(rows=0, logits=None) == tm.TM_OK and _logp_back(rows=0) == tm.TM_OK


@pytest.mark.parametrize("call,size", [
    (_logp, dict(rows=1 << 27, vocab=2000, ld=2000)), (_logp, dict(rows=1 << 24, vocab=8000, ld=8000)),
    (_logp, dict(rows=1 << 24, vocab=100000, ld=100000)), (_logp_back, dict(rows=1 << 24, vocab=64)),
    (_logp_back, dict(rows=1 << 30, vocab=1 << 20, ld=1 << 20, ldd=1 << 20)),
])
def test_launches_past_32_bits_of_threads_are_refused(call, size):
    assert call(**size) == UNSUPPORTED
    assert "too many blocks" in tm.last_error()


def test_python_checks_come_before_the_library():
    torch = pytest.importorskip("torch")
    x = torch.zeros((2, 4))
    i = torch.zeros((2, 1), dtype=torch.int32)
    for call in (lambda: tm.rms_norm(x), lambda: tm.rms_norm(x.double()), lambda: tm.rms_norm_backward(x, x, x[:, 0]),
                 lambda: tm.expert_route(x, 2), lambda: tm.expert_route_backward(x, i, i[0]), lambda: tm.expert_gather(x, i),
                 lambda: tm.expert_combine(x, i), lambda: tm.expert_combine_backward(x, x, i),
                 lambda: tm.token_logp(x, i[:, 0].long()), lambda: tm.token_logp_backward(x, i[:, 0].long(), x, x[:, 0])):
        with pytest.raises(ValueError):
            call()


def test_limits_match_the_header():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = open(os.path.join(root, "include", "turbomuon.h")).read()
    d = {k: int(v) for k, v in re.findall(r"#define\s+(TM_MAX_\w+)\s+(\d+)", text)}
    assert d["TM_MAX_TOP"] == tm.TM_MAX_TOP


@pytest.mark.parametrize("rows", [(1 << 26) - 3, (1 << 26) - 2, (1 << 26) - 1])
def test_four_rows_a_workgroup_are_counted_as_the_workgroup_that_they_fill(rows):
    """Rows of up to 2048 logits go four to a workgroup of 256: the last workgroup counts in full, and 2^24 of them are
    one thread too many for a launch."""
    for vocab in (2, 1000, 2048):
        for dtype in (0, 1):
            assert _logp(rows=rows, vocab=vocab, ld=vocab, top=min(vocab, 2), dtype=dtype) == UNSUPPORTED
            assert "too many blocks" in tm.last_error()
