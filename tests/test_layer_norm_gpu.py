"""Layer norm on the GPU against its definition in 64 bits.

Tolerances, from the arithmetic (u = 2^-24): a sum over d elements is a tree of
at most 16 + 10 additions per thread and row up to d = 16384 and of d / 1024 + 10
beyond, so a mean is off by at most S u mean|x| with S = 64 + d / 1024; the rest
of an output is a handful of roundings.  bf16 outputs are rounded once, 2^-8 of
themselves.  Column sums add at most rows / 4 + 64 terms after one another.
"""
import pytest

from gpu_helpers import log

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from paper_2512_04632_amd import _lib as tm, ops  # noqa: E402

U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _round(dtype):
    return 2.0 ** -8 if dtype == "bf16" else U


def _inputs(rows, d, dtype, seed=0, offset=0.5, scale=1.5):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = (torch.randn((rows, d), generator=g, device="cuda") * scale + offset).to(DT[dtype])
    w = 1 + 0.2 * torch.randn(d, generator=g, device="cuda")
    b = 0.2 * torch.randn(d, generator=g, device="cuda")
    dy = torch.randn((rows, d), generator=g, device="cuda").to(DT[dtype])
    return x, w, b, dy


def _forward64(x, w, b, eps):
    x = x.double()
    mean = x.mean(-1)
    var = (x - mean[:, None]).square().mean(-1)
    rstd = (var + eps).rsqrt()
    y = (x - mean[:, None]) * rstd[:, None]
    if w is not None:
        y = y * w.double()
    if b is not None:
        y = y + b.double()
    return y, mean, rstd


def _close(name, got, want, bound):
    off = (got.double() - want).abs()
    bad = ~(off <= bound)
    assert not bad.any(), (name, int(bad.sum()), float(off.max()), float((off / bound).max()))


def _check_forward(x, w, b, eps, dtype, got):
    y, mean, rstd = got
    want, m64, r64 = _forward64(x, w, b, eps)
    d = x.shape[1]
    S = 64 + d / 1024
    xa = x.double().abs()
    dm = S * U * xa.mean(-1)
    _close("mean", mean, m64, dm + U * m64.abs() + 1e-45)
    # the variance's own sum, and what the mean's error adds (its square: the mean minimises)
    rel = (S + 8) * U + dm.square() * r64.square()
    _close("rstd", rstd, r64, rel * r64)
    wa = torch.ones(d, device="cuda").double() if w is None else w.double().abs()
    part = (x.double() - m64[:, None]).abs() * r64[:, None] * wa
    bound = part * (rel[:, None] + 8 * U) + (dm * r64)[:, None] * wa * 1.01 + 4 * U * want.abs() \
        + (0 if b is None else 4 * U * b.double().abs())
    _close("y", y, want, bound * 1.01 + _round(dtype) * (want.abs() + bound) + 1e-38)


SIZES = [(1, 1), (3, 1), (1, 7), (5, 8), (2, 64), (7, 65), (9, 511), (4, 512), (5, 513), (33, 768), (6, 1001),
         (3, 1024), (4, 1025), (5, 2047), (3, 4096), (2, 4099), (3, 8192), (2, 8200), (2, 16384), (3, 16387),
         (2, 40001), (1, 65536)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,d", SIZES)
def test_forward(rows, d, dtype):
    log(f"case: layer norm forward {rows} x {d} {dtype}")
    x, w, b, _ = _inputs(rows, d, dtype)
    _check_forward(x, w, b, 1e-5, dtype, tm.layer_norm(x, w, b, eps=1e-5))
    _check_forward(x, None, None, 1e-3, dtype, tm.layer_norm(x, eps=1e-3))


def _check_backward(x, w, dy, mean, rstd, dtype, got):
    dx, dw, db = got
    rows, d = x.shape
    h = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    g = dy.double() * (1 if w is None else w.double())
    m0, m1 = g.mean(-1, keepdim=True), (g * h).mean(-1, keepdim=True)
    want = rstd.double()[:, None] * (g - m0 - h * m1)
    S = 64 + d / 1024
    r = rstd.double()[:, None]
    # h carries the rounding of x - mean, relative to x and mean
    dh = U * (4 * h.abs() + r * (x.double().abs() + mean.double().abs()[:, None]))
    e0 = S * U * g.abs().mean(-1, keepdim=True)
    e1 = S * U * (g * h).abs().mean(-1, keepdim=True) + (g.abs() * dh).mean(-1, keepdim=True)
    bound = r * (8 * U * (g.abs() + m0.abs() + (h * m1).abs()) + e0 + h.abs() * e1 + dh * m1.abs())
    _close("dx", dx, want, bound * 1.01 + _round(dtype) * (want.abs() + bound) + 1e-38)
    terms = dy.double().abs()
    n = rows / 4 + 80
    _close("dweight", dw, (dy.double() * h).sum(0), n * U * (terms * h.abs()).sum(0) + (terms * dh).sum(0) + 1e-38)
    _close("dbias", db, dy.double().sum(0), n * U * terms.sum(0) + 1e-38)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,d", SIZES + [(4001, 100), (2500, 768), (1300, 1500), (700, 5000)])
def test_backward(rows, d, dtype):
    log(f"case: layer norm backward {rows} x {d} {dtype}")
    x, w, b, dy = _inputs(rows, d, dtype, seed=1)
    _, mean, rstd = tm.layer_norm(x, w, b, eps=1e-3)
    _check_backward(x, w, dy, mean, rstd, dtype, tm.layer_norm_backward(dy, x, mean, rstd, w))
    dx, dw, db = tm.layer_norm_backward(dy, x, mean, rstd, None)
    _check_backward(x, None, dy, mean, rstd, dtype, (dx, dw, db))
    only, none, _ = tm.layer_norm_backward(dy, x, mean, rstd, None, param_grads=False)
    assert none is None and torch.equal(only, dx)


def test_same_bits_on_every_run():
    x, w, b, dy = _inputs(3000, 777, "bf16", seed=5)
    _, mean, rstd = tm.layer_norm(x, w, b)
    first = tm.layer_norm_backward(dy, x, mean, rstd, w)
    for _ in range(3):
        for a, c in zip(first, tm.layer_norm_backward(dy, x, mean, rstd, w)):
            assert torch.equal(a, c)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides_and_leading_dimensions(dtype):
    log("case: layer norm on strided rows")
    x, w, b, dy = _inputs(60, 333, dtype, seed=2)
    wide = torch.zeros((60, 1000), dtype=DT[dtype], device="cuda")
    wide[:, 5:338] = x
    cut = wide[:, 5:338]                        # rows 1000 apart, at an odd offset
    ref = tm.layer_norm(x, w, b)
    for a, c in zip(ref, tm.layer_norm(cut, w, b)):
        assert torch.equal(a, c)
    y3, mean3, _ = tm.layer_norm(x.view(3, 4, 5, 333), w, b)
    assert y3.shape == (3, 4, 5, 333) and torch.equal(y3.view(60, 333), ref[0]) and mean3.shape == (60,)
    t = x.t().contiguous().t()                  # columns contiguous: copied
    assert torch.equal(tm.layer_norm(t, w, b)[0], ref[0])
    grads = tm.layer_norm_backward(dy, x, ref[1], ref[2], w)
    wide2 = torch.zeros((60, 700), dtype=DT[dtype], device="cuda")
    wide2[:, 1:334] = dy
    for a, c in zip(grads, tm.layer_norm_backward(wide2[:, 1:334], cut, ref[1], ref[2], w)):
        assert torch.equal(a, c)
    one = torch.ones((), dtype=DT[dtype], device="cuda").expand(60, 333)   # a broadcast gradient
    for a, c in zip(tm.layer_norm_backward(one, x, ref[1], ref[2], w),
                    tm.layer_norm_backward(one.contiguous(), x, ref[1], ref[2], w)):
        assert torch.equal(a, c)


def test_rows_without_spread_and_large_offsets():
    """A constant row gives the bias; a mean a thousand times the spread costs no more than the
    inputs' own rounding (the variance is taken about the finished mean)."""
    d = 1000
    w, b = torch.full((d,), 2.0, device="cuda"), torch.full((d,), 0.25, device="cuda")
    x = torch.full((2, d), 3.0, device="cuda")
    y, mean, rstd = tm.layer_norm(x, w, b, eps=1e-5)
    assert torch.equal(mean, torch.full_like(mean, 3.0)) and torch.equal(y, torch.full_like(y, 0.25))
    assert torch.allclose(rstd, torch.full_like(rstd, 1e-5 ** -0.5), rtol=1e-6)
    x, w, b, _ = _inputs(5, d, "f32", offset=1000.0, scale=1.0)
    _check_forward(x, w, b, 1e-5, "f32", tm.layer_norm(x, w, b, eps=1e-5))


def test_nan_and_inf_stay_in_their_row():
    x, w, b, dy = _inputs(9, 300, "bf16", seed=3)
    ref = tm.layer_norm(x, w, b)
    bad = x.clone()
    bad[4, 17] = float("nan")
    bad[6, 0] = float("inf")
    y, mean, rstd = tm.layer_norm(bad, w, b)
    keep = torch.tensor([0, 1, 2, 3, 5, 7, 8], device="cuda")
    assert torch.equal(y[keep], ref[0][keep]) and torch.equal(mean[keep], ref[1][keep])
    assert y[4].isnan().all() and y[6].isnan().all()
    dx, _, _ = tm.layer_norm_backward(dy, bad, mean, rstd, w)
    assert torch.equal(dx[keep], tm.layer_norm_backward(dy, x, ref[1], ref[2], w)[0][keep])


def test_no_rows():
    w = torch.ones(64, device="cuda")
    x = torch.empty((0, 64), device="cuda")
    y, mean, rstd = tm.layer_norm(x, w, w)
    assert y.shape == (0, 64) and mean.shape == rstd.shape == (0,)
    dx, dw, db = tm.layer_norm_backward(x, x, mean, rstd, w)
    assert dx.shape == (0, 64) and not dw.any() and not db.any()


def test_in_place():
    for rows, d in ((300, 500), (3, 20000)):
        x, w, b, dy = _inputs(rows, d, "f32", seed=4)
        y, mean, rstd = tm.layer_norm(x, w, b)
        dx, dw, _ = tm.layer_norm_backward(dy, x, mean, rstd, w)
        s = torch.cuda.current_stream().cuda_stream
        xc, dyc = x.clone(), dy.clone()
        m2, r2, dw2 = torch.empty_like(mean), torch.empty_like(rstd), torch.empty_like(dw)
        L = tm.lib()
        assert L.tm_layer_norm_backward(dyc.data_ptr(), d, xc.data_ptr(), d, w.data_ptr(), mean.data_ptr(),
                                        rstd.data_ptr(), dyc.data_ptr(), d, dw2.data_ptr(), None, rows, d, 1, s) == 0
        assert L.tm_layer_norm(xc.data_ptr(), d, w.data_ptr(), b.data_ptr(), xc.data_ptr(), d, m2.data_ptr(),
                               r2.data_ptr(), rows, d, 1e-5, 1, s) == 0
        assert torch.equal(xc, y) and torch.equal(dyc, dx) and torch.equal(dw2, dw)


def test_gradient_against_differences():
    """autograd's gradients against central differences of the 64-bit definition."""
    x, w, b, dy = _inputs(4, 37, "f32", seed=6)
    leaves = [t.clone().requires_grad_() for t in (x, w, b)]
    ops.layer_norm(*leaves, 1e-3).backward(dy)

    def value(x, w, b):
        return float((_forward64(x, w, b, 1e-3)[0] * dy.double()).sum())

    g = torch.Generator().manual_seed(0)
    for k, leaf in enumerate(leaves):
        for _ in range(6):
            i = int(torch.randint(leaf.numel(), (), generator=g))
            args = [t.detach().double().clone() for t in (x, w, b)]
            flat = args[k].view(-1)
            flat[i] += 1e-4
            up = value(*args)
            flat[i] -= 2e-4
            diff = (up - value(*args)) / 2e-4
            got = float(leaf.grad.reshape(-1)[i])
            assert abs(got - diff) <= 1e-4 * (1 + abs(diff)), (k, i, got, diff)


def test_refusals():
    x, w, b, dy = _inputs(4, 32, "f32")
    _, mean, rstd = tm.layer_norm(x, w, b)
    for bad in (lambda: tm.layer_norm(x.cpu(), w, b), lambda: tm.layer_norm(x.half(), w, b),
                lambda: tm.layer_norm(x, w[:5], b), lambda: tm.layer_norm(x, w.bfloat16(), b),
                lambda: tm.layer_norm_backward(dy[:2], x, mean, rstd, w),
                lambda: tm.layer_norm_backward(dy.bfloat16(), x, mean, rstd, w),
                lambda: tm.layer_norm_backward(dy, x, mean[:3], rstd, w)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(tm.TurboMuonError) as e:
        tm.layer_norm(x, w, b, eps=-1.0)
    assert e.value.status == tm.TM_ERR_INVALID_ARG
    with pytest.raises(tm.TurboMuonError):
        tm.layer_norm(torch.empty((1, 70000), device="cuda"))
