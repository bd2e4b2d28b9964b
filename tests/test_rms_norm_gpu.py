"""Root-mean-square norm on the GPU against its definition in 64 bits.

Tolerances (u = 2^-24): a row's sum of squares is a tree of at most 64 + 6 + 16 additions of positive terms,
each of one rounding, off by under 88 u of itself; rstd is off by half of that and four roundings, R = 48 u;
y by two products more and its rounding.  Backwards the sum of g h is off by at most 90 u of the sum of |g h|
(the terms carry two roundings), and what it is multiplied with by a few u; a column's sum is one of at most
rows / 64 + 100 additions."""
import pytest

from gpu_helpers import log

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from op_helpers import DT, U, close, far, generator, rounded, spread  # noqa: E402
from paper_2512_04632_amd import _lib as tm, ops  # noqa: E402

R = 48 * U
EPS = 1e-5


def _inputs(rows, d, dtype, seed=0):
    g = generator(seed)

    def randn(*s):
        return torch.randn(s, generator=g, device="cuda")

    return dict(x=randn(rows, d).to(DT[dtype]), residual=(3 * randn(rows, d)).to(DT[dtype]), weight=1 + 0.3 * randn(d),
                dy=randn(rows, d).to(DT[dtype]), dsum=randn(rows, d).to(DT[dtype]))


def _check_forward(got, x, residual, weight, dtype, eps=EPS):
    y, s, rstd = got
    want = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    assert torch.equal(s, want)
    v = want.double()
    scale = (v.pow(2).mean(1) + eps).rsqrt()
    close("rstd", rstd, scale, R * scale)
    out = v * scale[:, None] * (1 if weight is None else weight.double())
    close("y", y, out, rounded(out, (R + 4 * U) * out.abs(), dtype))


def _check_backward(got, s, rstd, dy, dsum, weight, dtype):
    ds, dweight = got
    rows, d = s.shape
    r, g = rstd.double()[:, None], dy.double()
    h = s.double() * r
    if dweight is not None:
        want = (g * h).sum(0)
        close("dweight", dweight, want, (rows / 64 + 100) * U * (g * h).abs().sum(0) + 1e-38)
    if weight is not None:
        g = g * weight.double()
    m = (g * h).mean(1, keepdim=True)
    want = r * (g - h * m)
    off = r * (4 * U * g.abs() + 6 * U * (h * m).abs() + 92 * U * h.abs() * (g * h).abs().mean(1, keepdim=True))
    if dsum is not None:
        want = want + dsum.double()
        off = off + U * want.abs()
    close("ds", ds, want, rounded(want, off, dtype))


# one row to many; one element, rows below and above the sizes at which they get more threads, or are not
# held; odd ones
SIZES = [(1, 1), (3, 2), (5, 7), (64, 96), (700, 65), (9, 511), (9, 512), (33, 1000), (5, 1023), (6, 1025), (17, 2048),
         (300, 2050), (40, 4096), (3, 4099), (12, 8192), (5, 8190), (4, 16384), (3, 16383), (3, 16385), (2, 30011),
         (1, 65536), (2500, 130), (5000, 24)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,d", SIZES)
def test_forward_and_backward(rows, d, dtype):
    log(f"case: rms norm {rows} x {d} {dtype}")
    t = _inputs(rows, d, dtype, seed=rows + d)
    got = tm.rms_norm(t["x"], t["weight"], t["residual"], eps=EPS)
    _check_forward(got, t["x"], t["residual"], t["weight"], dtype)
    plain = tm.rms_norm(t["x"], eps=EPS)
    _check_forward(plain, t["x"], None, None, dtype)
    assert plain[1] is t["x"]
    args = (t["dy"], got[1], got[2])
    back = tm.rms_norm_backward(*args, t["weight"], t["dsum"])
    _check_backward(back, got[1], got[2], t["dy"], t["dsum"], t["weight"], dtype)
    _check_backward(tm.rms_norm_backward(*args, None, None), got[1], got[2], t["dy"], None, None, dtype)
    less = tm.rms_norm_backward(*args, t["weight"], t["dsum"], param_grads=False)
    assert less[1] is None and torch.equal(less[0], back[0])
    again = tm.rms_norm(t["x"], t["weight"], t["residual"], eps=EPS)
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    assert all(torch.equal(a, b) for a, b in zip(back, tm.rms_norm_backward(*args, t["weight"], t["dsum"])))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,d", [(7, 65), (30, 1001), (30, 2047), (9, 5000), (5, 9001), (3, 20001)])
def test_strides_and_other_orders(rows, d, dtype):
    t = _inputs(rows, d, dtype, seed=3)
    ref = tm.rms_norm(t["x"], t["weight"], t["residual"])
    back = tm.rms_norm_backward(t["dy"], ref[1], ref[2], t["weight"], t["dsum"])
    for other in (lambda a: spread(a, 13, 5), lambda a: a.t().contiguous().t()):
        got = tm.rms_norm(other(t["x"]), t["weight"], other(t["residual"]))
        assert all(torch.equal(a, b) for a, b in zip(ref, got))
        got = tm.rms_norm_backward(other(t["dy"]), other(ref[1]), ref[2], t["weight"], other(t["dsum"]))
        assert all(torch.equal(a, b) for a, b in zip(back, got))
    three = tm.rms_norm(t["x"].view(1, rows, d), t["weight"], t["residual"].view(1, rows, d))
    assert three[0].shape == (1, rows, d) and three[2].shape == (rows,) and torch.equal(three[0][0], ref[0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,d", [(70, 61), (70, 515), (70, 1999), (9, 5000), (9, 16001), (3, 20003)])
def test_in_place(rows, d, dtype):
    """s in the place of x or of the residual, y in that of the other; ds in the place of each of its inputs."""
    t = _inputs(rows, d, dtype, seed=4)
    y, s, rstd = tm.rms_norm(t["x"], t["weight"], t["residual"])
    ds, dw = tm.rms_norm_backward(t["dy"], s, rstd, t["weight"], t["dsum"])
    code, st = (0 if dtype == "bf16" else 1), torch.cuda.current_stream().cuda_stream
    for swap in (False, True):
        x, r, scale = t["x"].clone(), t["residual"].clone(), torch.empty_like(rstd)
        to_s, to_y = (r, x) if swap else (x, r)
        assert tm.lib().tm_rms_norm(x.data_ptr(), d, r.data_ptr(), d, t["weight"].data_ptr(), to_s.data_ptr(), d,
                                    to_y.data_ptr(), d, scale.data_ptr(), rows, d, 1e-5, code, st) == 0
        assert torch.equal(to_s, s) and torch.equal(to_y, y) and torch.equal(scale, rstd)
    x, scale = t["x"].clone(), torch.empty_like(rstd)
    alone = tm.rms_norm(x, t["weight"])
    assert tm.lib().tm_rms_norm(x.data_ptr(), d, None, 0, t["weight"].data_ptr(), None, 0, x.data_ptr(), d, scale.data_ptr(),
                                rows, d, 1e-5, code, st) == 0
    assert torch.equal(x, alone[0]) and torch.equal(scale, alone[2])
    for k in range(3):
        arrays = [t["dy"].clone(), s.clone(), t["dsum"].clone()]
        got = torch.empty_like(dw)
        assert tm.lib().tm_rms_norm_backward(arrays[0].data_ptr(), d, arrays[1].data_ptr(), d, t["weight"].data_ptr(),
                                             rstd.data_ptr(), arrays[2].data_ptr(), d, arrays[k].data_ptr(), d,
                                             got.data_ptr(), rows, d, code, st) == 0
        assert torch.equal(arrays[k], ds) and torch.equal(got, dw)


def test_rows_that_are_not_numbers_leave_the_others_alone():
    for d in (300, 5000, 20000):
        t = _inputs(6, d, "f32", seed=5)
        ref = tm.rms_norm(t["x"], t["weight"], t["residual"])
        t["x"][1, 3], t["x"][4, 0] = float("nan"), float("inf")
        t["x"][2], t["residual"][2] = 0.0, 0.0
        y, s, rstd = tm.rms_norm(t["x"], t["weight"], t["residual"])
        keep = [0, 3, 5]
        assert torch.equal(y[keep], ref[0][keep]) and torch.equal(rstd[keep], ref[2][keep])
        assert rstd[1].isnan() and y[1].isnan().all() and rstd[4] == 0
        assert not y[2].any() and abs(float(rstd[2]) - EPS ** -0.5) < 1e-3


def test_offsets_past_32_bits():
    for dtype, d in (("bf16", 4096), ("f32", 1001)):
        t = _inputs(20, d, dtype, seed=6)
        ref = tm.rms_norm(t["x"], t["weight"], t["residual"])
        got = tm.rms_norm(far(t["x"], 1 << 28), t["weight"], t["residual"])
        assert all(torch.equal(a, b) for a, b in zip(ref, got))
        back = tm.rms_norm_backward(t["dy"], ref[1], ref[2], t["weight"], t["dsum"])
        got = tm.rms_norm_backward(far(t["dy"], 1 << 28), ref[1], ref[2], t["weight"], t["dsum"])
        assert all(torch.equal(a, b) for a, b in zip(back, got))


@pytest.mark.parametrize("residual", [False, True])
def test_autograd(residual):
    """Against automatic differentiation of the definition in 64 bits, both results used, or one alone."""
    t = _inputs(50, 300, "f32", seed=7)
    for use in ("y", "s", "both") if residual else ("y",):
        leaves = [t["x"].clone().requires_grad_(), t["weight"].clone().requires_grad_()]
        wide = [v.detach().double().requires_grad_() for v in leaves]
        if residual:
            leaves.append(t["residual"].clone().requires_grad_())
            wide.append(t["residual"].double().requires_grad_())
            y, s = ops.rms_norm(*leaves)
        else:
            y, s = ops.rms_norm(*leaves), leaves[0]
        total = wide[0] + wide[2] if residual else wide[0]
        norm = total * (total.pow(2).mean(1, keepdim=True) + EPS).rsqrt() * wide[1]
        gy, gs = t["dy"] * (use != "s"), t["dsum"] * (use != "y")
        parts = ([(y, gy)] if use != "s" else []) + ([(s, gs)] if use != "y" else [])
        torch.autograd.backward([a for a, _ in parts], [b for _, b in parts])
        ((norm * gy.double()).sum() + (total * gs.double()).sum()).backward()
        for a, b in zip(leaves, wide):
            if use == "s" and a is leaves[1]:
                assert a.grad is None
                continue
            # s is rounded before it is normalised: 2^-24 of it, up to some tens in h and its sums
            assert torch.allclose(a.grad.double(), b.grad, rtol=1e-5, atol=1e-5 * float(b.grad.abs().max()))


def test_gradient_against_differences():
    t = _inputs(3, 40, "f32", seed=8)

    def value(x, w):
        return ((x * (x.pow(2).mean(1, keepdim=True) + EPS).rsqrt() * w) * t["dy"].double()).sum()

    x, w = t["x"].double(), t["weight"].double()
    _, s, rstd = tm.rms_norm(t["x"], t["weight"])
    ds, dw = tm.rms_norm_backward(t["dy"], s, rstd, t["weight"])
    for r, c in ((0, 0), (1, 17), (2, 39)):
        step = torch.zeros_like(x)
        step[r, c] = 1e-5
        diff = (value(x + step, w) - value(x - step, w)) / 2e-5
        assert abs(float(ds[r, c]) - float(diff)) <= 1e-5 * (1 + abs(float(diff)))
        diff = (value(x, w + step[r]) - value(x, w - step[r])) / 2e-5
        assert abs(float(dw[c]) - float(diff)) <= 1e-5 * (1 + abs(float(diff)))


def test_no_rows_and_refusals():
    t = _inputs(4, 64, "f32")
    y, s, rstd = tm.rms_norm(t["x"][:0], t["weight"], t["residual"][:0])
    assert y.shape == (0, 64) and s.shape == (0, 64) and rstd.shape == (0,)
    ds, dw = tm.rms_norm_backward(t["dy"][:0], s, rstd, t["weight"])
    assert ds.shape == (0, 64) and not dw.any()
    for bad in (dict(x=t["x"].half()), dict(x=t["x"].cpu()), dict(weight=t["weight"][:3]), dict(weight=t["weight"].double()),
                dict(residual=t["residual"][:2]), dict(residual=t["residual"].bfloat16()),
                dict(residual=t["residual"].cpu())):
        with pytest.raises(ValueError):
            tm.rms_norm(**dict(dict(x=t["x"], weight=t["weight"], residual=t["residual"]), **bad))
    y, s, rstd = tm.rms_norm(t["x"], t["weight"])
    for bad in (dict(dy=t["dy"][:2]), dict(dy=t["dy"].bfloat16()), dict(rstd=rstd[:2]), dict(rstd=rstd.double()),
                dict(dsum=t["dsum"][:, :5]), dict(weight=t["weight"][:3])):
        with pytest.raises(ValueError):
            tm.rms_norm_backward(**dict(dict(dy=t["dy"], s=s, rstd=rstd, weight=t["weight"]), **bad))
    with pytest.raises(tm.TurboMuonError) as e:
        tm.rms_norm(t["x"], eps=-1.0)
    assert e.value.status == tm.TM_ERR_INVALID_ARG
