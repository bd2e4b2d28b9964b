"""Rows to their experts and back on the GPU against plain indexing.

Rows on their way out are copied bit for bit.  Tolerances (u = 2^-24): a weighted sum of `top` rows and a residual is
off by (top + 2) u of the sum of sizes and rounded once; a weight's gradient is a sum over the columns of at most
d / 256 + 40 additions a thread and tree."""
import contextlib

import pytest

from gpu_helpers import log

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from op_helpers import DT, U, close, far, generator, rounded, spread  # noqa: E402
from paper_2512_04632_amd import _lib as tm, ops  # noqa: E402


def _inputs(rows, top, d, dtype, masked=0.2, seed=0):
    g = generator(seed)

    def randn(*s):
        return torch.randn(s, generator=g, device="cuda")

    count = rows * top
    active = torch.rand(rows, generator=g, device="cuda") >= masked
    slots = torch.full((rows, top), -1, dtype=torch.int32, device="cuda")
    used = int(active.sum()) * top
    slots[active] = torch.randperm(used, generator=g, device="cuda").int().view(-1, top)
    ends = torch.tensor([used // 3, used // 3, used], dtype=torch.int32, device="cuda")
    return dict(x=randn(rows, d).to(DT[dtype]), y=randn(count, d).to(DT[dtype]), slots=slots, ends=ends,
                weights=torch.rand((rows, top), generator=g, device="cuda") * active[:, None],
                residual=randn(rows, d).to(DT[dtype]), dout=randn(rows, d).to(DT[dtype]))


def _gathered(x, slots, count):
    out = x.new_zeros(count, x.shape[1])
    which = (slots >= 0).nonzero()
    out[slots[which[:, 0], which[:, 1]].long()] = x[which[:, 0]]
    return out


def _combined(t, weights, residual):
    """The sum in 64 bits, and the sum of sizes."""
    on = (t["slots"] >= 0)[..., None]
    parts = torch.where(on, t["y"][t["slots"].clamp(min=0).long()].double(), 0)
    if weights is not None:
        parts = parts * weights.double()[..., None]
    total, size = parts.sum(1), parts.abs().sum(1)
    if residual is not None:
        total, size = total + residual.double(), size + residual.double().abs()
    return total, size


def _check(t, dtype, rows, top, d):
    count = rows * top
    out = tm.expert_gather(t["x"], t["slots"], t["ends"])
    assert torch.equal(out, _gathered(t["x"], t["slots"], count))
    for weights, residual in ((t["weights"], t["residual"]), (t["weights"], None), (None, None)):
        want, size = _combined(t, weights, residual)
        got = tm.expert_combine(t["y"], t["slots"], weights, residual)
        close("combine", got, want, rounded(want, (top + 2) * U * size, dtype))
    dy, dw = tm.expert_combine_backward(t["dout"], t["y"], t["slots"], t["ends"], t["weights"])
    products = t["dout"].double()[:, None] * t["y"][t["slots"].clamp(min=0).long()].double()
    on = t["slots"] >= 0
    want = torch.where(on, products.sum(2), 0)
    close("dweights", dw, want, (d / 256 + 40) * U * products.abs().sum(2) + 1e-38)
    want = torch.zeros((count, d), dtype=torch.float64, device="cuda")
    at = on.nonzero()
    want[t["slots"][at[:, 0], at[:, 1]].long()] = (t["weights"].double()[..., None] * t["dout"].double()[:, None])[on]
    close("dy", dy, want, rounded(want, U * want.abs(), dtype))
    less = tm.expert_combine_backward(t["dout"], t["y"], t["slots"], t["ends"], t["weights"], weight_grads=False)
    assert less[1] is None and torch.equal(less[0], dy)
    again = tm.expert_combine_backward(t["dout"], t["y"], t["slots"], t["ends"], t["weights"])
    assert torch.equal(again[0], dy) and torch.equal(again[1], dw)


# rows, top, width: one of each to many; widths around those at which a row gets more threads; odd ones
SIZES = [(1, 1, 1), (2, 3, 2), (5, 2, 7), (70, 1, 33), (64, 2, 64), (100, 4, 127), (33, 8, 129), (300, 2, 512), (7, 64, 515),
         (50, 9, 1024), (20, 3, 1025), (17, 8, 2048), (9, 2, 2050), (31, 5, 4099), (4, 16, 8192), (3, 2, 65536), (2, 7, 30001),
         (3001, 3, 65), (9000, 2, 16)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,top,d", SIZES)
def test_out_and_back(rows, top, d, dtype):
    log(f"case: rows to experts {rows} top {top} x {d} {dtype}")
    _check(_inputs(rows, top, d, dtype, seed=rows + d), dtype, rows, top, d)


@pytest.mark.parametrize("masked", [0.0, 1.0])
def test_all_rows_or_none(masked):
    for rows, top, d in ((40, 3, 100), (9, 2, 5000)):
        _check(_inputs(rows, top, d, "bf16", masked=masked, seed=1), "bf16", rows, top, d)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [60, 1001, 3000])
def test_what_has_no_slot_is_not_read(d, dtype):
    """NaN in the rows of no slot, of x, y and the gradient, reaches nothing, and rows past the filled ones come
    out as zeros."""
    t = _inputs(50, 3, d, dtype, seed=2)
    off, used = (t["slots"] < 0).all(1), int(t["ends"][-1])
    assert off.any()
    for name in ("x", "dout", "weights"):
        t[name][off] = float("nan")
    t["y"][used:] = float("nan")
    out = tm.expert_gather(t["x"], t["slots"], t["ends"])
    back = tm.expert_combine(t["y"], t["slots"], t["weights"], t["residual"])
    dy, dw = tm.expert_combine_backward(t["dout"], t["y"], t["slots"], t["ends"], t["weights"])
    for a in (out, back, dy, dw):
        assert torch.isfinite(a).all()
    assert not out[used:].any() and not dy[used:].any() and not dw[off].any()
    assert torch.equal(back[off], t["residual"][off])


def test_slots_and_ends_that_are_wrong_stay_within_the_matrices():
    for d in (40, 900, 3000):
        t = _inputs(30, 2, d, "f32", masked=0.0, seed=3)
        count = 60
        ref = tm.expert_gather(t["x"], t["slots"], t["ends"])
        wild = t["slots"].clone()
        wild[4, 0], wild[9, 1], wild[11, 0], wild[20, 1] = count, 2 ** 31 - 1, -2 ** 31, -7
        kept = tm.expert_combine(t["y"], wild, t["weights"])
        on = (wild >= 0) & (wild < count)
        want, size = _combined(dict(t, slots=torch.where(on, wild, -1)), t["weights"], None)
        close("combine", kept, want, 4 * U * size + U * want.abs() + 1e-38)
        dw = tm.expert_combine_backward(t["dout"], t["y"], wild, t["ends"], t["weights"])[1]
        assert not dw[~on].any()
        guard = torch.full((count + 2, d), 5.0, device="cuda")
        for ends in (2 ** 31 - 1, count + 1, -3, 17):
            used = torch.tensor(ends, dtype=torch.int32, device="cuda")
            guard.fill_(5.0)
            assert tm.lib().tm_expert_gather(t["x"].data_ptr(), d, wild.data_ptr(), used.data_ptr(), guard[1].data_ptr(), d,
                                             count, 30, 2, d, 1, torch.cuda.current_stream().cuda_stream) == 0
            assert (guard[0] == 5).all() and (guard[-1] == 5).all()
            filled = min(max(ends, 0), count)
            assert not guard[1 + filled:-1].any()
            there = torch.zeros(count, dtype=torch.bool, device="cuda")
            there[wild[on & (wild < filled)].long()] = True
            assert torch.equal(guard[1:-1][there], ref[there]) and (guard[1:-1][:filled][~there[:filled]] == 5).all()


def test_one_row_named_twice():
    """A row of y may stand in several slots of the way back."""
    y = torch.randn((4, 70), generator=generator(4), device="cuda")
    slots = torch.tensor([[1, 1], [3, 1], [0, 0]], dtype=torch.int32, device="cuda")
    w = torch.rand((3, 2), generator=generator(5), device="cuda")
    want = (y.double()[slots.long()] * w.double()[..., None]).sum(1)
    close("combine", tm.expert_combine(y, slots, w), want, 4 * U * (y.double()[slots.long()].abs() * w[..., None]).sum(1))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [61, 700, 2050])
def test_strides_and_in_place(d, dtype):
    t = _inputs(40, 3, d, dtype, seed=6)
    out = tm.expert_gather(t["x"], t["slots"], t["ends"])
    back = tm.expert_combine(t["y"], t["slots"], t["weights"], t["residual"])
    dy, dw = tm.expert_combine_backward(t["dout"], t["y"], t["slots"], t["ends"], t["weights"])
    for other in (lambda a: spread(a, 13, 5), lambda a: a.t().contiguous().t()):
        s = {k: (other(v) if v.dim() == 2 and k not in ("slots", "weights") else v) for k, v in t.items()}
        s["slots"], s["weights"] = t["slots"].t().contiguous().t(), t["weights"].t().contiguous().t()
        assert torch.equal(tm.expert_gather(s["x"], s["slots"], s["ends"]), out)
        assert torch.equal(tm.expert_combine(s["y"], s["slots"], s["weights"], s["residual"]), back)
        got = tm.expert_combine_backward(s["dout"], s["y"], s["slots"], s["ends"], s["weights"])
        assert torch.equal(got[0], dy) and torch.equal(got[1], dw)
    code, st = (0 if dtype == "bf16" else 1), torch.cuda.current_stream().cuda_stream
    res, y, got = t["residual"].clone(), t["y"].clone(), torch.empty_like(dw)
    assert tm.lib().tm_expert_combine(y.data_ptr(), d, t["slots"].data_ptr(), None, t["weights"].data_ptr(), res.data_ptr(), d,
                                      res.data_ptr(), d, 120, 40, 3, d, code, st) == 0
    assert torch.equal(res, back)
    used = t["ends"].data_ptr() + 8
    assert tm.lib().tm_expert_combine_backward(t["dout"].data_ptr(), d, y.data_ptr(), d, t["slots"].data_ptr(), used,
                                               t["weights"].data_ptr(), y.data_ptr(), d, got.data_ptr(), 120, 40, 3, d, code,
                                               st) == 0
    assert torch.equal(y, dy) and torch.equal(got, dw)


def test_offsets_past_32_bits():
    t = _inputs(12, 2, 3000, "bf16", seed=7)
    out = tm.expert_gather(t["x"], t["slots"], t["ends"])
    back = tm.expert_combine(t["y"], t["slots"], t["weights"])
    grads = tm.expert_combine_backward(t["dout"], t["y"], t["slots"], t["ends"], t["weights"])
    s = dict(t, x=far(t["x"], 1 << 28), y=far(t["y"], 1 << 28))
    assert torch.equal(tm.expert_gather(s["x"], t["slots"], t["ends"]), out)
    assert torch.equal(tm.expert_combine(s["y"], t["slots"], t["weights"]), back)
    got = tm.expert_combine_backward(t["dout"], s["y"], t["slots"], t["ends"], t["weights"])
    assert all(torch.equal(a, b) for a, b in zip(grads, got))
    wide = torch.empty((1 << 28) * 23 + 3000, dtype=torch.bfloat16, device="cuda").as_strided((24, 3000), (1 << 28, 1))
    wide.zero_()
    assert tm.lib().tm_expert_gather(t["x"].data_ptr(), 3000, t["slots"].data_ptr(), None, wide.data_ptr(), 1 << 28, 24, 12,
                                     2, 3000, 0, torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(wide, out)


def test_autograd_and_differences():
    t = _inputs(30, 3, 50, "f32", seed=8)
    leaves = {k: t[k].clone().requires_grad_() for k in ("x", "y", "weights", "residual")}
    g1 = torch.randn((90, 50), generator=generator(9), device="cuda")
    out = ops.expert_gather(leaves["x"], t["slots"], t["ends"])
    back = ops.expert_combine(leaves["y"], t["slots"], leaves["weights"], leaves["residual"], t["ends"])
    ((out * g1).sum() + (back * t["dout"]).sum()).backward()

    def value(x, y, weights, residual):
        total = _combined(dict(t, y=y), weights, residual)[0]
        return (_gathered(x, t["slots"], 90) * g1.double()).sum() + (total * t["dout"].double()).sum()

    wide = {k: t[k].double().requires_grad_() for k in leaves}
    value(**wide).backward()
    for k, leaf in leaves.items():
        assert torch.allclose(leaf.grad.double(), wide[k].grad, rtol=1e-5, atol=1e-5), k
        flat = t[k].double()
        for at in (0, flat.numel() // 2, flat.numel() - 1):
            step = torch.zeros_like(flat)
            step.view(-1)[at] = 1e-4
            args = {n: t[n].double() for n in leaves}
            diff = float(value(**dict(args, **{k: flat + step})) - value(**dict(args, **{k: flat - step}))) / 2e-4
            assert abs(float(leaf.grad.reshape(-1)[at]) - diff) <= 1e-4 * (1 + abs(diff)), k
    # without weights, and gradients that are one value spread out
    x = t["x"].clone().requires_grad_()
    ops.expert_combine(ops.expert_gather(x, t["slots"], t["ends"]), t["slots"], ends=t["ends"]).sum().backward()
    assert torch.equal(x.grad, 3.0 * (t["slots"] >= 0).any(1)[:, None].expand(30, 50))


def test_slots_past_the_filled_rows_have_no_part_and_no_gradient():
    """Rows that are cut off: ends that stop before the last slots."""
    for d in (50, 600, 1800):
        t = _inputs(30, 3, d, "f32", seed=8)
        ends = t["ends"].clamp(max=40)
        cut = torch.where((t["slots"] >= 0) & (t["slots"] < 40), t["slots"], -1)
        assert ((cut < 0) & (t["slots"] >= 0)).any()
        leaves = {k: t[k].clone().requires_grad_() for k in ("x", "y", "weights", "residual")}
        g1 = torch.randn((90, d), generator=generator(9), device="cuda")
        out = ops.expert_gather(leaves["x"], t["slots"], ends)
        back = ops.expert_combine(leaves["y"], t["slots"], leaves["weights"], leaves["residual"], ends)
        assert torch.equal(tm.expert_combine(t["y"], cut, t["weights"], t["residual"]), back)
        ((out * g1).sum() + (back * t["dout"]).sum()).backward()
        wide = {k: t[k].double().requires_grad_() for k in leaves}
        total = _combined(dict(t, y=wide["y"], slots=cut), wide["weights"], wide["residual"])[0]
        ((_gathered(wide["x"], cut, 90) * g1.double()).sum() + (total * t["dout"].double()).sum()).backward()
        assert not out[40:].any()
        # sums of three terms or one; the weights' of d products, at most d / 16 of them by one lane, then joined
        dots = float((t["dout"].abs().sum(1) * t["y"].abs().amax()).max())
        off = {"weights": (d / 16 + 16) * U * dots}
        for k, leaf in leaves.items():
            assert torch.allclose(leaf.grad.double(), wide[k].grad, rtol=1e-5, atol=off.get(k, 1e-6)), k


def test_nothing_to_do_and_refusals():
    t = _inputs(6, 2, 20, "f32", masked=0.0)
    empty = t["slots"][:0]
    assert tm.expert_gather(t["x"][:0], empty, t["ends"]).shape == (0, 20)
    assert tm.expert_combine(t["y"], empty).shape == (0, 20)
    dy, dw = tm.expert_combine_backward(t["dout"][:0], t["y"], empty, 0 * t["ends"], t["weights"][:0])
    assert not dy.any() and dw.shape == (0, 2)
    none = torch.full_like(t["slots"], -1)
    got = tm.expert_combine(t["y"][:0], none, t["weights"], t["residual"])
    assert torch.equal(got, t["residual"])
    dy, dw = tm.expert_combine_backward(t["dout"], t["y"][:0], none, None, t["weights"])
    assert dy.shape == (0, 20) and not dw.any()
    for call in (lambda: tm.expert_gather(t["x"].half(), t["slots"]), lambda: tm.expert_gather(t["x"], t["slots"].long()),
                 lambda: tm.expert_gather(t["x"], t["slots"][:3]), lambda: tm.expert_gather(t["x"][0], t["slots"]),
                 lambda: tm.expert_gather(t["x"], t["slots"], t["ends"].long()),
                 lambda: tm.expert_gather(t["x"], t["slots"], t["ends"][:0]),
                 lambda: tm.expert_gather(t["x"], t["slots"].cpu()),
                 lambda: tm.expert_combine(t["y"], t["slots"], t["weights"][:, :1]),
                 lambda: tm.expert_combine(t["y"], t["slots"], t["weights"].double()),
                 lambda: tm.expert_combine(t["y"], t["slots"], None, t["residual"].bfloat16()),
                 lambda: tm.expert_combine(t["y"], t["slots"], None, t["residual"][:2]),
                 lambda: tm.expert_combine(t["y"], t["slots"][0]),
                 lambda: tm.expert_combine_backward(t["dout"][:, :5], t["y"], t["slots"]),
                 lambda: tm.expert_combine_backward(t["dout"].bfloat16(), t["y"], t["slots"]),
                 lambda: tm.expert_combine_backward(t["dout"], t["y"], t["slots"][:2])):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(tm.TurboMuonError):
        tm.expert_gather(t["x"], t["slots"][:, :0])
    with pytest.raises(tm.TurboMuonError):
        tm.expert_combine(t["y"], torch.zeros((2, 65), dtype=torch.int32, device="cuda"))


@contextlib.contextmanager
def new_memory_is_nan():
    """Tensors that torch allocates without filling them hold NaN (or the largest integer)."""
    was = torch.are_deterministic_algorithms_enabled(), torch.utils.deterministic.fill_uninitialized_memory
    torch.use_deterministic_algorithms(True)
    torch.utils.deterministic.fill_uninitialized_memory = True
    try:
        yield
    finally:
        torch.use_deterministic_algorithms(was[0])
        torch.utils.deterministic.fill_uninitialized_memory = was[1]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [3, 60, 1001, 3000])
def test_rows_of_no_slot_are_zeros_where_no_ends_are_given(d, dtype):
    """Masked rows, and choices that the caller has taken out, with `ends` left out: the rows that no slot names, of the
    rows on their way out and of the gradients on their way back, are zeros and not what stood in their memory."""
    log(f"case: rows without slots, no ends, 50 x {d} {dtype}")
    t = _inputs(50, 3, d, dtype, seed=10)
    count, slots, st = 150, t["slots"].clone(), torch.cuda.Stream()
    slots[::4, 1] = -1                         # gaps below the last of the filled rows too
    named = torch.zeros(count, dtype=torch.bool, device="cuda")
    named[slots[slots >= 0].long()] = True
    assert not named[:int(t["ends"][-1])].all() and not named[int(t["ends"][-1]):].any()
    weights = torch.where(slots >= 0, t["weights"], 0)
    want = _gathered(t["x"], slots, count)
    dy_want = _gathered((weights[..., None] * t["dout"].float()[:, None]).to(DT[dtype]).view(150, d),
                        slots.view(150, 1), count)
    torch.cuda.synchronize()
    with new_memory_is_nan():
        assert t["x"].new_empty_strided((count, d), (d, 1)).isnan().all()
        for stream in (None, st):
            out = tm.expert_gather(t["x"], slots, stream=stream)
            dy, dw = tm.expert_combine_backward(t["dout"], t["y"], slots, None, weights, stream=stream)
            torch.cuda.synchronize()
            assert torch.equal(out, want) and torch.equal(dy, dy_want) and not dw[slots < 0].any()
        x, y, w = (v.clone().requires_grad_() for v in (t["x"], t["y"], weights))
        out = ops.expert_gather(x, slots)
        ops.expert_combine(y, slots, w).backward(t["dout"])
        assert torch.equal(out, want) and torch.equal(y.grad, dy_want) and torch.equal(w.grad, dw)


def test_rows_of_no_slot_are_zeros_in_every_replay():
    log("case: rows without slots, no ends, captured")
    t, st = _inputs(40, 2, 500, "bf16", masked=0.3, seed=11), torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        out = tm.expert_gather(t["x"], t["slots"])
        dy, dw = tm.expert_combine_backward(t["dout"], t["y"], t["slots"], None, t["weights"])
    for seed in (12, 13, 14):
        other = _inputs(40, 2, 500, "bf16", masked=0.5, seed=seed)
        for k, v in t.items():
            v.copy_(other[k])
        for a in (out, dy, dw):
            a.fill_(7)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, _gathered(t["x"], t["slots"], 80)), seed
        want = tm.expert_combine_backward(t["dout"], t["y"], t["slots"], t["ends"], t["weights"])
        assert torch.equal(dy, want[0]) and torch.equal(dw, want[1]), seed
