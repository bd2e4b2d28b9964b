"""Routing of rows to experts on the GPU against its definition in 64 bits.

Choices, slots and ends are whole numbers and have to be equal.  Tolerances (u = 2^-24): with Z the largest
distance of a score from its row's maximum, an exponential is off by Z u of its argument's rounding and under
4 u of its own, a row's sum by 48 u more: a probability by P = (4 Z + 64) u of itself.  A sum of probabilities over
a block's rows is one of at most 64 turns + 16 additions, the blocks' are joined in 64 bits."""
import pytest

from gpu_helpers import log

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from op_helpers import DT, U, close, far, generator, rounded, spread  # noqa: E402
from paper_2512_04632_amd import _lib as tm, ops  # noqa: E402


def _logits(rows, experts, dtype, seed=0, scale=2.0):
    g = generator(seed)
    bias = torch.randn(experts, generator=g, device="cuda")
    return (scale * (torch.randn((rows, experts), generator=g, device="cuda") + bias)).to(DT[dtype])


def _exact(logits, top, active, renormalize, scale):
    """(chosen, weights, slots, ends, balance) in 64 bits."""
    rows, experts = logits.shape
    on = torch.ones(rows, dtype=torch.bool, device="cuda") if active is None else active
    z = logits.double()
    order = torch.where(z.isnan(), float("-inf"), z)
    chosen = order.sort(dim=1, descending=True, stable=True).indices[:, :top]
    p = z.softmax(1)
    w = p.gather(1, chosen)
    if renormalize:
        w = w / w.sum(1, keepdim=True)
    flat = torch.where(on[:, None], chosen, experts).reshape(-1)
    places = torch.empty_like(flat)
    places[flat.sort(stable=True).indices] = torch.arange(flat.numel(), device="cuda")
    counts = torch.bincount(flat, minlength=experts + 1)[:experts]
    n = int(on.sum())
    balance = experts * (counts.double() / max(1, n * top) * p[on].sum(0) / max(1, n)).sum()
    chosen, slots = (torch.where(on[:, None], t, -1) for t in (chosen, places.view(rows, top)))
    return chosen, torch.where(on[:, None], scale * w, 0), slots, counts.cumsum(0), balance


def _tolerance(logits, rows=0):
    z = logits.double()
    # from 110 on a probability is less than 1e-37, and zero in fp32
    apart = (z.amax(1, keepdim=True) - z).nan_to_num(0, posinf=0).clamp(max=110).amax() if z.numel() else 0
    return (4 * float(apart) + 64 + 64 * (rows // 65536 + 1) + 16) * U


def _check(got, logits, top, active=None, renormalize=True, scale=1.0):
    chosen, weights, slots, ends, balance = got
    want = _exact(logits, top, active, renormalize, scale)
    assert torch.equal(chosen, want[0].int()) and torch.equal(slots, want[2].int()) and torch.equal(ends, want[3].int())
    P = _tolerance(logits, logits.shape[0])
    close("weights", weights, want[1], 2 * P * want[1].abs() + 1e-37)
    close("balance", balance, want[4], 2 * P * want[4].abs())
    return want


def _gradient(logits, chosen, counts, taking, dweights, dbalance, renormalize, scale):
    """The gradient in 64 bits by automatic differentiation, and a bound of what rounding adds."""
    experts, top = logits.shape[1], chosen.shape[1]
    z = logits.double().requires_grad_()
    on = chosen[:, 0] >= 0
    p = z.softmax(1)
    at = chosen.clamp(min=0).long()
    w = p.gather(1, at)
    if renormalize:
        w = w / w.sum(1, keepdim=True)
    value = 0.0
    u = torch.zeros(experts, dtype=torch.float64, device="cuda")
    if dweights is not None:
        value = value + (scale * w * dweights.double())[on].sum()
    if dbalance is not None:
        u = dbalance.double() * experts * counts.double() / max(1, taking * top) / max(1, taking)
        value = value + (p[on] * u).sum()
    grad = torch.autograd.grad(value, z)[0]
    grad = torch.where(on[:, None], grad, 0)
    P = _tolerance(logits)
    p, w = p.detach(), w.detach()
    d = 0 * w if dweights is None else (scale * dweights.double()).abs()
    g = u.abs().expand_as(p).clone()
    bound = torch.zeros_like(p)
    if renormalize:
        bound.scatter_add_(1, at, w * (d + (w * d).sum(1, keepdim=True)))
    else:
        g.scatter_add_(1, at, d)
    bound = bound + p * (g + (p * g).sum(1, keepdim=True))
    # renormalised, the others' gradient is exactly zero; the reference takes it as a difference of equal numbers,
    # which leaves some roundings of 2^-53 of p times the sizes that cancel
    return grad, 4 * (P + (16 + 2 * top) * U) * bound + 2.0 ** -48 * p * (u.abs().amax() + d.sum(1, keepdim=True)) + 1e-37


def _check_gradient(got, logits, chosen, ends, dweights, dbalance, renormalize, scale, dtype):
    counts = ends.diff(prepend=ends.new_zeros(1))
    want, bound = _gradient(logits, chosen, counts, int(ends[-1]) // chosen.shape[1], dweights, dbalance, renormalize, scale)
    close("dlogits", got, want, rounded(want, bound, dtype))


# rows, experts, top: one of each to many; sizes around those at which a row gets more lanes, a block more
# rows, or the launch more blocks; odd ones
SIZES = [(1, 1, 1), (1, 2, 2), (3, 5, 3), (63, 8, 2), (64, 8, 2), (65, 8, 1), (200, 60, 4), (129, 64, 6), (1000, 65, 8),
         (77, 128, 64), (500, 129, 5), (333, 255, 8), (400, 256, 8), (70, 257, 7), (900, 512, 8), (130, 513, 31), (300, 400, 40), (90, 1000, 3), (65, 1025, 4), (30, 4097, 64),
         (66, 8192, 8), (5000, 16, 2), (20001, 7, 3), (70001, 12, 2), (131073, 4, 1)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,experts,top", SIZES)
def test_route_and_gradient(rows, experts, top, dtype):
    log(f"case: route {rows} x {experts} top {top} {dtype}")
    logits = _logits(rows, experts, dtype, seed=rows)   # bf16: many equal scores
    g = generator(1)
    dweights = torch.randn((rows, top), generator=g, device="cuda")
    dbalance = torch.full((), 0.7, device="cuda")
    for renormalize, scale in ((True, 1.0), (False, 2.5)):
        got = tm.expert_route(logits, top, renormalize=renormalize, scale=scale)
        _check(got, logits, top, None, renormalize, scale)
        for dw, db in ((dweights, dbalance), (dweights, None), (None, dbalance)):
            back = tm.expert_route_backward(logits, got[0], got[3], dw, db, renormalize=renormalize, scale=scale)
            _check_gradient(back, logits, got[0], got[3], dw, db, renormalize, scale, dtype)
        again = tm.expert_route(logits, top, renormalize=renormalize, scale=scale)
        assert all(torch.equal(a, b) for a, b in zip(got, again))
    assert not tm.expert_route_backward(logits, got[0], got[3]).any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,experts,top", [(1, 4, 2), (130, 8, 2), (900, 60, 4), (300, 700, 9), (70, 3000, 4)])
def test_rows_that_take_no_part_are_not_read(rows, experts, top, dtype):
    log(f"case: route, masked rows {rows} x {experts} top {top} {dtype}")
    logits = _logits(rows, experts, dtype, seed=2)
    active = torch.rand(rows, generator=generator(3), device="cuda") < 0.6
    clean = logits.clone()
    logits[~active] = float("nan")
    for mask in (active, torch.zeros_like(active), torch.ones_like(active)):
        source = logits if mask is active else clean
        got = tm.expert_route(source, top, mask)
        _check(got, torch.where(mask[:, None], source, 0), top, mask)
        dw = torch.where(mask[:, None], torch.ones((rows, top), device="cuda"), float("nan"))
        back = tm.expert_route_backward(source, got[0], got[3], dw, torch.ones((), device="cuda"))
        assert torch.isfinite(back).all() and not back[~mask].any()
    none = tm.expert_route(clean, top, torch.zeros_like(active))
    assert float(none[4]) == 0.0 and not none[3].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("experts", [6, 60, 200, 300, 2000])
def test_ties_and_masked_experts(experts, dtype):
    """Equal scores go to the lowest expert; -inf and the type's lowest value have no share; rows that are not
    numbers have choices all the same and leave the other rows alone."""
    rows, top = 100, 5
    logits = _logits(rows, experts, dtype, seed=4).round()
    low = torch.finfo(DT[dtype]).min
    logits[1] = 3.0
    logits[2] = -0.0
    logits[2, experts // 2] = 0.0
    logits[3, 3:] = float("-inf")       # fewer finite scores than choices
    logits[4, 2:] = low
    logits[5] = low
    got = tm.expert_route(logits, top)
    _check(got, logits, top)
    assert got[0][1].tolist() == list(range(top)) and got[0][2].tolist() == list(range(top))
    dw = torch.randn((rows, top), generator=generator(5), device="cuda")
    back = tm.expert_route_backward(logits, got[0], got[3], dw, torch.ones((), device="cuda"))
    _check_gradient(back, logits, got[0], got[3], dw, torch.ones((), device="cuda"), True, 1.0, dtype)
    bad = logits.clone()
    bad[7, 1], bad[8] = float("nan"), float("-inf")
    bad[9, 0] = float("inf")
    odd = [7, 8, 9]
    rest = [r for r in range(rows) if r not in odd]
    for renormalize in (True, False):
        ref = tm.expert_route(logits, top, renormalize=renormalize)
        chosen, weights, slots, ends, balance = tm.expert_route(bad, top, renormalize=renormalize)
        assert torch.equal(chosen[rest], ref[0][rest]) and torch.equal(weights[rest], ref[1][rest])
        assert weights[odd].isnan().all() and balance.isnan()
        assert chosen[8].tolist() == list(range(top)) and int(chosen[9, 0]) == 0 and 1 not in chosen[7].tolist()
        assert sorted(slots.reshape(-1).tolist()) == list(range(rows * top)) and int(ends[-1]) == rows * top
        back = tm.expert_route_backward(bad, chosen, ends, dw, renormalize=renormalize)
        assert torch.isfinite(back[rest]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("experts", [7, 61, 250, 999, 2001])
def test_strides_and_in_place(experts, dtype):
    rows, top = 150, 4
    logits = _logits(rows, experts, dtype, seed=6)
    ref = tm.expert_route(logits, top)
    dw = torch.randn((rows, top), generator=generator(7), device="cuda")
    db = torch.ones((), device="cuda")
    back = tm.expert_route_backward(logits, ref[0], ref[3], dw, db)
    for other in (spread(logits, 13, 5), logits.t().contiguous().t()):
        assert all(torch.equal(a, b) for a, b in zip(ref, tm.expert_route(other, top)))
        assert torch.equal(back, tm.expert_route_backward(other, ref[0], ref[3], dw.t().contiguous().t(), db))
    own = logits.clone()
    assert tm.lib().tm_expert_route_backward(own.data_ptr(), experts, ref[0].data_ptr(), ref[3].data_ptr(), dw.data_ptr(),
                                             db.data_ptr(), 1, 1.0, own.data_ptr(), experts, rows, experts, top,
                                             0 if dtype == "bf16" else 1, torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(own, back)
    away = far(logits[:20], 1 << 28)
    assert all(torch.equal(a, b) for a, b in zip(tm.expert_route(logits[:20], top), tm.expert_route(away, top)))
    assert torch.equal(tm.expert_route_backward(logits[:20], ref[0][:20], ref[3], dw[:20]),
                       tm.expert_route_backward(away, ref[0][:20], ref[3], dw[:20]))


def test_choices_that_are_no_experts_are_left_out():
    """Choices of the caller's own: past the experts, negative, the same one twice."""
    logits = _logits(4, 20, "f32", seed=8)
    chosen = torch.tensor([[3, 19, 20], [5, 5, 2], [7, -1, 2 ** 31 - 1], [-5, 3, 4]], dtype=torch.int32, device="cuda")
    ends = torch.arange(1, 21, dtype=torch.int32, device="cuda")
    dw = torch.tensor([[1.0, 2.0, 3.0], [0.5, -1.0, 2.0], [1.0, 5.0, 7.0], [1.0, 1.0, 1.0]], device="cuda")
    for renormalize in (True, False):
        got = tm.expert_route_backward(logits, chosen, ends, dw, renormalize=renormalize)
        z = logits.double().requires_grad_()
        p = z.softmax(1)
        value = 0.0
        for r, kept in ((0, [0, 1]), (1, [0, 1, 2]), (2, [0])):
            w = p[r, chosen[r, kept].long()]
            if renormalize:
                w = w / w.sum()
            value = value + (w * dw[r, kept].double()).sum()
        want = torch.autograd.grad(value, z)[0]
        close("dlogits", got, want, 400 * U * (want.abs() + 8 * p.detach()) + 40 * U)


def test_autograd_and_differences():
    logits = _logits(40, 12, "f32", seed=9)
    g = torch.randn((40, 3), generator=generator(10), device="cuda")
    for renormalize in (True, False):
        leaf = logits.clone().requires_grad_()
        weights, balance, chosen, slots, ends = ops.expert_route(leaf, 3, renormalize=renormalize, scale=1.5)
        assert not chosen.requires_grad and not slots.requires_grad and not ends.requires_grad
        ((weights * g).sum() + 2.0 * balance).backward()

        def value(z):
            p = z.softmax(1)
            w = p.gather(1, chosen.long())
            if renormalize:
                w = w / w.sum(1, keepdim=True)
            c = ends.diff(prepend=ends.new_zeros(1)).double()
            return (1.5 * w * g.double()).sum() + 2.0 * 12 * (c / 120 * p.mean(0)).sum()

        z = logits.double()
        for r, e in ((0, 0), (3, int(chosen[3, 0])), (17, 5), (39, 11)):
            step = torch.zeros_like(z)
            step[r, e] = 1e-5
            diff = float(value(z + step) - value(z - step)) / 2e-5
            assert abs(float(leaf.grad[r, e]) - diff) <= 1e-5 * (1 + abs(diff))
        alone = logits.clone().requires_grad_()
        out = ops.expert_route(alone, 3, renormalize=renormalize)
        out[1].backward()
        assert torch.equal(alone.grad, tm.expert_route_backward(logits, chosen, ends, None, torch.ones((), device="cuda"),
                                                                renormalize=renormalize))


def test_more_rows_than_16_bits_of_counts_hold_eight_times():
    log("case: route 8400000 x 4")
    logits = _logits(8400000, 4, "f32", seed=11)
    _check(tm.expert_route(logits, 1), logits, 1)


def test_equal_scores_everywhere():
    """A router that starts at zero: every row takes the first experts."""
    for experts in (5, 64, 256, 300, 1000, 1500):
        logits = torch.zeros((130, experts), device="cuda")
        got = tm.expert_route(logits, 4)
        _check(got, logits, 4)
        assert (got[0] == torch.arange(4, device="cuda")).all() and abs(float(got[4]) - 1.0) < 1e-5


def test_ends_of_other_strides():
    logits = _logits(100, 6, "f32", seed=12)
    chosen, _, slots, ends, _ = tm.expert_route(logits, 2)
    apart = torch.stack([ends, 0 * ends], 1)[:, 0]
    x = torch.randn((100, 33), generator=generator(13), device="cuda")
    assert torch.equal(tm.expert_gather(x, slots, ends), tm.expert_gather(x, slots, apart))
    assert torch.equal(tm.expert_route_backward(logits, chosen, ends, None, torch.ones((), device="cuda")),
                       tm.expert_route_backward(logits, chosen, apart, None, torch.ones((), device="cuda")))


def test_no_rows_and_refusals():
    logits = _logits(6, 5, "f32")
    chosen, weights, slots, ends, balance = tm.expert_route(logits[:0], 2)
    assert chosen.shape == weights.shape == slots.shape == (0, 2) and not ends.any() and float(balance) == 0.0
    assert tm.expert_route_backward(logits[:0], chosen, ends).shape == (0, 5)
    ok = tm.expert_route(logits, 2)
    for call in (lambda: tm.expert_route(logits.half(), 2), lambda: tm.expert_route(logits[0], 2),
                 lambda: tm.expert_route(logits.cpu(), 2), lambda: tm.expert_route(logits, 2, torch.ones(6, device="cuda")),
                 lambda: tm.expert_route(logits, 2, torch.ones(5, dtype=torch.bool, device="cuda")),
                 lambda: tm.expert_route_backward(logits, ok[0].long(), ok[3]),
                 lambda: tm.expert_route_backward(logits, ok[0][:3], ok[3]),
                 lambda: tm.expert_route_backward(logits, ok[0], ok[3][:2]),
                 lambda: tm.expert_route_backward(logits, ok[0], ok[3], ok[1][:, :1]),
                 lambda: tm.expert_route_backward(logits, ok[0], ok[3], None, 1.0 + ok[1][0])):
        with pytest.raises((ValueError, AttributeError)):
            call()
    for bad in (dict(top=0), dict(top=6), dict(top=-1), dict(top=10 ** 9), dict(top=2, scale=float("nan")),
                dict(top=2, scale=float("inf"))):
        with pytest.raises(tm.TurboMuonError) as e:
            tm.expert_route(logits, **bad)
        assert e.value.status == tm.TM_ERR_INVALID_ARG
    with pytest.raises(tm.TurboMuonError):
        tm.expert_route(_logits(4, 200, "f32"), 65)


# rows, experts, top, most rows that a block goes through: many blocks, some of several runs of 64 rows, at every
# number of lanes a row
MANY = [(20001, 300, 8, 64), (33001, 256, 8, 64), (60001, 400, 4, 128), (60001, 700, 3, 192), (9001, 1500, 2, 64),
        (30001, 1500, 2, 192), (9001, 8000, 2, 128)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,experts,top,run", MANY)
def test_many_rows_and_many_experts(rows, experts, top, run, dtype):
    """Masked rows among them.  A probability is off by P of itself, as above without the additions; the balance is a
    sum of them over at most `run` rows, the groups and waves of a block (16 more), and 64-bit sums."""
    log(f"case: route many {rows} x {experts} top {top} {dtype}")
    logits = _logits(rows, experts, dtype, seed=rows + experts)
    g = generator(4)
    active = torch.rand(rows, generator=g, device="cuda") < 0.8
    clean = logits.clone()
    logits[~active] = float("nan")
    got = tm.expert_route(logits, top, active)
    want = _exact(torch.where(active[:, None], clean, 0), top, active, True, 1.0)
    assert torch.equal(got[0], want[0].int()) and torch.equal(got[2], want[2].int()) and torch.equal(got[3], want[3].int())
    z = clean.double()
    P = (4 * float((z.amax(1, keepdim=True) - z).clamp(max=110).amax()) + 64) * U
    close("weights", got[1], want[1], 2 * P * want[1].abs() + 1e-37)
    close("balance", got[4], want[4], (P + (run + 16 + 2) * U) * want[4].abs())
    again = tm.expert_route(logits, top, active)
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    dw = torch.randn((rows, top), generator=g, device="cuda")
    db = torch.full((), 0.7, device="cuda")
    back = tm.expert_route_backward(logits, got[0], got[3], dw, db)
    assert not back[~active].any()
    _check_gradient(back, clean, got[0], got[3], dw, db, True, 1.0, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,experts", [(20, 8), (300, 60), (150, 300), (90, 1500)])
def test_plus_infinity(rows, experts, dtype):
    """It is chosen first and its row's weights are not a number; the other rows are as without it."""
    log(f"case: route, +inf in {rows} x {experts} {dtype}")
    logits = _logits(rows, experts, dtype, seed=5)
    logits[3, experts - 2] = float("inf")
    logits[7, 1] = logits[7, 4] = float("inf")
    rest = torch.ones(rows, dtype=torch.bool, device="cuda")
    rest[3] = rest[7] = False
    chosen, weights, slots, ends, balance = tm.expert_route(logits, 3)
    want = _exact(logits, 3, None, True, 1.0)
    assert torch.equal(chosen, want[0].int()) and torch.equal(slots, want[2].int()) and torch.equal(ends, want[3].int())
    assert weights[~rest].isnan().all() and balance.isnan()
    P = _tolerance(logits[rest], rows)
    close("weights", weights[rest], want[1][rest], 2 * P * want[1][rest].abs() + 1e-37)
