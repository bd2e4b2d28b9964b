"""Policy loss on the GPU against its definition in 64 bits.

Tolerances (u = 2^-24): the sum of exponentials is a tree of at most
V / 2048 + 48 additions of terms that are off by their argument's rounding
(2 u of at most Z = max|l| / tau, and of log2 e more) and an ulp, so a log
probability is off by at most D = (V / 2048 + 64 + 8 Z) u.  Ratios follow by
exp: relative D plus a few u of the exponent.  Gradients are a product with
slope; bf16 gradients are rounded once, 2^-8 of themselves.
"""
import pytest

from gpu_helpers import log

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from paper_2512_04632_amd import _lib as tm, ops  # noqa: E402

U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
LOW, HIGH, KL, TAU = 0.2, 0.28, 0.05, 0.8


def _inputs(rows, vocab, dtype, seed=0, masked=0.3, tau=TAU):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def randn(*s):
        return torch.randn(s, generator=g, device="cuda")

    logits = (randn(rows, vocab) * 2).to(DT[dtype])
    targets = torch.randint(vocab, (rows,), generator=g, device="cuda")
    logits[torch.arange(rows, device="cuda"), targets] = (randn(rows) + 8).to(DT[dtype])
    z = logits.double() / tau
    logp = (z.gather(1, targets[:, None])[:, 0] - z.logsumexp(1)).float()
    # ratios off the clipping bounds, where rounding would decide the gradient
    ratio = (0.3 * randn(rows)).exp()
    for bound in (1 - LOW, 1 + HIGH):
        ratio = torch.where((ratio - bound).abs() < 0.01, ratio + 0.03, ratio)
    weights = torch.rand(rows, generator=g, device="cuda") + 0.1
    weights[torch.rand(rows, generator=g, device="cuda") < masked] = 0.0
    return dict(logits=logits, targets=targets, old_logp=logp - ratio.log(), advantages=randn(rows),
                weights=weights, ref_logp=logp + 0.3 * randn(rows))


def _exact(s, kl=KL, tau=TAU, low=LOW, high=HIGH):
    """(loss, logp, lse, slope, gradient) in 64 bits, and the rows' shares."""
    z = s["logits"].double() / tau
    rows = z.shape[0]
    on = (s["weights"] != 0) & (s["targets"] >= 0)
    y = s["targets"].clamp(min=0)
    lse = z.logsumexp(1)
    logp = z.gather(1, y[:, None])[:, 0] - lse
    A, m = s["advantages"].double(), s["weights"].double()
    r = (logp - s["old_logp"].double()).exp()
    first, second = r * A, r.clamp(1 - low, 1 + high) * A
    value, slope = -torch.minimum(first, second), torch.where(first <= second, -first, 0 * first)
    if s["ref_logp"] is not None:
        gap = s["ref_logp"].double() - logp
        value, slope = value + kl * (gap.exp() - gap - 1), slope + kl * (1 - gap.exp())
    value, slope = torch.where(on, m * value, 0), torch.where(on, m * slope, 0)
    grad = -(z - lse[:, None]).exp()
    grad[torch.arange(rows, device="cuda"), y] += 1
    grad = torch.where(on[:, None], grad * (slope / tau)[:, None], 0)
    return value.sum(), torch.where(on, logp, 0), torch.where(on, lse, 0), slope, grad


def _close(name, got, want, bound):
    off = (got.double() - want).abs()
    bad = ~(off <= bound)
    assert not bad.any(), (name, int(bad.sum()), float(off.max()), float((off / bound).max()))


def _tolerances(s, vocab, kl=KL, tau=TAU):
    z = float(s["logits"].double().abs().max()) / tau
    D = (vocab / 2048 + 64 + 8 * z) * U
    logp = _exact(s, kl, tau)[1]
    gap = 0 if s["ref_logp"] is None else (s["ref_logp"].double() - logp)
    off = D + 8 * U * (1 + (logp - s["old_logp"].double()).abs())
    r = (logp - s["old_logp"].double()).exp()
    q = gap.exp() if s["ref_logp"] is not None else 0 * r
    terms = s["weights"].double() * (r * s["advantages"].double().abs() * 2 + kl * (q + abs(gap) + 1)) * (off + 8 * U)
    return D, terms * 1.01 + 1e-38


def _check(s, got, dtype, kl=KL, tau=TAU, grad=None):
    loss, logp, lse, slope = got
    rows, vocab = s["logits"].shape
    wl, wp, we, ws, wg = _exact(s, kl, tau)
    D, terms = _tolerances(s, vocab, kl, tau)
    _close("logp", logp, wp, D)
    if lse is not None:
        _close("lse", lse, we, D + U * we.abs())
        _close("slope", slope, ws, terms)
    _close("loss", loss, wl, terms.sum() + U * wl.abs())
    if grad is not None:
        p = wg.abs()
        bound = p * (D + 16 * U) * 2 + (terms / tau)[:, None] * (p / (ws.abs()[:, None] / tau + 1e-300)) \
            + (20 * U + D) * (ws.abs() / tau)[:, None] * (torch.arange(vocab, device="cuda")[None] == s["targets"][:, None])
        _close("grad", grad, wg, bound + (2.0 ** -8 if dtype == "bf16" else U) * (p + bound) + 1e-38)


# one row to many; one entry, vocabularies below and above the sizes at which rows are split,
# held in registers, or given more threads; odd ones
SIZES = [(1, 1), (3, 2), (5, 17), (1, 1000), (64, 4099), (700, 517), (1, 8192), (2, 50257), (16, 50257), (65, 8209),
         (200, 20001), (511, 9000), (513, 9000), (600, 33001), (520, 66000), (3, 131072), (1, 300001), (515, 131080)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab", SIZES)
def test_value_and_gradient(rows, vocab, dtype):
    log(f"case: policy loss {rows} x {vocab} {dtype}")
    s = _inputs(rows, vocab, dtype, seed=rows)
    kw = dict(clip_low=LOW, clip_high=HIGH, kl=KL, temperature=TAU)
    got = tm.policy_loss(**s, **kw)
    _check(s, got, dtype)
    grad = tm.policy_loss_backward(s["logits"], s["targets"], got[2], got[3], temperature=TAU)
    _check(s, got, dtype, grad=grad)
    loss, logp, both = tm.policy_loss_with_grad(**s, **kw)
    assert torch.equal(loss, got[0]) and torch.equal(logp, got[1])
    _check(s, got, dtype, grad=both)
    again = tm.policy_loss_with_grad(**s, **kw)
    assert all(torch.equal(a, b) for a, b in zip((loss, logp, both), again))


@pytest.mark.parametrize("rows", [6, 600])
def test_without_reference_and_at_other_temperatures(rows):
    for tau in (1.0, 0.25, 3.0):
        s = _inputs(rows, 9001, "f32", seed=3, tau=tau)
        s["ref_logp"] = None
        got = tm.policy_loss(**s, clip_low=LOW, clip_high=HIGH, kl=0.5, temperature=tau)
        grad = tm.policy_loss_with_grad(**s, clip_low=LOW, clip_high=HIGH, kl=0.5, temperature=tau)[2]
        _check(s, got, "f32", kl=0.0, tau=tau, grad=grad)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab", [(9, 700), (9, 9000), (600, 700), (600, 20000)])
def test_masked_rows_are_not_read(rows, vocab, dtype):
    """NaN and Inf in rows of weight 0 or with a negative target, and in their other inputs."""
    log(f"case: policy loss, masked rows {rows} x {vocab} {dtype}")
    s = _inputs(rows, vocab, dtype, seed=5, masked=0.0)
    s["weights"][1] = 0.0
    s["targets"][4] = -100
    kw = dict(clip_low=LOW, clip_high=HIGH, kl=KL, temperature=TAU)
    off = [1, 4]
    for t in (s["logits"], s["old_logp"], s["advantages"], s["ref_logp"]):
        t[1], t[4] = float("nan"), float("inf")
    loss, logp, lse, slope = tm.policy_loss(**s, **kw)
    one = tm.policy_loss_with_grad(**s, **kw)
    two = tm.policy_loss_backward(s["logits"], s["targets"], lse, slope, temperature=TAU)
    assert torch.isfinite(loss) and torch.isfinite(one[2]).all()
    for t in (logp, lse, slope, one[2], two):
        assert not t[off].any()
    rest = torch.ones(rows, dtype=torch.bool, device="cuda")
    rest[off] = False
    part = {k: v[rest] for k, v in s.items()}
    want = _exact(part)
    assert abs(float(loss) - float(want[0])) <= float(_tolerances(part, vocab)[1].sum()) + U * abs(float(want[0]))
    # nothing but masked rows
    s["weights"].zero_()
    loss, logp, grad = tm.policy_loss_with_grad(**s, **kw)
    assert float(loss) == 0.0 and not logp.any() and not grad.any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab", [(4, 600), (4, 20000), (600, 20000)])
def test_masked_vocabulary(rows, vocab, dtype):
    """Entries of -inf or of the type's lowest value have no share and no gradient; a row of
    nothing but -inf gives NaN and leaves the others alone."""
    s = _inputs(rows, vocab, dtype, seed=6, masked=0.0)
    kw = dict(clip_low=LOW, clip_high=HIGH, kl=KL, temperature=TAU)
    low = torch.finfo(DT[dtype]).min
    half = torch.arange(vocab, device="cuda") % 2 == 1
    ref = tm.policy_loss_with_grad(**s, **kw)
    for value in (float("-inf"), low):
        t = dict(s, logits=s["logits"].clone())
        hidden = half[None] & (torch.arange(vocab, device="cuda")[None] != s["targets"][:, None])
        t["logits"][hidden] = value
        t["logits"][0] = s["logits"][0]
        hidden[0] = False
        got = tm.policy_loss_with_grad(**t, **kw)
        lse, slope = tm.policy_loss(**t, **kw)[2:]
        back = tm.policy_loss_backward(t["logits"], t["targets"], lse, slope, temperature=TAU)
        for grad in (got[2], back):
            assert torch.isfinite(grad).all() and not grad[hidden].any()
        assert torch.equal(got[2][0], ref[2][0]) and torch.equal(got[1][0], ref[1][0])
    t["logits"][2] = float("-inf")
    loss, logp, grad = tm.policy_loss_with_grad(**t, **kw)
    assert logp[2].isnan() and loss.isnan() and torch.isfinite(logp[[0, 1, 3]]).all()
    assert torch.isfinite(grad[[0, 1, 3]]).all() and grad[2].isnan().all()
    # a row of nothing but the lowest value: every entry the same
    t["logits"][2] = low
    loss, logp, grad = tm.policy_loss_with_grad(**t, **dict(kw, temperature=1.0))
    assert abs(float(logp[2]) + float(torch.tensor(float(vocab)).log())) < 1e-4 or vocab >= 8192
    assert not logp[2].isnan()
    t["logits"][1, 5] = float("nan")
    loss, logp, grad = tm.policy_loss_with_grad(**t, **kw)
    assert logp[1].isnan() and loss.isnan() and torch.isfinite(logp[[0, 3]]).all()


def test_target_past_the_vocabulary_is_nan():
    for rows, vocab in ((4, 100), (4, 20000)):
        s = _inputs(rows, vocab, "f32", masked=0.0)
        s["targets"][2] = vocab
        loss, logp, grad = tm.policy_loss_with_grad(**s)
        assert loss.isnan() and logp[2].isnan() and grad[2].isnan().all()
        assert torch.isfinite(logp[[0, 1, 3]]).all() and torch.isfinite(grad[[0, 1, 3]]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab", [(7, 9001), (600, 9001), (600, 40001)])
def test_strides_and_in_place(rows, vocab, dtype):
    s = _inputs(rows, vocab, dtype, seed=8)
    ref = tm.policy_loss_with_grad(**s, kl=KL)
    wide = torch.zeros((rows, vocab + 13), dtype=DT[dtype], device="cuda")
    wide[:, 5:5 + vocab] = s["logits"]
    cut = dict(s, logits=wide[:, 5:5 + vocab])
    got = tm.policy_loss_with_grad(**cut, kl=KL)
    # other alignment, other order of the same sums
    assert torch.allclose(got[1], ref[1], rtol=0, atol=1e-5)
    assert torch.allclose(got[2].float(), ref[2].float(), rtol=2.0 ** -7, atol=1e-7)
    loss, logp = torch.empty((), device="cuda"), torch.empty(rows, device="cuda")
    st = tm.lib().tm_policy_loss(wide.data_ptr() + 5 * wide.element_size(), vocab + 13, s["targets"].data_ptr(),
                                 s["old_logp"].data_ptr(), s["advantages"].data_ptr(), s["weights"].data_ptr(),
                                 s["ref_logp"].data_ptr(), 0.2, 0.2, KL, 1.0, loss.data_ptr(), logp.data_ptr(), None,
                                 None, wide.data_ptr() + 5 * wide.element_size(), vocab + 13, rows, vocab,
                                 0 if dtype == "bf16" else 1, torch.cuda.current_stream().cuda_stream)
    assert st == 0 and torch.equal(wide[:, 5:5 + vocab], got[2])
    assert not wide[:, :5].any() and not wide[:, 5 + vocab:].any()


def test_offsets_past_32_bits():
    rows, vocab = 20, 131072
    stride = 1 << 28                        # 20 rows, 5.4e9 elements from end to end
    s = _inputs(rows, vocab, "bf16", seed=9)
    ref = tm.policy_loss_with_grad(**s, kl=KL)
    store = torch.empty(stride * (rows - 1) + vocab, dtype=torch.bfloat16, device="cuda")
    far = store.as_strided((rows, vocab), (stride, 1))
    far.copy_(s["logits"])
    got = tm.policy_loss_with_grad(**dict(s, logits=far), kl=KL)
    assert all(torch.equal(a, b) for a, b in zip(ref, got))


def test_autograd_scales_by_the_upstream_gradient():
    s = _inputs(40, 3001, "f32", seed=10)
    logits = s["logits"].clone().requires_grad_()
    loss, logp = ops.policy_loss(logits, s["targets"], s["old_logp"], s["advantages"], s["weights"], s["ref_logp"],
                                 LOW, HIGH, KL, TAU)
    assert not logp.requires_grad
    (loss * 3.5).backward()
    _check(s, tm.policy_loss(**s, clip_low=LOW, clip_high=HIGH, kl=KL, temperature=TAU), "f32", grad=logits.grad / 3.5)


def test_gradient_against_differences():
    s = _inputs(6, 50, "f32", seed=11, masked=0.0)
    grad = tm.policy_loss_with_grad(**s, clip_low=LOW, clip_high=HIGH, kl=KL, temperature=TAU)[2]
    for r in range(6):
        for v in (int(s["targets"][r]), 3, 49):
            t = dict(s, logits=s["logits"].double())
            t["logits"][r, v] += 1e-5
            up = float(_exact(t)[0])
            t["logits"][r, v] -= 2e-5
            diff = (up - float(_exact(t)[0])) / 2e-5
            assert abs(float(grad[r, v]) - diff) <= 1e-5 * (1 + abs(diff))


def test_no_rows_and_refusals():
    s = _inputs(4, 64, "f32")
    none = {k: v[:0] for k, v in s.items()}
    loss, logp, grad = tm.policy_loss_with_grad(**none)
    assert float(loss) == 0.0 and logp.shape == (0,) and grad.shape == (0, 64)
    for bad in (dict(s, logits=s["logits"].half()), dict(s, logits=s["logits"][0]), dict(s, targets=s["targets"].int()),
                dict(s, weights=s["weights"][:2]), dict(s, old_logp=s["old_logp"].double()),
                dict(s, ref_logp=s["ref_logp"].cpu()), dict(s, logits=s["logits"].cpu())):
        with pytest.raises(ValueError):
            tm.policy_loss(**bad)
    for bad in (dict(temperature=0.0), dict(temperature=float("nan")), dict(temperature=float("inf")),
                dict(clip_low=-0.1), dict(clip_low=1.5), dict(clip_high=-1.0), dict(kl=-1.0), dict(kl=float("nan"))):
        with pytest.raises(tm.TurboMuonError) as e:
            tm.policy_loss(**s, **bad)
        assert e.value.status == tm.TM_ERR_INVALID_ARG


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab", [(1, 32768), (4, 40001), (16, 33333), (20, 70001), (32, 131072), (33, 131072)])
def test_few_long_rows(rows, vocab, dtype):
    """Rows that are cut into parts: sizes, masks, strides."""
    log(f"case: policy loss, few long rows {rows} x {vocab} {dtype}")
    test_value_and_gradient(rows, vocab, dtype)
    if rows >= 20:
        test_masked_rows_are_not_read(rows, vocab, dtype)
    test_masked_vocabulary(max(rows, 4), vocab, dtype)
    test_strides_and_in_place(rows, vocab, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab", [(4, 600), (4, 20000), (4, 40001), (16, 32768), (32, 70001), (33, 70001),
                                        (40, 32001)])
def test_gradient_of_logits_of_large_size(rows, vocab, dtype):
    """However the rows are run, the gradient depends on the distances of the logits from their maximum
    alone: rows of nothing but the type's lowest value, and logits with a common offset of 10^4.

    With Z the largest distance over tau of a row, a probability is off by 2 (D + 16 u) of itself, where D =
    (V / 2048 + 64 + 8 Z) u (see above), the target's 1 - p by a rounding more; the slope is policy_loss's own."""
    log(f"case: policy loss, gradient of large logits {rows} x {vocab} {dtype}")
    s = _inputs(rows, vocab, dtype, seed=12, masked=0.0)
    s["logits"] = (s["logits"].double() + 1e4).to(DT[dtype])
    s["logits"][2] = torch.finfo(DT[dtype]).min
    at = torch.arange(rows, device="cuda")
    z = s["logits"].double() / TAU
    z = z - z.amax(1, keepdim=True)   # 64 bits hold no log V beside the lowest value either
    logp = z[at, s["targets"]] - z.logsumexp(1)
    s["old_logp"], s["ref_logp"] = (logp - 0.05).float(), (logp + 0.2).float()
    kw = dict(clip_low=LOW, clip_high=HIGH, kl=KL, temperature=TAU)
    slope = tm.policy_loss(**s, **kw)[3].double()
    _, got_logp, grad = tm.policy_loss_with_grad(**s, **kw)
    assert (slope != 0).all()
    D = (vocab / 2048 + 64 + 8 * -z.amin(1)) * U
    _close("logp", got_logp, logp, D + 2 * U * logp.abs())
    p = z.softmax(1)
    hit = torch.zeros_like(p)
    hit[at, s["targets"]] = 1
    want = (slope / TAU)[:, None] * (hit - p)
    bound = (slope.abs() / TAU)[:, None] * (2 * p * (D + 16 * U)[:, None] + 4 * U * hit)
    _close("grad", grad, want, bound + (2.0 ** -8 if dtype == "bf16" else 2 * U) * (want.abs() + bound) + 1e-38)
    assert (p[2] == 1 / vocab).all()


@pytest.mark.parametrize("rows,vocab", [(20, 600), (16, 40001)])
def test_kl_term_of_policies_close_to_each_other(rows, vocab):
    """q - log q - 1 and 1 - q keep their digits where q is next to 1.

    The gap ref_logp - logp is exact for values this close, taken from the call's own logp.  Below 1 the terms are
    sums and products of values of one size (alternating ones at most twice their sum): a handful of roundings, and
    those of the factors kl, weight and of the result, under 16 u in all.  From 1 on the differences are off by
    the exponential's last bits, 8 u of q + |gap| + 1."""
    log(f"case: policy loss, KL term of close policies {rows} x {vocab}")
    s = _inputs(rows, vocab, "f32", seed=16, masked=0.0)
    s["advantages"].zero_()
    kw = dict(kl=KL, temperature=TAU)
    logp = tm.policy_loss(**s, **kw)[1]
    gaps = torch.tensor([1e-4, -1e-4, 3e-4, -1e-3, 1e-3, 1e-2, -1e-2, 0.1, -0.1, 0.5, -0.5, 0.99, -0.99, 1.2, -1.2, 4.0,
                         -4.0, 1e-5, 0.0, 2e-2][:rows], device="cuda")
    s["ref_logp"] = logp + gaps
    gap = s["ref_logp"].double() - logp.double()
    m = KL * s["weights"].double()
    want = m * (torch.special.expm1(gap) - gap)
    series = gap * gap * (0.5 + gap / 6 + gap ** 2 / 24 + gap ** 3 / 120)   # where 64 bits cancel too
    want = torch.where(gap.abs() < 1e-2, m * series, want)
    near = gap.abs() < 1
    rough = 8 * U * m * (gap.exp() + gap.abs() + 1)
    slope = tm.policy_loss(**s, **kw)[3]
    wslope = -m * torch.special.expm1(gap)
    _close("slope", slope, wslope, torch.where(near, 16 * U * wslope.abs(), rough))
    loss = torch.stack([tm.policy_loss(**dict(s, weights=torch.where(torch.arange(rows, device="cuda") == r,
                                                                    s["weights"], 0)), **kw)[0] for r in range(rows)])
    _close("loss", loss, want, torch.where(near, 16 * U * want, rough))
