"""Token log probabilities, entropies and alternatives on the GPU against their definition in 64 bits.

Places of alternatives have to be equal.  Tolerances (u = 2^-24): a thread's longest chain of additions has at most
n = min(256, V / 256 + 32) terms (64 threads: 16 of each 32 values in a chain, then V / 2048 such sums), and it moves its
sums to another maximum at most n / 4 times, by a product of three roundings; some thirty joins follow; with Z the largest
distance over tau of a logit from its row's maximum, exponentials and moves are off by 8 Z u more: the sum of
exponentials, and so a logarithm, by D = (2 n + 100 + 8 Z) u.  The sum of e u is off by as much of the sum of sizes."""
import pytest

from gpu_helpers import log

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from op_helpers import DT, U, close, far, generator, rounded, spread  # noqa: E402
from paper_2512_04632_amd import _lib as tm, ops  # noqa: E402

TAU = 0.8


def _inputs(rows, vocab, dtype, seed=0, masked=0.2):
    g = generator(seed)

    def randn(*s):
        return torch.randn(s, generator=g, device="cuda")

    logits = (randn(rows, vocab) * 2).to(DT[dtype])
    targets = torch.randint(vocab, (rows,), generator=g, device="cuda")
    logits[torch.arange(rows, device="cuda"), targets] = (randn(rows) + 8).to(DT[dtype])
    targets[torch.rand(rows, generator=g, device="cuda") < masked] = -100
    return dict(logits=logits, targets=targets, dlogp=randn(rows), dentropy=randn(rows))


def _exact(logits, targets, top, tau):
    on = targets >= 0
    l = logits.double()
    m = l.amax(1)
    z = (l - m[:, None]) / tau
    s = z.exp().sum(1)
    logq = z - s.log()[:, None]
    p = logq.exp()
    logp = logq.gather(1, targets.clamp(min=0)[:, None])[:, 0]
    spread_ = torch.where(p > 0, p * z, 0).sum(1)
    entropy = s.log() - spread_
    ids = logits.float().sort(dim=1, descending=True, stable=True).indices[:, :top]
    likely = logq.gather(1, ids)
    ids = torch.where(logits.gather(1, ids) > float("-inf"), ids, -1)
    return dict(on=on, m=m, s=s, z=z, p=p, logp=logp, entropy=entropy, spread=-spread_, ids=ids, likely=likely)


def _check(s, got, top, tau=TAU):
    logp, entropy, stats, top_logp, top_ids = got
    vocab = s["logits"].shape[1]
    w = _exact(s["logits"], s["targets"], top, tau)
    on = w["on"]
    n = min(256, vocab / 256 + 32)
    D = (2 * n + 100 + 8 * -torch.where(w["z"] > -1e30, w["z"], 0).amin(1).clamp(min=-200)) * U
    for t in (logp, entropy, stats):
        assert not t[~on].any()
    close("logp", logp[on], w["logp"][on], (D + 4 * U * w["logp"].abs())[on])
    close("entropy", entropy[on], w["entropy"][on], (D + 2 * D * w["spread"] + 4 * U * (w["s"].log() + w["spread"]))[on])
    assert torch.equal(stats[on, 0].double(), w["m"][on])
    close("s", stats[on, 1], w["s"][on], (D * w["s"])[on])
    if top:
        assert torch.equal(top_ids, torch.where(on[:, None], w["ids"], -1))
        there = on[:, None] & (w["ids"] >= 0)
        past = there & (w["likely"] < -3e38)      # of the type's lowest value: next to fp32's end, or past it
        assert (top_logp[past] < -2.9e38).all()
        there = there & ~past
        close("top", top_logp[there], w["likely"][there], (D[:, None] + 4 * U * w["likely"].abs())[there])
        assert not top_logp[~on].any() and (top_logp[on[:, None] & (w["ids"] < 0)] == float("-inf")).all()


def _check_gradient(s, got, stats, entropy, dlogp, dentropy, dtype, tau=TAU):
    on = (s["targets"] >= 0)[:, None]
    z = (s["logits"].double() - stats[:, :1].double()) / tau
    logs = stats[:, 1:].double().log()
    p = z.exp() / stats[:, 1:].double()
    g = 0 * logs if dlogp is None else dlogp.double()[:, None]
    h = 0 * logs if dentropy is None else dentropy.double()[:, None]
    H = entropy.double()[:, None]
    zc = z.clamp(min=-140)                 # beyond it p is zero in fp32
    want = -p * (g + h * (zc - logs + H))
    hit = torch.arange(z.shape[1], device="cuda")[None] == s["targets"][:, None]
    want = (want + hit * g) / tau
    size = g.abs() + h.abs() * (zc.abs() + logs.abs() + H.abs())
    off = (p * size * (4 * zc.abs() + 24) * U + hit * g.abs() * 4 * U + 1e-37 * size) / tau
    want, off = torch.where(on, want, 0), torch.where(on, off, 0)
    close("dlogits", got, want, rounded(want, off, dtype))


# one row to many; one entry, vocabularies around the sizes at which a wave holds the row, a row gets more threads or is
# cut into parts; odd ones
SIZES = [(1, 1, 1), (3, 2, 2), (5, 17, 5), (9, 64, 64), (1, 1000, 20), (700, 517, 3), (64, 1024, 1), (33, 1025, 20), (40, 2049, 8),
         (64, 4099, 20), (1, 8192, 64), (2, 50257, 20), (16, 50257, 5), (300, 8209, 20), (260, 24577, 20), (257, 50000, 1),
         (256, 82000, 5), (255, 9000, 7), (600, 33001, 20), (3, 131072, 64), (1, 300001, 20), (270, 131080, 4), (2, 600011, 64), (130, 270001, 5), (100, 110000, 20),
         (200, 6144, 20), (200, 6145, 64), (150, 12288, 64), (150, 12289, 5)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab,top", SIZES)
def test_values_and_gradient(rows, vocab, top, dtype):
    log(f"case: token logp {rows} x {vocab} top {top} {dtype}")
    s = _inputs(rows, vocab, dtype, seed=rows)
    got = tm.token_logp(s["logits"], s["targets"], top, TAU)
    _check(s, got, top)
    bare = tm.token_logp(s["logits"], s["targets"], temperature=TAU)
    assert bare[3] is None and bare[4] is None and all(torch.equal(a, b) for a, b in zip(got[:3], bare[:3]))
    again = tm.token_logp(s["logits"], s["targets"], top, TAU)
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    for g, h in ((s["dlogp"], s["dentropy"]), (s["dlogp"], None), (None, s["dentropy"])):
        back = tm.token_logp_backward(s["logits"], s["targets"], got[2], got[1], g, h, TAU)
        _check_gradient(s, back, got[2], got[1], g, h, dtype)
    assert not tm.token_logp_backward(s["logits"], s["targets"], got[2], got[1], temperature=TAU).any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab", [(6, 900), (6, 20000), (300, 3000), (300, 20000), (6, 300000)])
def test_rows_that_take_no_part_are_not_read(rows, vocab, dtype):
    s = _inputs(rows, vocab, dtype, seed=5, masked=0.0)
    s["targets"][1], s["targets"][4] = -1, -2 ** 62
    ref = tm.token_logp(s["logits"], s["targets"], 5, TAU)
    off = [1, 4]
    s["logits"][off] = float("nan")
    s["dlogp"][off], s["dentropy"][off] = float("nan"), float("inf")
    got = tm.token_logp(s["logits"], s["targets"], 5, TAU)
    assert all(torch.equal(a, b) for a, b in zip(ref, got)) and (got[4][off] == -1).all() and not got[3][off].any()
    back = tm.token_logp_backward(s["logits"], s["targets"], got[2], got[1], s["dlogp"], s["dentropy"], TAU)
    assert torch.isfinite(back).all() and not back[off].any()
    s["logits"][2], s["dlogp"][2], s["dentropy"][2] = float("nan"), 0.0, 0.0   # a gradient of zero: not read
    back = tm.token_logp_backward(s["logits"], s["targets"], got[2], got[1], s["dlogp"], s["dentropy"], TAU)
    assert torch.isfinite(back).all() and not back[2].any()
    s["targets"].fill_(-1)
    got = tm.token_logp(s["logits"], s["targets"], 5, TAU)
    assert not got[0].any() and (got[4] == -1).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab", [(8, 700), (8, 3000), (8, 20000), (300, 20000), (8, 140000)])
def test_masked_vocabulary(rows, vocab, dtype):
    """Entries of -inf are no alternatives, those of the type's lowest value the last ones, in order; neither has
    a share in the entropy or a gradient.  Rows that are not numbers leave the others alone."""
    log(f"case: token logp, masked vocabulary {rows} x {vocab} {dtype}")
    top = 9
    low = torch.finfo(DT[dtype]).min
    s = _inputs(rows, vocab, dtype, seed=6, masked=0.0)
    place = torch.arange(vocab, device="cuda")
    keep = place[None] == s["targets"][:, None]
    keep[0] |= place % 2 == 0
    keep[1] |= place % (vocab // 3) == 1
    for value in (float("-inf"), low):
        t = dict(s, logits=torch.where(keep, s["logits"], torch.tensor(value, dtype=DT[dtype], device="cuda")))
        got = tm.token_logp(t["logits"], t["targets"], top, TAU)
        _check(t, got, top)
        back = tm.token_logp_backward(t["logits"], t["targets"], got[2], got[1], t["dlogp"], t["dentropy"], TAU)
        assert torch.isfinite(back).all() and not back[~keep].any()
    assert (got[1][2:].abs() <= 1e-6).all()
    # nothing but one value; nothing at all; not a number
    t["logits"][2], t["logits"][3], t["logits"][5, 7] = low, float("-inf"), float("nan")
    ref = got
    got = tm.token_logp(t["logits"], t["targets"], top, TAU)
    assert abs(float(got[0][2]) + float(torch.tensor(float(vocab)).log())) < 1e-3
    assert abs(float(got[1][2]) - float(torch.tensor(float(vocab)).log())) < 1e-3
    assert got[4][2].tolist() == list(range(top))
    assert got[0][3].isnan() and got[1][3].isnan() and (got[4][3] == -1).all()
    assert got[0][5].isnan() and got[1][5].isnan() and 7 not in got[4][5].tolist()
    rest = [0, 1, 4, 6, 7]
    assert all(torch.equal(a[rest], b[rest]) for a, b in zip(ref, got))
    back = tm.token_logp_backward(t["logits"], t["targets"], got[2], got[1], t["dlogp"], t["dentropy"], TAU)
    assert torch.isfinite(back[rest]).all() and back[3].isnan().all() and torch.isfinite(back[2]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab", [(3, 900), (3, 2000), (4, 20000), (300, 20000), (300, 130000), (3, 270000)])
def test_alternatives_in_every_order(rows, vocab, dtype):
    """Rows that rise, fall, hold a few values only, or one: what costs a selection most, and ties without number."""
    log(f"case: token logp, orders {rows} x {vocab} {dtype}")
    place = torch.arange(vocab, device="cuda").float()
    rows_of = [place / vocab, -place / vocab, (place * 7919 % 3), 0 * place, (place * 31 % 257).floor(), -(place % 2)]
    logits = torch.stack([rows_of[i % len(rows_of)] for i in range(rows)]).to(DT[dtype])
    s = dict(logits=logits, targets=torch.arange(rows, device="cuda") % vocab)
    for top in (1, 20, 64):
        _check(s, tm.token_logp(logits, s["targets"], top, 1.0), top, tau=1.0)


def test_target_past_the_vocabulary_is_nan():
    for rows, vocab in ((4, 100), (4, 20000), (300, 20000)):
        s = _inputs(rows, vocab, "f32", masked=0.0)
        ref = tm.token_logp(s["logits"], s["targets"], 3)
        s["targets"][2] = vocab
        got = tm.token_logp(s["logits"], s["targets"], 3)
        assert got[0][2].isnan() and torch.equal(got[1], ref[1]) and torch.equal(got[4], ref[4])
        back = tm.token_logp_backward(s["logits"], s["targets"], got[2], got[1], s["dlogp"])
        assert back[2].isnan().all() and torch.isfinite(back[[0, 1, 3]]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab", [(9, 501), (9, 1700), (9, 9001), (300, 9001), (300, 40001)])
def test_strides_and_in_place(rows, vocab, dtype):
    s = _inputs(rows, vocab, dtype, seed=8)
    ref = tm.token_logp(s["logits"], s["targets"], 10)
    back = tm.token_logp_backward(s["logits"], s["targets"], ref[2], ref[1], s["dlogp"], s["dentropy"])
    for other in (spread(s["logits"], 13, 5), s["logits"].t().contiguous().t()):
        got = tm.token_logp(other, s["targets"], 10)
        assert all(torch.equal(a, b) for a, b in zip(ref, got))
        assert torch.equal(back, tm.token_logp_backward(other, s["targets"], ref[2], ref[1], s["dlogp"], s["dentropy"]))
    own = spread(s["logits"], 13, 5)
    assert tm.lib().tm_token_logp_backward(own.data_ptr(), own.stride(0), s["targets"].data_ptr(), ref[2].data_ptr(),
                                           ref[1].data_ptr(), s["dlogp"].data_ptr(), s["dentropy"].data_ptr(), 1.0,
                                           own.data_ptr(), own.stride(0), rows, vocab, 0 if dtype == "bf16" else 1,
                                           torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(own, back)


def test_offsets_past_32_bits():
    for rows, vocab in ((20, 131072), (20, 1500)):
        s = _inputs(rows, vocab, "bf16", seed=9)
        ref = tm.token_logp(s["logits"], s["targets"], 20)
        away = far(s["logits"], 1 << 28)
        assert all(torch.equal(a, b) for a, b in zip(ref, tm.token_logp(away, s["targets"], 20)))
        args = (s["targets"], ref[2], ref[1], s["dlogp"], s["dentropy"])
        assert torch.equal(tm.token_logp_backward(s["logits"], *args), tm.token_logp_backward(away, *args))


@pytest.mark.parametrize("rows,vocab", [(6, 700), (6, 30000), (300, 30000)])
def test_logits_of_large_size(rows, vocab):
    """Results depend on the distances from the maximum alone."""
    s = _inputs(rows, vocab, "f32", seed=10, masked=0.0)
    s["logits"] = (s["logits"].double() + 1e4).float()
    got = tm.token_logp(s["logits"], s["targets"], 4, TAU)
    _check(s, got, 4)
    back = tm.token_logp_backward(s["logits"], s["targets"], got[2], got[1], s["dlogp"], s["dentropy"], TAU)
    _check_gradient(s, back, got[2], got[1], s["dlogp"], s["dentropy"], "f32")


def test_autograd_and_differences():
    s = _inputs(12, 90, "f32", seed=11)
    for use in ("logp", "entropy", "both"):
        leaf = s["logits"].clone().requires_grad_()
        logp, entropy, top_logp, top_ids = ops.token_logp(leaf, s["targets"], 4, TAU)
        assert not top_logp.requires_grad and not top_ids.requires_grad
        g, h = s["dlogp"] * (use != "entropy"), s["dentropy"] * (use != "logp")
        {"logp": logp @ g, "entropy": entropy @ h, "both": logp @ g + entropy @ h}[use].backward()

        def value(l):
            q = (l / TAU).log_softmax(1)
            on = s["targets"] >= 0
            lp = q.gather(1, s["targets"].clamp(min=0)[:, None])[:, 0]
            return (on * (lp * g.double() - (q.exp() * q).sum(1) * h.double())).sum()

        l = s["logits"].double()
        for r, v in ((0, 3), (5, int(s["targets"][5]) % 90), (11, 89)):
            step = torch.zeros_like(l)
            step[r, v] = 1e-5
            diff = float(value(l + step) - value(l - step)) / 2e-5
            assert abs(float(leaf.grad[r, v]) - diff) <= 1e-5 * (1 + abs(diff))
    logp, entropy = ops.token_logp(s["logits"], s["targets"])
    assert torch.equal(logp, tm.token_logp(s["logits"], s["targets"])[0])


def test_it_gives_what_the_policy_loss_takes():
    s = _inputs(100, 5000, "bf16", seed=12, masked=0.0)
    logp = tm.token_logp(s["logits"], s["targets"], temperature=TAU)[0]
    one = torch.ones(100, device="cuda")
    loss, own = tm.policy_loss(s["logits"], s["targets"], logp, one, one / 100, temperature=TAU)[:2]
    close("logp", own, logp.double(), 2 * (2 * 60 + 100 + 8 * 30) * U)
    assert abs(float(loss) + 1.0) < 1e-4      # ratios of one


def test_no_rows_and_refusals():
    s = _inputs(4, 64, "f32")
    got = tm.token_logp(s["logits"][:0], s["targets"][:0], 3)
    assert got[0].shape == (0,) and got[2].shape == (0, 2) and got[4].shape == (0, 3)
    assert tm.token_logp_backward(s["logits"][:0], s["targets"][:0], got[2], got[1]).shape == (0, 64)
    ok = tm.token_logp(s["logits"], s["targets"])
    for call in (lambda: tm.token_logp(s["logits"].half(), s["targets"]), lambda: tm.token_logp(s["logits"][0], s["targets"]),
                 lambda: tm.token_logp(s["logits"], s["targets"].int()), lambda: tm.token_logp(s["logits"], s["targets"][:2]),
                 lambda: tm.token_logp(s["logits"].cpu(), s["targets"]),
                 lambda: tm.token_logp_backward(s["logits"], s["targets"], ok[2][:, :1], ok[1]),
                 lambda: tm.token_logp_backward(s["logits"], s["targets"], ok[2], ok[1][:1]),
                 lambda: tm.token_logp_backward(s["logits"], s["targets"], ok[2], ok[1], s["dlogp"].double())):
        with pytest.raises(ValueError):
            call()
    for bad in (dict(top=65), dict(top=-1), dict(top=10 ** 9), dict(temperature=0.0), dict(temperature=float("nan"))):
        with pytest.raises(tm.TurboMuonError) as e:
            tm.token_logp(s["logits"], s["targets"], **bad)
        assert e.value.status == tm.TM_ERR_INVALID_ARG
    with pytest.raises(tm.TurboMuonError):
        tm.token_logp(s["logits"][:, :5].contiguous(), s["targets"], 6)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [30, 1500, 9000, 60000, 300000])
def test_plus_infinity(vocab, dtype):
    """A row with it gives NaN, the place itself is found; the other rows are as without it."""
    log(f"case: log probabilities, +inf among {vocab} {dtype}")
    logits = torch.randn((6, vocab), generator=generator(40), device="cuda").to(DT[dtype])
    targets = torch.randint(vocab, (6,), generator=generator(41), device="cuda")
    clean = tm.token_logp(logits, targets, 4)
    logits[2, vocab - 3] = float("inf")
    logits[4, 5] = logits[4, vocab // 2] = float("inf")
    got = tm.token_logp(logits, targets, 4)
    rest = torch.tensor([0, 1, 3, 5], device="cuda")
    assert all(torch.equal(a[rest], b[rest]) for a, b in zip(got, clean))
    for r in (2, 4):
        assert got[0][r].isnan() and got[1][r].isnan() and got[3][r].isnan().all()
    assert int(got[4][2, 0]) == vocab - 3 and got[4][4, :2].tolist() == [5, vocab // 2]
    back = tm.token_logp_backward(logits, targets, got[2], got[1], torch.ones(6, device="cuda"))
    assert back[rest].isfinite().all() and back[2].isnan().any() and back[4].isnan().any()
