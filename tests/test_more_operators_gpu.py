"""Norm, routing, rows to their experts and back, products and log probabilities as a program uses them together:
the block against 64 bits, streams, graphs, workspaces, timing."""
import pytest

from gpu_helpers import log

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from op_helpers import generator  # noqa: E402
from paper_2512_04632_amd import _lib as tm, ops  # noqa: E402

ROWS, D, HIDDEN, EXPERTS, TOP, VOCAB = 300, 256, 512, 8, 2, 40000


def _all(seed, rows=ROWS, vocab=VOCAB):
    g = generator(seed)

    def randn(*s):
        return torch.randn(s, generator=g, device="cuda")

    targets = torch.randint(vocab, (rows,), generator=g, device="cuda")
    targets[::9] = -1
    return dict(x=randn(rows, D).bfloat16(), residual=randn(rows, D).bfloat16(), norm=1 + 0.1 * randn(D),
                scores=randn(rows, EXPERTS), active=torch.rand(rows, generator=g, device="cuda") < 0.9,
                up=randn(EXPERTS, D, HIDDEN).bfloat16() * D ** -0.5, down=randn(EXPERTS, HIDDEN, D).bfloat16() * HIDDEN ** -0.5,
                logits=randn(rows, vocab).bfloat16(), targets=targets, long=randn(3, 131072).bfloat16(), gw=randn(rows, TOP), gb=randn(1)[0],
                gx=randn(rows, D).bfloat16(), gl=randn(rows), gh=randn(rows))


def _run(s):
    """Every call once, each on what the one before it gave."""
    y, total, rstd = tm.rms_norm(s["x"], s["norm"], s["residual"])
    chosen, weights, slots, ends, balance = tm.expert_route(s["scores"], TOP, s["active"])
    out = tm.expert_gather(y, slots, ends)
    back = tm.expert_matmul(tm.expert_matmul(out, s["up"], ends), s["down"], ends)
    x = tm.expert_combine(back, slots, weights, total)
    dy, dw = tm.expert_combine_backward(s["gx"], back, slots, ends, weights)
    dscores = tm.expert_route_backward(s["scores"], chosen, ends, dw, s["gb"])
    dh = tm.expert_combine(dy, slots)
    ds, dnorm = tm.rms_norm_backward(dh, total, rstd, s["norm"], s["gx"])
    found = tm.token_logp(s["logits"], s["targets"], 5)
    dl = tm.token_logp_backward(s["logits"], s["targets"], found[2], found[1], s["gl"], s["gh"])
    few = tm.token_logp(s["long"], s["targets"][1:4], 5)
    return [y, total, rstd, chosen, weights, slots, ends, balance, out, back, x, dy, dw, dscores, dh, ds, dnorm, *found, dl, *few]


def _same(a, b):
    return len(a) == len(b) and all(torch.equal(x, y) for x, y in zip(a, b))


def test_a_block_and_its_gradients():
    """Norm, routing, products, combination and log probabilities in one graph of gradients, against the same in
    64 bits with the same choices.  The activations between the operators are fp32, so that what is off comes of
    sums and exponentials alone: some hundred roundings of 2^-24 each, of sums of up to 512 terms of both signs."""
    log("case: an expert block with its gradients")
    s = _all(1, rows=120, vocab=500)
    names = ("x", "residual", "norm", "router", "up", "down", "head")
    g = generator(2)
    leaves = {k: s[k].float() for k in ("x", "residual", "norm", "up", "down")}
    leaves["router"] = torch.randn((D, EXPERTS), generator=g, device="cuda") * D ** -0.5
    leaves["head"] = torch.randn((1, D, 500), generator=g, device="cuda") * D ** -0.5
    leaves = {k: v.clone().requires_grad_() for k, v in leaves.items()}
    wide = {k: v.detach().double().requires_grad_() for k, v in leaves.items()}
    everyone = torch.full((1,), 120, dtype=torch.int32, device="cuda")
    h, total = ops.rms_norm(leaves["x"], leaves["norm"], leaves["residual"])
    weights, balance, chosen, slots, ends = ops.expert_route(h @ leaves["router"], TOP, s["active"])
    a = ops.expert_linear(ops.expert_gather(h, slots, ends), leaves["up"], ends)
    x = ops.expert_combine(ops.expert_linear(a.relu(), leaves["down"], ends), slots, weights, total, ends)
    logp, entropy = ops.token_logp(ops.expert_linear(x, leaves["head"], everyone), s["targets"])
    value = logp @ s["gl"] + 0.3 * (entropy @ s["gh"]) + 2.0 * balance
    value.backward()

    t = wide["x"] + wide["residual"]
    h = t * (t.pow(2).mean(1, keepdim=True) + 1e-5).rsqrt() * wide["norm"]
    p = (h @ wide["router"]).softmax(1)
    on = s["active"]
    w = p.gather(1, chosen.clamp(min=0).long())
    w = torch.where(on[:, None], w / w.sum(1, keepdim=True), 0)
    x = t
    for j in range(TOP):
        e = chosen[:, j].clamp(min=0).long()
        part = (torch.bmm(h[:, None], wide["up"][e].contiguous())).relu()
        x = x + w[:, j:j + 1] * torch.bmm(part, wide["down"][e].contiguous())[:, 0]
    q = (x @ wide["head"][0]).log_softmax(1)
    has = s["targets"] >= 0
    lp = torch.where(has, q.gather(1, s["targets"].clamp(min=0)[:, None])[:, 0], 0)
    ent = torch.where(has, -(q.exp() * q).sum(1), 0)
    counts = ends.diff(prepend=ends.new_zeros(1)).double()
    n = on.sum()
    want = lp @ s["gl"].double() + 0.3 * (ent @ s["gh"].double()) + 2.0 * EXPERTS * (counts / (TOP * n) * p[on].sum(0) / n).sum()
    want.backward()
    assert abs(float(value.detach()) - float(want.detach())) <= 1e-4 * (1 + abs(float(want.detach())))
    for k in names:
        got, exact = leaves[k].grad.double(), wide[k].grad
        assert float((got - exact).norm()) <= 2e-5 * float(exact.norm()), k


def test_two_streams_match_one():
    log("case: the operators on two streams at once")
    sets = [_all(3), _all(4)]
    ref = [_run(s) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        got = []
        for st, s in zip(streams, sets):
            with torch.cuda.stream(st):
                got.append(_run(s))
        torch.cuda.synchronize()
        assert _same(ref[0], got[0]) and _same(ref[1], got[1])


def test_explicit_stream_orders_the_copies_it_needs():
    log("case: the operators on a stream given by name, inputs of other strides")
    s = _all(5)
    ref = _run(s)
    y, total, rstd, chosen, weights, slots, ends = ref[:7]
    back, found = ref[9], ref[17:22]

    def calls(f, **kw):
        return [*tm.rms_norm(f(s["x"]), s["norm"], f(s["residual"]), **kw),
                *tm.rms_norm_backward(f(s["gx"]), f(total), rstd, s["norm"], f(s["gx"]), **kw),
                *tm.expert_route(f(s["scores"]), TOP, s["active"], **kw),
                tm.expert_route_backward(f(s["scores"]), f(chosen), ends, f(s["gw"]), s["gb"], **kw),
                tm.expert_gather(f(y), f(slots), ends, **kw), tm.expert_combine(f(back), f(slots), f(weights), f(total), **kw),
                *tm.expert_combine_backward(f(s["gx"]), f(back), f(slots), ends, f(weights), **kw),
                *tm.token_logp(f(s["logits"]), s["targets"], 5, **kw),
                tm.token_logp_backward(f(s["logits"]), s["targets"], f(found[2]), found[1], s["gl"], s["gh"], **kw)]

    ref = calls(lambda t: t)
    flipped = {}

    def flip(t):
        if t.data_ptr() not in flipped:
            flipped[t.data_ptr()] = t.t().contiguous().t()
        return flipped[t.data_ptr()]

    calls(flip)
    busy = torch.randn(4096, 4096, device="cuda")
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(20):
        busy @ busy                               # milliseconds of work ahead on the current stream
    got = calls(flip, stream=st)
    st.synchronize()
    with torch.cuda.stream(st):
        same = _same(got, ref)
    torch.cuda.synchronize()
    assert same


def test_graph_replays_match_eager():
    log("case: the operators in a captured graph")
    s, first, other = _all(6), _all(6), _all(7)
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        _run(s)                                   # sizes the stream's workspaces
    st.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        out = _run(s)
    for rep in range(4):
        for k, v in s.items():
            v.copy_((other if rep % 2 else first)[k])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        kept = [t.clone() for t in out]
        assert _same(kept, _run(s)), rep


def test_captured_gradients_match_eager():
    """Forward and backward of the differentiable calls, captured on leaves of their own."""
    log("case: captured gradients")
    s = _all(8, vocab=3000)

    def step(t):
        x, r, w, scores, logits = (t[k].detach().clone().requires_grad_() for k in ("x", "residual", "norm", "scores", "logits"))
        h, total = ops.rms_norm(x, w, r)
        weights, balance, _, slots, ends = ops.expert_route(scores, TOP, s["active"])
        out = ops.expert_combine(ops.expert_gather(h, slots, ends), slots, weights, total, ends)
        logp, entropy = ops.token_logp(logits, s["targets"])
        parts = [out, balance, logp, entropy]
        return torch.autograd.grad(parts, [x, r, w, scores, logits], [s["gx"], s["gb"], s["gl"], s["gh"]])

    want = [g.clone() for g in step(s)]
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        step(s)
    st.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        got = step(s)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert _same(want, got)
        assert _same(want, step(s))


def test_capture_without_workspace_is_refused():
    tm.release_workspaces()
    s = _all(9)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        kept = s["x"] + 1
        for call in (lambda: tm.expert_route(s["scores"], TOP), lambda: tm.token_logp(s["long"], s["targets"][1:4])):
            with pytest.raises(tm.TurboMuonError) as e:
                call()
            assert e.value.status == tm.TM_ERR_UNSUPPORTED
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(kept, s["x"] + 1)


def test_failed_allocation_is_reported(monkeypatch):
    s = _all(10)
    ref = _run(s)
    tm.release_workspaces()
    monkeypatch.setenv("TM_TEST_FAIL_ALLOC", "1")
    for call in (lambda: tm.expert_route(s["scores"], TOP), lambda: tm.token_logp(s["long"], s["targets"][1:4]),
                 lambda: tm.rms_norm_backward(s["gx"], ref[1], ref[2], s["norm"])):
        with pytest.raises(tm.TurboMuonError) as e:
            call()
        assert e.value.status == tm.TM_ERR_NO_MEMORY
    monkeypatch.delenv("TM_TEST_FAIL_ALLOC")
    assert _same(ref, _run(s))


def test_timing_records_each_operator():
    s = _all(11)
    _run(s)
    tm.timing_reset()
    tm.timing_enable(True)
    try:
        _run(s)
    finally:
        tm.timing_enable(False)
    for phase, calls in (("rms_norm", 1), ("rms_norm_backward", 1), ("expert_route", 1), ("expert_route_backward", 1),
                         ("expert_gather", 1), ("expert_combine", 2), ("expert_combine_backward", 1), ("token_logp", 2),
                         ("token_logp_backward", 1)):
        ms, n = tm.timing_read(phase)
        assert n == calls and ms > 0.0, phase
    tm.timing_reset()
