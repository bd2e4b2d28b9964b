"""The operators as a program uses them: the example, streams, graphs, workspaces, timing."""
import importlib.util
import os

import pytest

from gpu_helpers import log

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from paper_2512_04632_amd import _lib as tm  # noqa: E402
from paper_2512_04632_amd.optim import TurboMuon  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _all(seed, rows=300):
    """Inputs of every operator."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def randn(*s):
        return torch.randn(s, generator=g, device="cuda")

    counts = torch.tensor([rows // 3, 0, rows - rows // 3])
    return dict(x=randn(rows, 256).bfloat16(), dy=randn(rows, 256).bfloat16(), w=randn(256), b=randn(256),
                m=randn(3, 256, 512).bfloat16(), ends=counts.cumsum(0).to(torch.int32).cuda(),
                logits=randn(rows, 10000), targets=torch.randint(10000, (rows,), generator=g, device="cuda"),
                v=randn(3, rows), weights=torch.rand(rows, generator=g, device="cuda"))


def _run(s):
    y, mean, rstd = tm.layer_norm(s["x"], s["w"], s["b"])
    grads = tm.layer_norm_backward(s["dy"], s["x"], mean, rstd, s["w"])
    up = tm.expert_matmul(y, s["m"], s["ends"])
    down = tm.expert_matmul(up, s["m"], s["ends"], transposed=True)
    dw = tm.expert_wgrad(y, up, s["ends"])
    loss, logp, lse, slope = tm.policy_loss(s["logits"], s["targets"], s["v"][0] * 0.1 - 9, s["v"][1], s["weights"],
                                            s["v"][2] * 0.1 - 9, kl=0.1)
    back = tm.policy_loss_backward(s["logits"], s["targets"], lse, slope)
    few = tm.policy_loss_with_grad(s["logits"][:7], s["targets"][:7], s["v"][0, :7] - 9, s["v"][1, :7], s["weights"][:7])
    return [y, mean, rstd, *grads, up, down, dw, loss, logp, lse, slope, back, *few]


def _same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def test_two_streams_match_one():
    log("case: operators on two streams at once")
    sets = [_all(1), _all(2)]
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


def test_explicit_stream():
    s = _all(3)
    ref = tm.layer_norm(s["x"], s["w"], s["b"])
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    got = tm.layer_norm(s["x"], s["w"], s["b"], stream=st)
    st.synchronize()
    assert _same(ref, got)


def test_explicit_stream_orders_the_copies_it_needs():
    """Inputs that are copied first (columns outermost) are copied on the call's stream, not behind the work
    of the current one."""
    log("case: operators on a stream given by name, inputs of other strides")
    s = _all(4)
    flip = {k: v.t().contiguous().t() for k, v in s.items() if k in ("x", "dy", "logits")}
    mt = s["m"].transpose(1, 2).contiguous().transpose(1, 2)
    mean, rstd = tm.layer_norm(s["x"])[1:]
    lse, slope = tm.policy_loss(s["logits"], s["targets"], s["v"][0] - 9, s["v"][1], s["weights"])[2:]

    def calls(x, dy, m, logits, **kw):
        return [*tm.layer_norm(x, s["w"], s["b"], **kw), *tm.layer_norm_backward(dy, x, mean, rstd, s["w"], **kw),
                tm.expert_matmul(x, m, s["ends"], **kw), tm.expert_wgrad(x, dy, s["ends"], **kw),
                *tm.policy_loss(logits, s["targets"], s["v"][0] - 9, s["v"][1], s["weights"], **kw),
                *tm.policy_loss_with_grad(logits, s["targets"], s["v"][0] - 9, s["v"][1], s["weights"], **kw),
                tm.policy_loss_backward(logits, s["targets"], lse, slope, **kw)]

    ref = calls(s["x"], s["dy"], s["m"], s["logits"])
    busy = torch.randn(4096, 4096, device="cuda")
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(20):
        busy @ busy                               # milliseconds of work ahead on the current stream
    got = calls(flip["x"], flip["dy"], mt, flip["logits"], stream=st)
    st.synchronize()
    with torch.cuda.stream(st):
        same = _same(got, ref)
    torch.cuda.synchronize()
    assert same


def test_graph_replays_match_eager():
    log("case: operators in a captured graph")
    s, other = _all(4), _all(5)
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        _run(s)                                   # sizes the stream's workspaces
    st.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        out = _run(s)
    for rep in range(4):
        src = other if rep % 2 else _all(4)
        for k, v in s.items():
            v.copy_(src[k])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        kept = [t.clone() for t in out]
        assert _same(kept, _run(s)), rep


def test_capture_without_workspace_is_refused():
    tm.release_workspaces()
    s = _all(6)
    y, mean, rstd = tm.layer_norm(s["x"], s["w"], s["b"])
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        kept = s["x"] + 1
        with pytest.raises(tm.TurboMuonError) as e:
            tm.layer_norm_backward(s["dy"], s["x"], mean, rstd, s["w"])
    assert e.value.status == tm.TM_ERR_UNSUPPORTED
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(kept, s["x"] + 1)


def test_failed_allocation_is_reported(monkeypatch):
    s = _all(7)
    ref = _run(s)
    tm.release_workspaces()
    monkeypatch.setenv("TM_TEST_FAIL_ALLOC", "1")
    with pytest.raises(tm.TurboMuonError) as e:
        tm.layer_norm_backward(s["dy"], s["x"], ref[1], ref[2], s["w"])
    assert e.value.status == tm.TM_ERR_NO_MEMORY
    monkeypatch.delenv("TM_TEST_FAIL_ALLOC")
    assert _same(ref, _run(s))


def test_timing_records_each_operator():
    s = _all(8)
    tm.timing_reset()
    tm.timing_enable(True)
    try:
        _run(s)
    finally:
        tm.timing_enable(False)
    for phase, calls in (("layer_norm", 1), ("layer_norm_backward", 1), ("expert_matmul", 2), ("expert_wgrad", 1),
                         ("policy_loss", 2), ("policy_loss_backward", 1)):
        ms, n = tm.timing_read(phase)
        assert n == calls and ms > 0.0, phase
    tm.timing_reset()


def test_optimizer_takes_stacks_of_matrices():
    """A stack of expert matrices is updated as its matrices are one by one."""
    g = torch.Generator(device="cuda")
    g.manual_seed(9)
    stack = torch.randn((3, 64, 96), generator=g, device="cuda")
    grad = torch.randn((3, 64, 96), generator=g, device="cuda")
    together = torch.nn.Parameter(stack.clone())
    single = [torch.nn.Parameter(m.clone()) for m in stack]
    a, b = TurboMuon([together], lr=0.1), TurboMuon(single, lr=0.1)
    for _ in range(3):
        together.grad = grad.clone()
        for p, m in zip(single, grad):
            p.grad = m.clone()
        a.step()
        b.step()
    assert torch.equal(together.detach(), torch.stack([p.detach() for p in single]))
    assert not torch.equal(together.detach(), stack)


def test_example_learns():
    log("case: the expert policy example")
    spec = importlib.util.spec_from_file_location("expert_policy", os.path.join(ROOT, "examples", "expert_policy.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    right = example.train(steps=20, rows=2048, say=log)
    assert right[0] < 0.05 and right[-1] > 0.3
