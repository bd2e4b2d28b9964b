"""What training steps around the optimizer ask of the framework's operators, as timed cases.

Three operators: layer norm (forward; backward with the gradients of weight and bias), products of
ragged groups of rows with one matrix per expert (forward, gradient of the rows, gradient of the
matrices) and the clipped policy loss with a KL term (value, gradient, both in one pass).
"""
import math

import torch

own = False

EPS = 1e-5
CLIP_LOW, CLIP_HIGH, KL, TEMPERATURE = 0.2, 0.28, 0.02, 0.9


def listed():
    return [
        # one short sequence of a 768-wide model: nothing but latency
        {"name": "ln_fwd_64x768", "op": "ln_fwd", "rows": 64, "d": 768, "dtype": "bf16"},
        # a training batch of a 4096-wide model, forward and backward
        {"name": "ln_fwd_16384x4096", "op": "ln_fwd", "rows": 16384, "d": 4096, "dtype": "bf16"},
        {"name": "ln_bwd_16384x4096", "op": "ln_bwd", "rows": 16384, "d": 4096, "dtype": "bf16"},
        # an odd width in fp32, ragged batch
        {"name": "ln_bwd_4001x1001_f32", "op": "ln_bwd", "rows": 4001, "d": 1001, "dtype": "f32"},
        # a few tokens through the experts of a 768-wide model: the matrices are read for a row or two each
        {"name": "expert_fwd_24x8x768x2048", "op": "expert_fwd", "rows": 24, "experts": 8, "k": 768,
         "n": 2048, "skew": 0.5, "dtype": "bf16"},
        # a training batch through the MLP matrices of an 8B-class model, forward and the matrices' gradient
        {"name": "expert_fwd_16384x8x4096x14336", "op": "expert_fwd", "rows": 16384, "experts": 8,
         "k": 4096, "n": 14336, "skew": 0.4, "dtype": "bf16"},
        {"name": "expert_dw_16384x8x4096x14336", "op": "expert_dw", "rows": 16384, "experts": 8,
         "k": 4096, "n": 14336, "skew": 0.4, "dtype": "bf16"},
        # many small experts, unevenly used, some not at all: the rows' gradient
        {"name": "expert_dx_8192x64x2048x1408", "op": "expert_dx", "rows": 8192, "experts": 64,
         "k": 2048, "n": 1408, "skew": 1.2, "dtype": "bf16"},
        # odd sizes in fp32
        {"name": "expert_fwd_3001x5x515x777_f32", "op": "expert_fwd", "rows": 3001, "experts": 5,
         "k": 515, "n": 777, "skew": 0.7, "dtype": "f32"},
        # the value alone for the tokens of one short answer, with a vocabulary of odd size
        {"name": "loss_fwd_16x50257", "op": "loss_fwd", "rows": 16, "vocab": 50257, "masked": 0.0,
         "dtype": "bf16"},
        # a training batch over a large vocabulary, value and gradient; a quarter of it is prompt
        {"name": "loss_grad_8192x131072", "op": "loss_grad", "rows": 8192, "vocab": 131072,
         "masked": 0.25, "dtype": "bf16"},
        # the gradient as automatic differentiation asks for it, odd sizes in fp32
        {"name": "loss_bwd_3000x32001_f32", "op": "loss_bwd", "rows": 3000, "vocab": 32001,
         "masked": 0.1, "dtype": "f32"},
    ]


def _log_uniform(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    """One more case: 1 to 32768 rows; widths 32 to 8192; 1 to 64 experts of sides 64 to 8192;
    vocabularies 1000 to 131072; odd sizes in half of the cases, fp32 in a third."""
    dtype = rng.choice(["bf16", "bf16", "f32"])
    unit = rng.choice([1, 64])

    def size(lo, hi):
        v = _log_uniform(rng, lo, hi)
        return max(1, round(v)) if unit == 1 else max(unit, unit * round(v / unit))

    kind = rng.choice(["ln", "expert", "expert", "loss"])
    if kind == "ln":
        d = size(32, 8192)
        rows = max(1, min(round(_log_uniform(rng, 1, 32768)), 16384 * 4096 // 2 // d))
        return {"op": rng.choice(["ln_fwd", "ln_bwd"]), "rows": rows, "d": d, "dtype": dtype}
    if kind == "expert":
        k, n = size(64, 8192), size(64, 8192)
        experts = max(1, min(round(_log_uniform(rng, 1, 64)), int(2e8 / (k * n)) or 1))
        most = 4e11 if dtype == "bf16" else 4e10
        rows = max(1, min(round(_log_uniform(rng, 1, 32768)), int(most / (k * n))))
        return {"op": rng.choice(["expert_fwd", "expert_dx", "expert_dw"]), "rows": rows,
                "experts": experts, "k": k, "n": n, "skew": round(rng.uniform(0.0, 1.5), 2), "dtype": dtype}
    vocab = size(1000, 131072)
    rows = max(1, min(round(_log_uniform(rng, 1, 32768)), int(4e8 / vocab)))
    return {"op": rng.choice(["loss_fwd", "loss_grad", "loss_bwd"]), "rows": rows, "vocab": vocab,
            "masked": round(rng.uniform(0.0, 0.5), 2), "dtype": dtype}


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _counts(case):
    """Rows of each expert, most used first: shares that fall as a power of the rank, rounded to
    whole rows by the largest remainders."""
    shares = [(i + 1.0) ** -case["skew"] for i in range(case["experts"])]
    exact_rows = [case["rows"] * s / sum(shares) for s in shares]
    counts = [int(v) for v in exact_rows]
    order = sorted(range(len(counts)), key=lambda i: (counts[i] - exact_rows[i], i))
    for i in order[:case["rows"] - sum(counts)]:
        counts[i] += 1
    return counts


def _masked(case):
    return int(case["masked"] * case["rows"])


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    host = torch.Generator()
    host.manual_seed(int(seed))
    dt = _dtype(case)

    def randn(*shape, dtype=dt, scale=1.0):
        return torch.randn(shape, generator=g, device="cuda", dtype=dtype).mul_(scale)

    state = {"case": case}
    if case["op"] in ("ln_fwd", "ln_bwd"):
        rows, d = case["rows"], case["d"]
        # a residual stream: channels with means of their own, a few of them large
        offset = randn(d, dtype=torch.float32, scale=0.5) + 0.2
        x = (randn(rows, d, dtype=torch.float32, scale=1.5) + offset).to(dt)
        state.update(x=x, weight=1.0 + randn(d, dtype=torch.float32, scale=0.1),
                     bias=randn(d, dtype=torch.float32, scale=0.1))
        if case["op"] == "ln_bwd":
            mean, rstd = _moments(x.float())
            state.update(dy=randn(rows, d, scale=0.1), mean=mean, rstd=rstd)
    elif case["op"] in ("expert_fwd", "expert_dx", "expert_dw"):
        rows, experts, k, n = case["rows"], case["experts"], case["k"], case["n"]
        counts = _counts(case)
        counts = [counts[i] for i in torch.randperm(experts, generator=host).tolist()]
        state["counts"] = counts
        state["ends"] = torch.tensor(counts).cumsum(0).to(torch.int32).cuda()
        if case["op"] != "expert_dx":
            state["x"] = randn(rows, k)
        if case["op"] != "expert_fwd":
            state["dy"] = randn(rows, n, scale=0.02)
        if case["op"] != "expert_dw":
            state["w"] = randn(experts, k, n, scale=k ** -0.5)
    else:
        rows, vocab = case["rows"], case["vocab"]
        logits = randn(rows, vocab, scale=2.0)
        targets = torch.randint(vocab, (rows,), generator=g, device="cuda")
        at = torch.arange(rows, device="cuda")
        # sampled tokens are mostly likely ones
        logits[at, targets] = (randn(rows, dtype=torch.float32, scale=2.0) + 12.0).to(dt)
        weights = torch.full((rows,), 1.0 / max(1, rows - _masked(case)), device="cuda")
        weights[torch.randperm(rows, generator=g, device="cuda")[:_masked(case)]] = 0.0
        logp = torch.cat([_log_prob(part, t)[0] for part, t in
                          zip(logits.split(512), targets.split(512))]) * (weights != 0)
        # the policy that sampled was a little different: ratios around one, none within a
        # thousandth of a clipping bound, where the last bit would decide the gradient
        ratio = (randn(rows, dtype=torch.float32, scale=0.2)).exp()
        ratio = _away(_away(ratio, 1 - CLIP_LOW), 1 + CLIP_HIGH)
        state.update(logits=logits, targets=targets, weights=weights, old_logp=logp - ratio.log(),
                     ref_logp=logp + randn(rows, dtype=torch.float32, scale=0.3),
                     advantages=randn(rows, dtype=torch.float32) + 0.3)
        if case["op"] == "loss_bwd":
            lse = torch.cat([_log_prob(part, t)[1] for part, t in
                             zip(logits.split(512), targets.split(512))]) * (weights != 0)
            state.update(lse=lse, slope=_terms(state, logp)[1])
    return state


def _away(ratio, bound):
    near = (ratio - bound).abs() < 1e-3
    return torch.where(near, bound + torch.where(ratio >= bound, 2e-3, -2e-3), ratio)


def _moments(x):
    mean = x.mean(-1)
    centred = x - mean[:, None]
    return mean, torch.rsqrt((centred * centred).mean(-1) + EPS)


def _log_prob(logits, targets):
    """Log probability of each target and the log of the row's sum of exponentials, at the
    temperature, in 32 bits."""
    z = logits.float() / TEMPERATURE
    top = z.amax(-1, keepdim=True)
    lse = (z - top).exp().sum(-1).log() + top[:, 0]
    return z.gather(-1, targets[:, None])[:, 0] - lse, lse


def _terms(s, logp):
    """Each row's share of the loss, and its derivative by the log probability."""
    m, a = s["weights"], s["advantages"]
    ratio = (logp - s["old_logp"]).exp()
    clipped = ratio.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH)
    gap = s["ref_logp"] - logp
    grad = torch.where(ratio * a <= clipped * a, -ratio * a, torch.zeros_like(a)) + KL * (1 - gap.exp())
    value = -torch.minimum(ratio * a, clipped * a) + KL * (gap.exp() - gap - 1)
    active = m != 0
    return torch.where(active, m * value, 0), torch.where(active, m * grad, 0)


def _loss_gradient(s, lse, slope):
    z = s["logits"].float() / TEMPERATURE
    grad = (z - lse[:, None]).exp().neg()
    grad.scatter_add_(-1, s["targets"][:, None], torch.ones_like(slope)[:, None])
    grad = grad * (slope / TEMPERATURE)[:, None]
    return torch.where((s["weights"] != 0)[:, None], grad, 0).to(s["logits"].dtype)


def _plain(s, op):
    if op == "ln_fwd":
        x = s["x"].float()
        mean, rstd = _moments(x)
        y = (x - mean[:, None]) * rstd[:, None] * s["weight"] + s["bias"]
        return y.to(s["x"].dtype), mean, rstd
    if op == "ln_bwd":
        dy = s["dy"].float()
        h = (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
        g = dy * s["weight"]
        dx = s["rstd"][:, None] * (g - g.mean(-1, keepdim=True) - h * (g * h).mean(-1, keepdim=True))
        return dx.to(s["x"].dtype), (dy * h).sum(0), dy.sum(0)
    if op == "expert_fwd":
        parts = zip(s["x"].split(s["counts"]), s["w"])
        return torch.cat([x.float() @ w.float() for x, w in parts if len(x)]).to(s["x"].dtype)
    if op == "expert_dx":
        parts = zip(s["dy"].split(s["counts"]), s["w"])
        return torch.cat([dy.float() @ w.float().t() for dy, w in parts if len(dy)]).to(s["dy"].dtype)
    if op == "expert_dw":
        parts = zip(s["x"].split(s["counts"]), s["dy"].split(s["counts"]))
        return torch.stack([x.float().t() @ dy.float() for x, dy in parts])
    if op == "loss_bwd":
        return _loss_gradient(s, s["lse"], s["slope"])
    logp, lse = _log_prob(s["logits"], s["targets"])
    active = s["weights"] != 0
    logp, lse = torch.where(active, logp, 0), torch.where(active, lse, 0)
    value, slope = _terms(s, logp)
    if op == "loss_fwd":
        return value.sum(), logp, lse, slope
    return value.sum(), logp, _loss_gradient(s, lse, slope)


def run(state):
    op = state["case"]["op"]
    if not own:
        return _plain(state, op)
    from paper_2512_04632_amd import _lib as tm
    if op == "ln_fwd":
        return tm.layer_norm(state["x"], state["weight"], state["bias"], eps=EPS)
    if op == "ln_bwd":
        return tm.layer_norm_backward(state["dy"], state["x"], state["mean"], state["rstd"], state["weight"])
    if op == "expert_fwd":
        return tm.expert_matmul(state["x"], state["w"], state["ends"])
    if op == "expert_dx":
        return tm.expert_matmul(state["dy"], state["w"], state["ends"], transposed=True)
    if op == "expert_dw":
        return tm.expert_wgrad(state["x"], state["dy"], state["ends"])
    if op == "loss_bwd":
        return tm.policy_loss_backward(state["logits"], state["targets"], state["lse"], state["slope"],
                                       temperature=TEMPERATURE)
    call = tm.policy_loss if op == "loss_fwd" else tm.policy_loss_with_grad
    return call(state["logits"], state["targets"], state["old_logp"], state["advantages"],
                state["weights"], ref_logp=state["ref_logp"], clip_low=CLIP_LOW, clip_high=CLIP_HIGH,
                kl=KL, temperature=TEMPERATURE)


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    rows, op = case["rows"], case["op"]
    if op == "ln_fwd":
        return {"bytes": 2 * size * rows * case["d"] + 8 * (rows + case["d"]), "flops": 8 * rows * case["d"]}
    if op == "ln_bwd":
        return {"bytes": 3 * size * rows * case["d"] + 8 * rows + 12 * case["d"], "flops": 15 * rows * case["d"]}
    if op in ("expert_fwd", "expert_dx", "expert_dw"):
        k, n = case["k"], case["n"]
        if op == "expert_dw":
            matrices = 4 * case["experts"] * k * n
        else:
            matrices = size * sum(c > 0 for c in _counts(case)) * k * n
        return {"bytes": size * rows * (k + n) + matrices + 4 * case["experts"], "flops": 2 * rows * k * n}
    active, vocab = rows - _masked(case), case["vocab"]
    if op == "loss_fwd":
        return {"bytes": size * active * vocab + 36 * rows, "flops": 4 * active * vocab}
    return {"bytes": size * (active + rows) * vocab + 28 * rows,
            "flops": (8 if op == "loss_grad" else 4) * active * vocab}


def exact(case, seed):
    """The definitions in 64 bits, one part of the rows at a time."""
    s = prepare(case, seed)
    op = case["op"]
    d = {k: v.double() for k, v in s.items()
         if isinstance(v, torch.Tensor) and v.is_floating_point() and k not in ("logits", "w")}
    if op == "ln_fwd":
        x = d["x"]
        mu = x.sum(1) / case["d"]
        var = (x - mu.unsqueeze(1)).pow(2).sum(1) / case["d"]
        scale = 1 / (var + EPS).sqrt()
        return (x - mu.unsqueeze(1)) * scale.unsqueeze(1) * d["weight"] + d["bias"], mu, scale
    if op == "ln_bwd":
        h = (d["x"] - d["mean"].unsqueeze(1)) * d["rstd"].unsqueeze(1)
        dh = d["dy"] * d["weight"]
        along = (dh * h).sum(1, keepdim=True) / case["d"]
        dx = (dh - dh.sum(1, keepdim=True) / case["d"] - h * along) * d["rstd"].unsqueeze(1)
        return dx, (d["dy"] * h).sum(0), d["dy"].sum(0)
    if op in ("expert_fwd", "expert_dx", "expert_dw"):
        rows, k, n = case["rows"], case["k"], case["n"]
        shape = {"expert_fwd": (rows, n), "expert_dx": (rows, k), "expert_dw": (case["experts"], k, n)}[op]
        out = torch.zeros(shape, dtype=torch.float64, device="cuda")
        first = 0
        for e, count in enumerate(s["counts"]):
            last = first + count
            if op == "expert_fwd":
                out[first:last] = d["x"][first:last] @ s["w"][e].double()
            elif op == "expert_dx":
                out[first:last] = d["dy"][first:last] @ s["w"][e].double().t()
            else:
                out[e] = d["x"][first:last].t() @ d["dy"][first:last]
            first = last
        return out
    rows = case["rows"]
    loss = torch.zeros((), dtype=torch.float64, device="cuda")
    logp, lse, slope = (torch.zeros(rows, dtype=torch.float64, device="cuda") for _ in range(3))
    grad = torch.zeros(s["logits"].shape, dtype=torch.float64, device="cuda") if op != "loss_fwd" else None
    for first in range(0, rows, 512):
        at = torch.arange(first, min(first + 512, rows), device="cuda")
        at = at[d["weights"][at] != 0]
        if at.numel() == 0:
            continue
        z, y = s["logits"][at].double() / TEMPERATURE, s["targets"][at]
        one = torch.arange(at.numel(), device="cuda")
        if op == "loss_bwd":
            lse[at], slope[at] = d["lse"][at], d["slope"][at]
        else:
            lse[at] = torch.logsumexp(z, 1)
            logp[at] = z[one, y] - lse[at]
            m, adv, r = d["weights"][at], d["advantages"][at], (logp[at] - d["old_logp"][at]).exp()
            inside = torch.where(adv >= 0, r <= 1 + CLIP_HIGH, r >= 1 - CLIP_LOW)
            bound = torch.where(adv >= 0, 1 + CLIP_HIGH, 1 - CLIP_LOW).double()
            q = (d["ref_logp"][at] - logp[at]).exp()
            loss += (m * (-torch.where(inside, r, bound) * adv + KL * (q - 1 - q.log()))).sum()
            slope[at] = m * (KL * (1 - q) - inside * r * adv)
        if grad is not None:
            p = (z - lse[at].unsqueeze(1)).exp().neg_()
            p[one, y] += 1
            grad[at] = p * (slope[at] / TEMPERATURE).unsqueeze(1)
    if op == "loss_fwd":
        return loss, logp, lse, slope
    return grad if op == "loss_bwd" else (loss, logp, grad)
