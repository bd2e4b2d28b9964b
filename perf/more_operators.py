"""What stands between the products of an expert policy, as timed cases.

Four operators: root-mean-square norm with the residual's addition (forward, backward), the routing of
rows to experts with its balance loss (forward, backward), rows on their way to the experts' order and,
weighted, back (out, back, backward), and the log probabilities of given tokens with entropy and the
most likely alternatives (forward, backward).
"""
import math

import torch

own = False

EPS = 1e-5
TEMPERATURE = 0.9
SCALE = 1.5   # of the routing weights


def listed():
    return [
        # one token each of four answers that are being sampled: nothing but latency
        {"name": "rms_fwd_4x4096", "op": "rms_fwd", "rows": 4, "d": 4096, "residual": True, "dtype": "bf16"},
        # a training batch of a 4096-wide model, forward and backward
        {"name": "rms_fwd_16384x4096", "op": "rms_fwd", "rows": 16384, "d": 4096, "residual": True, "dtype": "bf16"},
        {"name": "rms_bwd_16384x4096", "op": "rms_bwd", "rows": 16384, "d": 4096, "residual": True, "dtype": "bf16"},
        # a short prompt's rows over the few experts of a small model
        {"name": "route_fwd_64x8", "op": "route_fwd", "rows": 64, "experts": 8, "top": 2, "masked": 0.0,
         "renormalize": True, "dtype": "f32"},
        # a training batch over many small experts
        {"name": "route_fwd_32768x256", "op": "route_fwd", "rows": 32768, "experts": 256, "top": 8, "masked": 0.0,
         "renormalize": True, "dtype": "f32"},
        # backwards, odd sizes, a tenth of the rows is padding, weights as the softmax gives them
        {"name": "route_bwd_16381x60", "op": "route_bwd", "rows": 16381, "experts": 60, "top": 4, "masked": 0.1,
         "renormalize": False, "dtype": "bf16"},
        # a training batch's rows to two experts each
        {"name": "gather_16384x4096_top2", "op": "gather", "rows": 16384, "d": 4096, "experts": 8, "top": 2,
         "masked": 0.0, "dtype": "bf16"},
        # eight experts' results for each row, added to the residual stream
        {"name": "combine_8192x2048_top8", "op": "combine", "rows": 8192, "d": 2048, "experts": 64, "top": 8,
         "masked": 0.0, "residual": True, "dtype": "bf16"},
        # backwards, odd sizes in fp32, padding among the rows
        {"name": "combine_bwd_3001x1023_top3", "op": "combine_bwd", "rows": 3001, "d": 1023, "experts": 5, "top": 3,
         "masked": 0.1, "dtype": "f32"},
        # the tokens of one short answer and what else was likely, a vocabulary of odd size
        {"name": "logp_fwd_16x50257_top20", "op": "logp_fwd", "rows": 16, "vocab": 50257, "top": 20, "masked": 0.0,
         "dtype": "bf16"},
        # what the sampling policy thought of a batch of answers over a large vocabulary; a quarter is prompt
        {"name": "logp_fwd_4096x131072_top5", "op": "logp_fwd", "rows": 4096, "vocab": 131072, "top": 5,
         "masked": 0.25, "dtype": "bf16"},
        # the gradient of log probabilities and entropies, odd sizes in fp32
        {"name": "logp_bwd_3000x32001", "op": "logp_bwd", "rows": 3000, "vocab": 32001, "masked": 0.1, "dtype": "f32"},
    ]


def _log_uniform(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    """One more case: 1 to 32768 rows; widths 32 to 8192; 2 to 512 experts of which each row takes 1 to 8;
    vocabularies 1000 to 131072 with up to 20 alternatives; odd sizes in half of the cases, fp32 in a third."""
    dtype = rng.choice(["bf16", "bf16", "f32"])
    unit = rng.choice([1, 64])

    def size(lo, hi):
        v = _log_uniform(rng, lo, hi)
        return max(1, round(v)) if unit == 1 else max(unit, unit * round(v / unit))

    kind = rng.choice(["rms", "route", "rows", "logp"])
    rows = max(1, round(_log_uniform(rng, 1, 32768)))
    masked = rng.choice([0.0, round(rng.uniform(0.0, 0.5), 2)])
    if kind == "rms":
        d = size(32, 8192)
        return {"op": rng.choice(["rms_fwd", "rms_bwd"]), "rows": min(rows, 16384 * 4096 // 2 // d), "d": d,
                "residual": rng.choice([True, True, False]), "dtype": dtype}
    experts = max(2, round(_log_uniform(rng, 2, 512)))
    top = rng.randint(1, min(8, experts))
    if kind == "route":
        return {"op": rng.choice(["route_fwd", "route_bwd"]), "rows": min(rows, 32768 * 256 // experts),
                "experts": experts, "top": top, "masked": masked, "renormalize": rng.choice([True, False]),
                "dtype": dtype}
    if kind == "rows":
        d = size(32, 8192)
        op = rng.choice(["gather", "combine", "combine_bwd"])
        case = {"op": op, "rows": max(1, min(rows, 16384 * 4096 // d // top)), "d": d, "experts": experts, "top": top,
                "masked": masked, "dtype": dtype}
        if op == "combine":
            case["residual"] = rng.choice([True, False])
        return case
    vocab = size(1000, 131072)
    case = {"op": rng.choice(["logp_fwd", "logp_bwd"]), "rows": min(rows, int(2e8 / vocab)), "vocab": vocab,
            "masked": masked, "dtype": dtype}
    if case["op"] == "logp_fwd":
        case["top"] = rng.choice([0, 1, 5, 20])
    return case


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _masked(case):
    return int(case["masked"] * case["rows"])


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    dt, op, rows = _dtype(case), case["op"], case["rows"]

    def randn(*shape, dtype=dt, scale=1.0):
        return torch.randn(shape, generator=g, device="cuda", dtype=dtype).mul_(scale)

    state = {"case": case}
    if op in ("rms_fwd", "rms_bwd"):
        d = case["d"]
        # a residual stream some channels of which are large, and a layer's smaller result
        stream = (randn(rows, d, dtype=torch.float32) * (1 + 4 * randn(d, dtype=torch.float32).abs() ** 3)).to(dt)
        state["weight"] = 1.0 + randn(d, dtype=torch.float32, scale=0.1)
        if op == "rms_fwd":
            state.update(x=randn(rows, d, scale=0.5) if case["residual"] else stream,
                         residual=stream if case["residual"] else None)
        else:
            state.update(sum=stream, rstd=_rstd(stream.float()), dy=randn(rows, d, scale=0.1),
                         dsum=randn(rows, d, scale=0.1) if case["residual"] else None)
        return state
    active = None
    if _masked(case):
        active = torch.ones(rows, dtype=torch.bool, device="cuda")
        active[torch.randperm(rows, generator=g, device="cuda")[:_masked(case)]] = False
    if op in ("logp_fwd", "logp_bwd"):
        vocab = case["vocab"]
        logits = randn(rows, vocab, scale=2.0)
        targets = torch.randint(vocab, (rows,), generator=g, device="cuda")
        # sampled tokens are mostly likely ones
        logits[torch.arange(rows, device="cuda"), targets] = (randn(rows, dtype=torch.float32, scale=2.0) + 12.0).to(dt)
        if active is not None:
            targets = torch.where(active, targets, -1)
        state.update(logits=logits, targets=targets)
        if op == "logp_bwd":
            _, entropy, stats = _token_values(logits, targets)
            state.update(stats=stats, entropy=entropy, dlogp=randn(rows, dtype=torch.float32, scale=1.0 / rows),
                         dentropy=randn(rows, dtype=torch.float32, scale=0.01 / rows))
        return state
    # router scores: some experts are liked by most rows
    experts, top = case["experts"], case["top"]
    logits = (randn(rows, experts, dtype=torch.float32) + randn(experts, dtype=torch.float32)).to(dt)
    if op in ("route_fwd", "route_bwd"):
        state.update(logits=logits, active=active)
        if op == "route_bwd":
            chosen, _, _, ends, _ = _route(logits, top, active, case["renormalize"])
            state.update(chosen=chosen, ends=ends, dweights=randn(rows, top, dtype=torch.float32, scale=0.1),
                         dbalance=torch.full((), 0.01, device="cuda"))
        return state
    _, weights, slots, ends, _ = _route(logits, top, active, True)
    state.update(slots=slots, ends=ends)
    if op == "gather":
        state["x"] = randn(rows, case["d"])
        return state
    state.update(weights=weights, y=randn(rows * top, case["d"]))
    if op == "combine":
        state["residual"] = randn(rows, case["d"]) if case["residual"] else None
    else:
        state["dout"] = randn(rows, case["d"], scale=0.1)
    return state


def _rstd(s):
    return torch.rsqrt((s * s).mean(-1) + EPS)


def _largest(x, top):
    """Indices of each row's `top` largest entries, largest first, of equal ones the lowest index: the
    entry's bits in an order of whole numbers, its distance from the end below them."""
    bits = (x.float() + 0.0).view(torch.int32)
    place = torch.arange(x.shape[1], device=x.device)
    key = torch.where(bits < 0, bits ^ 0x7fffffff, bits).long() * 2 ** 31 + (2 ** 31 - 1 - place)
    return 2 ** 31 - 1 - (key.topk(top, dim=1).values & (2 ** 31 - 1))


def _route(logits, top, active, renormalize):
    """(chosen, weights, slots, ends, balance): slots are the places of the rows' choices in the experts'
    order, rows in their own order within an expert; -1, as their choices, for rows that take no part."""
    rows, experts = logits.shape
    z = logits.float()
    p = (z - z.amax(1, keepdim=True)).exp()
    p = p / p.sum(1, keepdim=True)
    chosen = _largest(logits, top)
    weights = p.gather(1, chosen)
    if renormalize:
        weights = weights / weights.sum(1, keepdim=True)
    weights = weights * SCALE
    if active is not None:
        chosen = torch.where(active[:, None], chosen, experts)
        weights = torch.where(active[:, None], weights, 0)
        p = torch.where(active[:, None], p, 0)
    flat = chosen.reshape(-1)
    counts = torch.zeros(experts + 1, dtype=torch.int64, device=flat.device).scatter_add_(0, flat, torch.ones_like(flat))
    order = flat.argsort(stable=True)
    slots = torch.empty_like(order).scatter_(0, order, torch.arange(len(order), device=order.device))
    used = counts[:experts]
    taking = (rows * top - counts[experts]) / top
    balance = experts * (used / (top * taking).clamp(min=1) * (p.sum(0) / taking.clamp(min=1))).sum()
    slots = torch.where(flat < experts, slots, -1).view(rows, top)
    chosen = torch.where(chosen < experts, chosen, -1)
    return chosen.int(), weights, slots.int(), used.cumsum(0).int(), balance.float()


def _route_gradient(s, case):
    rows, experts = s["logits"].shape
    z = s["logits"].float()
    p = (z - z.amax(1, keepdim=True)).exp()
    p = p / p.sum(1, keepdim=True)
    used = s["ends"].float()
    counts = used - torch.cat([used.new_zeros(1), used[:-1]])
    taking = used[-1] / case["top"]
    u = (s["dbalance"] * experts * counts / (used[-1] * taking).clamp(min=1)).expand(rows, -1)
    on = (s["chosen"][:, :1] >= 0)
    at = s["chosen"].clamp(min=0).long()
    dw = s["dweights"] * SCALE
    grad = torch.zeros_like(z)
    if case["renormalize"]:
        share = p.gather(1, at)
        share = share / share.sum(1, keepdim=True)
        grad = grad.scatter(1, at, share * (dw - (share * dw).sum(1, keepdim=True)))
    else:
        u = u.scatter_add(1, at, dw)
    grad = grad + p * (u - (p * u).sum(1, keepdim=True))
    return torch.where(on, grad, 0).to(s["logits"].dtype)


def _token_values(logits, targets):
    """(logp, entropy, stats) of the targets' rows; stats are the largest logit and the sum of the
    exponentials of the distances from it at the temperature.  Rows of negative targets: zeros."""
    on = targets >= 0
    l = logits.float()
    m = l.amax(1)
    z = (l - m[:, None]) / TEMPERATURE
    e = z.exp()
    s = e.sum(1)
    logp = z.gather(1, targets.clamp(min=0)[:, None])[:, 0] - s.log()
    entropy = s.log() - (e * z).sum(1) / s
    return torch.where(on, logp, 0), torch.where(on, entropy, 0), torch.where(on[:, None], torch.stack([m, s], 1), 0)


def _token_gradient(s):
    m, total = s["stats"][:, :1], s["stats"][:, 1:]
    on = (s["targets"] >= 0)[:, None]
    z = (s["logits"].float() - m) / TEMPERATURE
    p = z.exp() / total
    grad = -p * (s["dlogp"][:, None] + s["dentropy"][:, None] * (z - total.log() + s["entropy"][:, None]))
    grad = grad.scatter_add(1, s["targets"].clamp(min=0)[:, None], s["dlogp"][:, None])
    return torch.where(on, grad / TEMPERATURE, 0).to(s["logits"].dtype)


def _plain(s, case):
    op, dt = case["op"], _dtype(case)
    if op == "rms_fwd":
        total = s["x"]
        if s["residual"] is not None:
            total = (s["x"].float() + s["residual"].float()).to(dt)
        rstd = _rstd(total.float())
        return (total.float() * rstd[:, None] * s["weight"]).to(dt), total, rstd
    if op == "rms_bwd":
        h = s["sum"].float() * s["rstd"][:, None]
        dy = s["dy"].float()
        g = dy * s["weight"]
        ds = s["rstd"][:, None] * (g - h * (g * h).mean(-1, keepdim=True))
        if s["dsum"] is not None:
            ds = ds + s["dsum"].float()
        return ds.to(dt), (dy * h).sum(0)
    if op == "route_fwd":
        return _route(s["logits"], case["top"], s["active"], case["renormalize"])
    if op == "route_bwd":
        return _route_gradient(s, case)
    if op in ("gather", "combine", "combine_bwd"):
        flat = s["slots"].reshape(-1).long()
        on = flat >= 0
        count = case["rows"] * case["top"]
        if op == "gather":
            out = s["x"].new_zeros(count + 1, case["d"])   # the last line takes what has no slot
            out[torch.where(on, flat, count)] = s["x"].repeat_interleave(case["top"], 0)
            return out[:count]
        if op == "combine":
            parts = s["y"][flat.clamp(min=0)].float() * torch.where(on, s["weights"].reshape(-1), 0)[:, None]
            out = parts.view(case["rows"], case["top"], -1).sum(1)
            if s["residual"] is not None:
                out = out + s["residual"].float()
            return out.to(dt)
        dout = s["dout"].float().repeat_interleave(case["top"], 0)
        dweights = torch.where(on, (dout * s["y"][flat.clamp(min=0)].float()).sum(1), 0).view(case["rows"], case["top"])
        dy = s["y"].new_zeros(count + 1, case["d"])
        dy[torch.where(on, flat, count)] = (dout * s["weights"].reshape(-1, 1)).to(dt)
        return dy[:count], dweights
    if op == "logp_bwd":
        return _token_gradient(s)
    logp, entropy, stats = _token_values(s["logits"], s["targets"])
    if case["top"] == 0:
        return logp, entropy, stats
    on = (s["targets"] >= 0)[:, None]
    ids = _largest(s["logits"], case["top"])
    top = (s["logits"].gather(1, ids).float() - stats[:, :1]) / TEMPERATURE - stats[:, 1:].log()
    return logp, entropy, stats, torch.where(on, top, 0), torch.where(on, ids, -1)


def run(state):
    case = state["case"]
    op = case["op"]
    if not own:
        return _plain(state, case)
    from paper_2512_04632_amd import _lib as tm
    if op == "rms_fwd":
        return tm.rms_norm(state["x"], state["weight"], state["residual"], eps=EPS)
    if op == "rms_bwd":
        return tm.rms_norm_backward(state["dy"], state["sum"], state["rstd"], state["weight"], state["dsum"])
    if op == "route_fwd":
        return tm.expert_route(state["logits"], case["top"], state["active"], renormalize=case["renormalize"],
                               scale=SCALE)
    if op == "route_bwd":
        return tm.expert_route_backward(state["logits"], state["chosen"], state["ends"], state["dweights"],
                                        state["dbalance"], renormalize=case["renormalize"], scale=SCALE)
    if op == "gather":
        return tm.expert_gather(state["x"], state["slots"], state["ends"])
    if op == "combine":
        return tm.expert_combine(state["y"], state["slots"], state["weights"], state["residual"])
    if op == "combine_bwd":
        return tm.expert_combine_backward(state["dout"], state["y"], state["slots"], state["ends"], state["weights"])
    if op == "logp_bwd":
        return tm.token_logp_backward(state["logits"], state["targets"], state["stats"], state["entropy"],
                                      state["dlogp"], state["dentropy"], temperature=TEMPERATURE)
    out = tm.token_logp(state["logits"], state["targets"], top=case["top"], temperature=TEMPERATURE)
    return out if case["top"] else out[:3]


def work(case):
    size, rows, op = 2 if case["dtype"] == "bf16" else 4, case["rows"], case["op"]
    if op in ("rms_fwd", "rms_bwd"):
        d = case["d"]
        arrays = 4 if case["residual"] else 2 if op == "rms_fwd" else 3
        return {"bytes": arrays * size * rows * d + 4 * rows + (4 if op == "rms_fwd" else 8) * d,
                "flops": (5 if op == "rms_fwd" else 11) * rows * d}
    on = rows - _masked(case)
    if op in ("logp_fwd", "logp_bwd"):
        vocab = case["vocab"]
        if op == "logp_fwd":
            return {"bytes": size * on * vocab + (24 + 12 * case["top"]) * rows, "flops": 5 * on * vocab}
        return {"bytes": size * (on + rows) * vocab + 28 * rows, "flops": 9 * on * vocab}
    experts, top = case["experts"], case["top"]
    if op == "route_fwd":
        return {"bytes": size * on * experts + 12 * rows * top + 4 * experts + (rows if _masked(case) else 0),
                "flops": (5 + top) * on * experts}
    if op == "route_bwd":
        return {"bytes": size * (on + rows) * experts + 8 * rows * top + 4 * experts, "flops": 8 * on * experts}
    d = case["d"]
    if op == "gather":
        return {"bytes": size * (on + rows * top) * d + 4 * rows * top, "flops": 0}
    if op == "combine":
        arrays = on * top + rows + (rows if case["residual"] else 0)
        return {"bytes": size * arrays * d + 8 * rows * top, "flops": 2 * on * top * d}
    return {"bytes": size * (on + on * top + rows * top) * d + 12 * rows * top, "flops": 3 * on * top * d}


def exact(case, seed):
    """The definitions in 64 bits, row by row or expert by expert where that is plainer."""
    s = prepare(case, seed)
    op, rows = case["op"], case["rows"]
    if op == "rms_fwd":
        total = s["x"] if s["residual"] is None else s["x"] + s["residual"]   # one rounding: both are of the type
        t = total.double()
        scale = (t.pow(2).sum(1) / case["d"] + EPS).pow(-0.5)
        return t * scale.unsqueeze(1) * s["weight"].double(), total.double(), scale
    if op == "rms_bwd":
        x, r, dy = s["sum"].double(), s["rstd"].double().unsqueeze(1), s["dy"].double()
        dh = dy * s["weight"].double()
        ds = dh * r - x * r.pow(3) * (dh * x).sum(1, keepdim=True) / case["d"]
        if s["dsum"] is not None:
            ds += s["dsum"].double()
        return ds, (dy * x * r).sum(0)
    if op in ("route_fwd", "route_bwd"):
        top, experts = case["top"], case["experts"]
        on = s["active"] if s["active"] is not None else torch.ones(rows, dtype=torch.bool, device="cuda")
        where = on.nonzero()[:, 0]
        p = torch.softmax(s["logits"][where].double(), 1)
        n = max(1, where.numel())
        if op == "route_fwd":
            ids = s["logits"][where].double().sort(dim=1, descending=True, stable=True).indices[:, :top]
        else:
            ids = s["chosen"][where].long()
        counts = torch.bincount(ids.reshape(-1), minlength=experts)
        if op == "route_fwd":
            chosen = torch.full((rows, top), -1, dtype=torch.int64, device="cuda")
            slots, weights = chosen.clone(), torch.zeros((rows, top), dtype=torch.float64, device="cuda")
            chosen[where] = ids
            first = 0
            for e in range(experts):
                mine = (chosen == e).reshape(-1).nonzero()[:, 0]
                slots.view(-1)[mine] = torch.arange(first, first + mine.numel(), device="cuda")
                first += mine.numel()
            w = p.gather(1, ids)
            weights[where] = SCALE * (w / w.sum(1, keepdim=True) if case["renormalize"] else w)
            balance = experts * torch.dot(counts.double() / (n * top), p.sum(0) / n)
            return chosen.int(), weights, slots.int(), counts.cumsum(0).int(), balance
        # by automatic differentiation of the two results
        z = s["logits"].double().requires_grad_()
        q = torch.softmax(z[where], 1)
        w = q.gather(1, ids)
        if case["renormalize"]:
            w = w / w.sum(1, keepdim=True)
        share = counts.double() / (n * top)
        value = (SCALE * w * s["dweights"][where].double()).sum()
        value = value + s["dbalance"].double() * experts * (share * q.sum(0) / n).sum()
        return torch.autograd.grad(value, z)[0]
    if op in ("gather", "combine", "combine_bwd"):
        top, d, count = case["top"], case["d"], rows * case["top"]
        row = torch.full((count,), -1, dtype=torch.int64, device="cuda")   # whose choice stands in each place
        which = (s["slots"] >= 0).nonzero()
        row[s["slots"][which[:, 0], which[:, 1]].long()] = which[:, 0] * top + which[:, 1]
        full = row >= 0
        if op == "gather":
            out = torch.zeros((count, d), dtype=torch.float64, device="cuda")
            out[full] = s["x"].double()[row[full] // top]
            return out
        w = torch.zeros(count, dtype=torch.float64, device="cuda")
        w[full] = s["weights"].double().view(-1)[row[full]]
        if op == "combine":
            out = torch.zeros((rows, d), dtype=torch.float64, device="cuda")
            if s["residual"] is not None:
                out += s["residual"].double()
            return out.index_add_(0, row[full] // top, w[full].unsqueeze(1) * s["y"][full].double())
        dout = torch.zeros((count, d), dtype=torch.float64, device="cuda")
        dout[full] = s["dout"].double()[row[full] // top]
        dweights = torch.zeros(count, dtype=torch.float64, device="cuda")
        dweights[row[full]] = (dout[full] * s["y"][full].double()).sum(1)
        return dout * w.unsqueeze(1), dweights.view(rows, top)
    vocab, top = case["vocab"], case.get("top", 0)
    logp, entropy = (torch.zeros(rows, dtype=torch.float64, device="cuda") for _ in range(2))
    stats = torch.zeros((rows, 2), dtype=torch.float64, device="cuda")
    likely = torch.zeros((rows, top), dtype=torch.float64, device="cuda")
    ids = torch.full((rows, top), -1, dtype=torch.int64, device="cuda")
    grad = torch.zeros((rows, vocab), dtype=torch.float64, device="cuda") if op == "logp_bwd" else None
    for at in (s["targets"] >= 0).nonzero()[:, 0].split(256):
        if at.numel() == 0:
            continue
        z, y = s["logits"][at].double() / TEMPERATURE, s["targets"][at]
        one = torch.arange(at.numel(), device="cuda")
        if grad is not None:
            st = s["stats"][at].double()
            logq = z - (st[:, :1] / TEMPERATURE + st[:, 1:].log())
            part = logq.exp() * -(s["dlogp"][at].double()[:, None] + s["dentropy"][at].double()[:, None]
                                  * (logq + s["entropy"][at].double()[:, None]))
            part[one, y] += s["dlogp"][at].double()
            grad[at] = part / TEMPERATURE
            continue
        logq = torch.log_softmax(z, 1)
        logp[at] = logq[one, y]
        entropy[at] = -(logq.exp() * logq).sum(1)
        stats[at, 0] = s["logits"][at].double().max(1).values
        stats[at, 1] = (z - stats[at, :1] / TEMPERATURE).exp().sum(1)
        if top:
            ids[at] = s["logits"][at].sort(dim=1, descending=True, stable=True).indices[:, :top]
            likely[at] = logq.gather(1, ids[at])
    if grad is not None:
        return grad
    return (logp, entropy, stats, likely, ids) if top else (logp, entropy, stats)
