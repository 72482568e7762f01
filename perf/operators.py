"""The operators of a length predictor, as cases that can be timed.

The router takes predicted lengths; the paper's predictor of them is a mixture of experts: a small
network scores the experts of a request, the experts are multilayer networks, their results are added
up by the scores.  A case is one call of one operator, inputs and outputs in device memory.

Plain values of a case:

  op        "route"    scores -> chosen experts, weights, and the slots in the order of experts
            "linear"   a layer of every expert on the rows that chose it
            "combine"  the weighted sum of a row's results
            "clip"     the global norm of a list of gradients, and clipping by it
  back      False: forward; True: the gradient of the forward
  dtype     "float32", "bfloat16" or "float16": what scores, features, weights, gradients are held in
  rows, experts, top_k   requests; experts; experts that each request goes to

  route     scoring ("softmax" or "sigmoid"), bias (True: one per expert, for the choice only), groups and
            kept (of equal size; only the best `kept` are chosen from), renorm (weights of a request sum
            to 1), masked (some requests may not go to some experts, a few of them to none)
  linear    n_in, n_out, relu, gather (True: rows are requests, taken by slot; False: rows are slots already),
            skew (0: experts are chosen alike; larger: some much more often, some hardly or never)
  combine   n_out
  clip      tensors: how many; total: elements; clipped: whether the norm is above the limit; predictor: the
            tensors of a predictor with these experts rather than random lengths
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
NO_EXPERT = float("-inf")
MOST_FLOPS, MOST_BYTES = 1.2e12, 3.0e9      # of a drawn case


def _route(name, dtype, rows, experts, top_k, scoring="softmax", bias=False, groups=1, kept=1, renorm=True, masked=False,
           back=False):
    return dict(name=name, op="route", back=back, dtype=dtype, rows=rows, experts=experts, top_k=top_k, scoring=scoring,
                bias=bias, groups=groups, kept=kept, renorm=renorm, masked=masked)


def _linear(name, dtype, rows, experts, top_k, n_in, n_out, relu=True, gather=True, skew=0.5, back=False):
    return dict(name=name, op="linear", back=back, dtype=dtype, rows=rows, experts=experts, top_k=top_k, n_in=n_in,
                n_out=n_out, relu=relu, gather=gather, skew=skew)


def _combine(name, dtype, rows, experts, top_k, n_out, back=False):
    return dict(name=name, op="combine", back=back, dtype=dtype, rows=rows, experts=experts, top_k=top_k, n_out=n_out)


def _clip(name, dtype, tensors, total, clipped=True, predictor=False):
    return dict(name=name, op="clip", back=False, dtype=dtype, tensors=tensors, total=total, clipped=clipped,
                predictor=predictor)


def listed():
    return [
        # the arrivals of a moment on the tiny fleet, the paper's nine experts, all of them asked: launches and host time
        _route("route_arrivals", "float32", 16, 9, 9, renorm=False),
        # a batch of the mid fleet, many small experts in groups with a bias for balance, masks
        _route("route_groups", "bfloat16", 4096, 64, 6, scoring="sigmoid", bias=True, groups=8, kept=4, masked=True),
        # a quarter of a million arrivals of the heavy fleet
        _route("route_heavy", "bfloat16", 262144, 64, 8, bias=True),
        # a training step's batch: the gradient of the scores
        _route("route_back", "float32", 65536, 64, 8, renorm=True, masked=True, back=True),
        # one arriving request, all nine experts: every weight is read for one row
        _linear("linear_one", "bfloat16", 1, 9, 9, 4096, 1024, skew=0.0),
        # a batch of the mid fleet, odd widths (a vocabulary cut at no round number), single precision
        _linear("linear_odd", "float32", 4099, 9, 2, 1023, 511, skew=1.0),
        # the arrivals of the large fleet through the first and widest layer
        _linear("linear_large", "bfloat16", 65536, 9, 2, 4096, 1024),
        # a training step's batch through the same layer
        _linear("linear_back", "bfloat16", 32768, 9, 2, 4096, 1024, back=True),
        # the results of the large fleet's arrivals, wide, two experts each
        _combine("combine_large", "float16", 65536, 64, 2, 1024),
        # the gradient of the predictor's last sum: one number per expert
        _combine("combine_back", "float32", 65536, 9, 9, 1, back=True),
        # the router's own gradients: a few small tensors
        _clip("clip_small", "float32", 4, 60000),
        # all gradients of a predictor of the paper's size
        _clip("clip_predictor", "bfloat16", 20, 45_000_000, predictor=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    n = _log_int(rng, lo, hi)
    return n if rng.random() < 0.5 or n < 64 else n // 64 * 64


def draw(rng):
    op = rng.choice(["route", "route", "linear", "linear", "linear", "combine", "clip"])
    dtype = rng.choice(["float32", "bfloat16", "bfloat16", "float16"])
    back = rng.random() < 0.4
    while True:
        if op == "clip":
            case = _clip("", dtype, _log_int(rng, 1, 60), _log_int(rng, 1000, 64_000_000), rng.random() < 0.75)
        else:
            rows = _log_int(rng, 1, 262144)
            experts = rng.choice([1, 4, 8, 9, 9, 16, 33, 64, 128, 256])
            top_k = rng.randint(1, min(experts, rng.choice([2, 9, 9, 16])))
            if op == "route":
                # (one expert, or the only choice's share of itself, would be the same whatever the scores)
                experts = max(experts, 4)
                renorm = rng.random() < 0.6
                top_k = max(top_k, 2 if renorm else 1)
                groups = rng.choice([1, 1] + [g for g in (2, 4, 8) if experts % g == 0 and experts // g >= 2])
                kept = rng.randint(max(1, -(-top_k * groups // experts)), groups)
                case = _route("", dtype, rows, experts, top_k, rng.choice(["softmax", "sigmoid"]), rng.random() < 0.5,
                              groups, kept, renorm, rng.random() < 0.4, back)
            elif op == "linear":
                experts = min(experts, 64)
                top_k, n_out = min(top_k, experts), _width(rng, 1, 2048)
                # (a handful of results may all be zero behind a rectifier)
                case = _linear("", dtype, rows, experts, top_k, _width(rng, 16, 4096), n_out,
                               rng.random() < 0.7 and rows * top_k * n_out >= 64, rng.random() < 0.5, rng.choice([0.0, 0.5, 1.0, 3.0]), back)
            else:
                case = _combine("", dtype, rows, experts, top_k, _width(rng, 1, 2048), back)
        w = work(case)
        # (single precision has no wide products: a tenth of the largest case's operations cost as much)
        if w["bytes"] <= MOST_BYTES and w["flops"] <= MOST_FLOPS * (0.1 if dtype == "float32" else 1.0):
            del case["name"]
            return case


def work(case):
    b = DTYPES[case["dtype"]].itemsize
    if case["op"] == "clip":
        return {"bytes": 2 * case["total"] * b, "flops": 3 * case["total"]}
    T, E, k = case["rows"], case["experts"], case["top_k"]
    S = T * k
    if case["op"] == "route":
        if case["back"]:
            return {"bytes": 2 * T * E * b + 8 * S, "flops": 6 * T * E}
        return {"bytes": T * E * b + 16 * S + 4 * (E + 1) + (4 * E if case["bias"] else 0), "flops": 4 * T * E}
    O = case["n_out"]
    if case["op"] == "combine":
        if case["back"]:
            return {"bytes": (2 * S + T) * O * b + 12 * S, "flops": 3 * S * O}
        return {"bytes": (S + T) * O * b + 8 * S, "flops": 2 * S * O}
    I = case["n_in"]
    n_x, used = (T if case["gather"] else S), min(E, S)
    if case["back"]:
        dz = 2 if case["relu"] else 0       # (the results are read, and the gradient before them is one of the outputs)
        return {"bytes": b * (n_x * I + S * O * (1 + dz) + used * I * O + S * I + E * (I + 1) * O) + 4 * S, "flops": 4 * S * I * O}
    return {"bytes": b * (n_x * I + used * (I + 1) * O + S * O) + 4 * S, "flops": 2 * S * I * O}


# ---- inputs -----------------------------------------------------------------------------------


def _plan(expert, n_expert):
    """off, slot, pos of choices [rows, top_k]: the slots in the order of experts, -1 (no expert) last."""
    e = expert.reshape(-1).long()
    e = torch.where(e < 0, n_expert, e)
    order = torch.sort(e, stable=True).indices
    off = torch.zeros(n_expert + 1, dtype=torch.int32, device=e.device)
    count = torch.zeros(n_expert + 1, dtype=torch.int64, device=e.device).index_add_(0, e, torch.ones_like(e))
    off[1:] = torch.cumsum(count[:n_expert], 0).int()
    kept = torch.arange(e.numel(), device=e.device) < off[n_expert]
    slot = torch.where(kept, order, -1 - order).int()
    pos = torch.empty_like(order)
    pos[order] = torch.where(kept, torch.arange(e.numel(), device=e.device), -1)
    return off, slot, pos.int().reshape(expert.shape)


def _scores(logits, scoring, wide):
    x = logits.to(wide)
    if scoring == "sigmoid":
        return 1 / (1 + torch.exp(-x))
    m = x.max(1, keepdim=True).values
    e = torch.exp(x - torch.where(m == NO_EXPERT, torch.zeros_like(m), m))
    e = torch.where(x == NO_EXPERT, torch.zeros_like(e), e)
    return e / torch.where(m == NO_EXPERT, torch.ones_like(m), e.sum(1, keepdim=True))


def _choose(s, logits, bias, top_k, groups, kept):
    T, E = s.shape
    masked = logits == NO_EXPERT
    c = s if bias is None else s + bias.to(s.dtype)
    c = torch.where(masked, torch.full_like(c, NO_EXPERT), c)
    if kept < groups:
        two = torch.sort(c.reshape(T, groups, E // groups), dim=2, descending=True).values[:, :, :2]
        none = two[:, :, 0] == NO_EXPERT
        group = torch.where(two == NO_EXPERT, torch.zeros_like(two), two).sum(2)
        group = torch.where(none, torch.full_like(group, NO_EXPERT), group)
        best = torch.sort(group, dim=1, descending=True, stable=True).indices[:, :kept]
        keep = torch.zeros_like(none).scatter_(1, best, True)
        c = torch.where(keep.repeat_interleave(E // groups, dim=1), c, torch.full_like(c, NO_EXPERT))
    top = torch.sort(c, dim=1, descending=True, stable=True)
    none = top.values[:, :top_k] == NO_EXPERT
    return torch.where(none, -1, top.indices[:, :top_k]).int()


def _weights(s, expert, renorm, scale):
    w = torch.gather(s, 1, expert.long().clamp(min=0))
    w = torch.where(expert < 0, torch.zeros_like(w), w)
    if renorm:
        r = w.sum(1, keepdim=True)
        w = torch.where(r == 0, torch.zeros_like(w), w / r)
    return w * scale


def _logits(case, g, dev):
    """Scores of a trained router, with requests left out whose choice hangs on a rounding."""
    T, E = case["rows"], case["experts"]
    x = 1.5 * torch.randn(T, E, generator=g, device=dev) + 0.5 * torch.randn(1, E, generator=g, device=dev)
    if case["masked"]:
        out = torch.rand(T, E, generator=g, device=dev) < 0.2 * (torch.rand(T, 1, generator=g, device=dev) < 0.25)
        out |= torch.rand(T, 1, generator=g, device=dev) < 1 / 512
        x = torch.where(out, torch.full_like(x, NO_EXPERT), x)
    x = x.to(DTYPES[case["dtype"]])
    bias = 0.05 * torch.randn(E, generator=g, device=dev) if case["bias"] else None
    s = _scores(x, case["scoring"], torch.float64)
    c = s if bias is None else s + bias.double()
    c = torch.where(x == NO_EXPERT, torch.full_like(c, NO_EXPERT), c)
    near = torch.zeros(T, dtype=torch.bool, device=dev)
    lists = [c]
    if case["kept"] < case["groups"]:
        two = torch.sort(c.reshape(T, case["groups"], -1), dim=2, descending=True).values[:, :, :2]
        lists.append(torch.where(two == NO_EXPERT, torch.zeros_like(two), two).sum(2))
    for v in lists:
        v = torch.sort(v, dim=1, descending=True).values
        gap, size = v[:, :-1] - v[:, 1:], v[:, :-1].abs() + v[:, 1:].abs() + (0.0 if bias is None else 0.05)
        near |= ((gap > 0) & (gap < 2e-6 * size)).any(1)
    good = torch.nonzero(~near).flatten()
    if good.numel():
        stand = good[torch.arange(T, device=dev) % good.numel()]
        x = torch.where(near[:, None], x[stand], x)
    return x.contiguous(), bias


def _choices(case, g, dev):
    """Experts of requests as a router chooses them, some more often than others, distinct per request."""
    T, E, k = case["rows"], case["experts"], case["top_k"]
    liked = case.get("skew", 0.5) * torch.randn(1, E, generator=g, device=dev)
    noise = -torch.log(-torch.log(torch.rand(T, E, generator=g, device=dev).clamp(1e-9, 1 - 1e-7)))
    return torch.sort(liked + noise, dim=1, descending=True).indices[:, :k].int().contiguous()


def _lengths(case):
    if case["predictor"]:       # nine experts of four layers and a router of two, 45 M in all
        E, w = 9, [4096, 1024, 512, 128, 1]
        shapes = [s for i, o in zip(w, w[1:]) for s in ((E, o, i), (E, o))] + [(512, 4096), (512,), (E, 512), (E,)]
        n = [math.prod(s) for s in shapes]
        return n + [max(1, case["total"] - sum(n))]
    rng = random.Random(case["tensors"] * 1000003 + case["total"])      # (a model's lengths do not change from step to step)
    cut = [rng.random() ** 3 + 1e-6 for _ in range(case["tensors"])]
    return [max(1, int(x / sum(cut) * case["total"])) for x in cut]


def prepare(case, seed):
    dev = torch.device("cuda", torch.cuda.current_device())
    g = torch.Generator(device=dev)
    g.manual_seed(seed * 1000003 + 17)
    dt = DTYPES[case["dtype"]]
    s = dict(case)

    def randn(*shape, scale=1.0, of=dt):
        return torch.randn(*shape, generator=g, device=dev, dtype=of if of.itemsize > 2 else torch.float32).mul_(scale).to(of)

    def out(*shape, of=dt):
        return torch.empty(*shape, dtype=of, device=dev)

    if case["op"] == "clip":
        n = _lengths(case)
        s["grads"] = [randn(m, scale=1e-3) for m in n]
        s["max_norm"] = (0.25 if case["clipped"] else 4.0) * 1e-3 * math.sqrt(sum(n))
    else:
        T, E, k = case["rows"], case["experts"], case["top_k"]
        S = T * k
        s["scale"] = 1.0
    if case["op"] == "route":
        s["logits"], s["bias"] = _logits(case, g, dev)
        if case["back"]:
            sc = _scores(s["logits"], case["scoring"], torch.float32)
            s["expert"] = _choose(sc, s["logits"], s["bias"], k, case["groups"], case["kept"])
            s["dweight"] = randn(T, k, of=torch.float32)
    elif case["op"] in ("linear", "combine"):
        s["off"], s["slot"], s["pos"] = _plan(_choices(case, g, dev), E)
    if case["op"] == "linear":
        I, O = case["n_in"], case["n_out"]
        s["x"] = randn(T if case["gather"] else S, I).clamp_(min=-0.5)
        s["w"] = randn(E, O, I, scale=I ** -0.5)
        s["b"] = randn(E, O, scale=0.1)
        if case["back"]:
            s["dy"] = randn(S, O)
            s["y"] = randn(S, O).clamp_(min=0) if case["relu"] else None
    elif case["op"] == "combine":
        s["y"] = randn(S, case["n_out"])
        s["weight"] = torch.rand(T, k, generator=g, device=dev)
        s["weight"] /= s["weight"].sum(1, keepdim=True)
        if case["back"]:
            s["dout"] = randn(T, case["n_out"])
    if own:
        from paper_2605_16867_amd import binding
        if case["op"] == "clip":
            s["h"] = binding.Experts(1, 1, 1)
            s["out"], s["norm"] = [torch.empty_like(x) for x in s["grads"]], out(1, of=torch.float32)
        else:
            s["h"] = binding.Experts(E, T, k)
        if case["op"] == "route":
            if case["back"]:
                s["out"] = out(T, E)
            else:
                s["out"] = dict(weight=out(T, k, of=torch.float32), expert=out(T, k, of=torch.int32),
                                off=out(E + 1, of=torch.int32), slot=out(S, of=torch.int32), pos=out(T, k, of=torch.int32))
        elif case["op"] == "linear":
            if case["back"]:
                s["out"] = dict(dx=out(S, I), dw=out(E, O, I), db=out(E, O))
                if case["relu"]:
                    s["out"]["dz"] = out(S, O)
            else:
                s["out"] = out(S, O)
        elif case["op"] == "combine":
            s["out"] = dict(dy=out(S, case["n_out"]), dweight=out(T, k, of=torch.float32)) if case["back"] else out(T, case["n_out"])
    return s


# ---- one pass ---------------------------------------------------------------------------------


def run(s):
    if own:
        return _run_own(s)
    return _compute(s, torch.float32, lambda x: x.to(DTYPES[s["dtype"]]))


def _run_own(s):
    h = s["h"]
    if s["op"] == "clip":
        h.gr_clip_gradients(s["grads"], s["max_norm"], s["norm"], out=s["out"])
        return {"norm": s["norm"], "grads": s["out"]}
    o = s["out"]
    if s["op"] == "route":
        if s["back"]:
            h.gr_expert_route_backward(s["logits"], s["expert"], s["dweight"], o, scoring=s["scoring"], renormalise=s["renorm"],
                                       scale=s["scale"])
        else:
            h.gr_expert_route(s["logits"], o["weight"], o["expert"], o["off"], o["slot"], o["pos"], bias=s["bias"],
                              scoring=s["scoring"], n_group=s["groups"], n_group_kept=s["kept"], renormalise=s["renorm"],
                              scale=s["scale"])
    elif s["op"] == "linear":
        slot, k = (s["slot"], s["top_k"]) if s["gather"] else (None, 1)
        if s["back"]:
            h.gr_expert_linear_backward(s["x"], s["w"], s["dy"], out_dx=o["dx"], out_dw=o["dw"], out_db=o["db"], y=s["y"],
                                        out_dz=o.get("dz"), off=s["off"], slot=slot, top_k=k)
        else:
            h.gr_expert_linear(s["x"], s["w"], o, bias=s["b"], off=s["off"], slot=slot, top_k=k, relu=s["relu"])
    elif s["back"]:
        h.gr_expert_combine_backward(s["dout"], s["y"], s["slot"], o["dy"], weight=s["weight"], out_dweight=o["dweight"])
    else:
        h.gr_expert_combine(s["y"], s["pos"], o, weight=s["weight"])
    return o


def _compute(s, wide, narrow):
    if s["op"] == "clip":
        return _clip_plain(s, wide, narrow)
    if s["op"] == "route":
        return _route_back(s, wide, narrow) if s["back"] else _route_plain(s, wide)
    if s["op"] == "linear":
        return _linear_back(s, wide, narrow) if s["back"] else _linear_plain(s, wide, narrow)
    return _combine_back(s, wide, narrow) if s["back"] else _combine_plain(s, wide, narrow)


def _route_plain(s, wide):
    sc = _scores(s["logits"], s["scoring"], wide)
    expert = _choose(sc, s["logits"], s["bias"], s["top_k"], s["groups"], s["kept"])
    off, slot, pos = _plan(expert, s["experts"])
    return dict(weight=_weights(sc, expert, s["renorm"], s["scale"]), expert=expert, off=off, slot=slot, pos=pos)


def _route_back(s, wide, narrow):
    sc = _scores(s["logits"], s["scoring"], wide)
    chosen, at = s["expert"] >= 0, s["expert"].long().clamp(min=0)
    u = torch.where(chosen, s["dweight"].to(wide), torch.zeros_like(s["dweight"], dtype=wide)) * s["scale"]
    p = torch.where(chosen, torch.gather(sc, 1, at), torch.zeros_like(u))
    if s["renorm"]:
        # of w = p / R: (u - sum of u w) / R to every chosen score
        r = p.sum(1, keepdim=True)
        r = torch.where(r > 0, r, torch.full_like(r, float("inf")))
        u = torch.where(chosen, (u - (u * p / r).sum(1, keepdim=True)) / r, torch.zeros_like(u))
    ds = torch.zeros_like(sc).scatter_add_(1, at, u)
    if s["scoring"] == "sigmoid":
        return narrow(ds * sc * (1 - sc))
    return narrow(sc * (ds - (ds * sc).sum(1, keepdim=True)))


def _rows(s):
    """Every position's row of x."""
    p = s["slot"].long()
    return torch.where(p < 0, -1 - p, p) // s["top_k"] if s["gather"] else torch.arange(p.numel(), device=p.device)


def _linear_plain(s, wide, narrow):
    off, row = s["off"].tolist(), _rows(s)
    w, b, x = s["w"].to(wide), s["b"].to(wide), s["x"].to(wide)
    y = torch.zeros(row.numel(), s["n_out"], dtype=wide, device=w.device)
    for e, (lo, hi) in enumerate(zip(off, off[1:])):
        if hi > lo:
            y[lo:hi] = x[row[lo:hi]] @ w[e].t() + b[e]
    return narrow(y.clamp_(min=0) if s["relu"] else y)


def _linear_back(s, wide, narrow):
    off, row = s["off"].tolist(), _rows(s)
    w, x, dz = s["w"].to(wide), s["x"].to(wide), s["dy"].to(wide)
    if s["relu"]:
        dz = torch.where(s["y"] > 0, dz, torch.zeros_like(dz))
    dx = torch.zeros(row.numel(), s["n_in"], dtype=wide, device=w.device)
    dw = torch.zeros_like(w)
    db = torch.zeros(w.shape[0], w.shape[1], dtype=wide, device=w.device)
    for e, (lo, hi) in enumerate(zip(off, off[1:])):
        if hi > lo:
            d = dz[lo:hi]
            dx[lo:hi] = d @ w[e]
            dw[e] = d.t() @ x[row[lo:hi]]
            db[e] = d.sum(0)
    out = dict(dx=narrow(dx), dw=narrow(dw), db=narrow(db))
    if s["relu"]:
        out["dz"] = narrow(dz)
    return out


def _combine_plain(s, wide, narrow):
    pos = s["pos"].long()
    o = torch.zeros(s["rows"], s["n_out"], dtype=wide, device=pos.device)
    for j in range(s["top_k"]):
        got = s["y"][pos[:, j].clamp(min=0)].to(wide) * s["weight"][:, j, None].to(wide)
        o += torch.where(pos[:, j, None] < 0, torch.zeros_like(got), got)
    return narrow(o)


def _combine_back(s, wide, narrow):
    p = s["slot"].long()
    kept, at = p >= 0, torch.where(p < 0, -1 - p, p)
    d = s["dout"].to(wide)[at // s["top_k"]]
    d = torch.where(kept[:, None], d, torch.zeros_like(d))
    dw = torch.zeros(p.numel(), dtype=wide, device=p.device)
    dw[at] = torch.where(kept, (d * s["y"].to(wide)).sum(1), torch.zeros_like(dw))
    dy = d * s["weight"].reshape(-1)[at, None].to(wide)
    return dict(dy=narrow(dy), dweight=dw.to(torch.float32 if wide == torch.float32 else wide).reshape(s["weight"].shape))


def _clip_plain(s, wide, narrow):
    total = torch.zeros((), dtype=wide, device=s["grads"][0].device)
    for x in s["grads"]:
        total = total + (x.to(wide) * x.to(wide)).sum()
    norm = torch.sqrt(total)
    ratio = torch.where(norm > s["max_norm"], s["max_norm"] / norm, torch.ones_like(norm))
    ratio = torch.where(torch.isfinite(norm), ratio, torch.ones_like(norm))
    return {"norm": norm.reshape(1), "grads": [narrow(x.to(wide) * ratio) for x in s["grads"]]}


# ---- the definition in 64 bits ----------------------------------------------------------------


def exact(case, seed):
    """Element by element from the definitions, in double precision."""
    s = prepare(case, seed)
    s.pop("h", None)
    s.pop("out", None)
    D = torch.float64
    if case["op"] == "clip":
        squares = [torch.dot(x.to(D), x.to(D)) for x in s["grads"]]
        norm = torch.stack(squares).sum().sqrt()
        factor = min(1.0, s["max_norm"] / float(norm)) if float(norm) > 0 else 1.0
        return {"norm": norm.reshape(1), "grads": [x.to(D) * factor for x in s["grads"]]}
    k = case["top_k"]
    if case["op"] == "route":
        x = s["logits"].to(D)
        if case["scoring"] == "softmax":
            sc = torch.nan_to_num(torch.exp(x - torch.logsumexp(x, 1, keepdim=True)), nan=0.0)
        else:
            sc = torch.sigmoid(x)
        if not case["back"]:
            expert = _choose(sc, s["logits"], s["bias"], k, case["groups"], case["kept"])
            hot = (expert[:, :, None] == torch.arange(case["experts"], device=x.device)) if x.numel() * k < 1 << 28 else None
            w = (hot * sc[:, None, :]).sum(2) if hot is not None else torch.where(expert < 0, 0.0, torch.gather(sc, 1, expert.long().clamp(min=0)))
            if case["renorm"]:
                w = torch.nan_to_num(w / w.sum(1, keepdim=True), nan=0.0)
            return dict(weight=w * s["scale"], expert=None, off=None, slot=None, pos=None)
        # through the matrix of derivatives, row by row: d w_j / d l_e
        hot = (s["expert"][:, :, None] == torch.arange(case["experts"], device=x.device)).to(D)
        u = s["dweight"].to(D) * (s["expert"] >= 0)
        pick = (hot * u[:, :, None]).sum(1)                   # gradient of the weights, at the experts
        any_ = hot.sum(1)
        if case["renorm"]:
            r = (any_ * sc).sum(1, keepdim=True).clamp(min=1e-300)
            pick = any_ * (pick / r - (pick * sc).sum(1, keepdim=True) / r / r)
        if case["scoring"] == "sigmoid":
            return pick * sc * torch.sigmoid(-x)
        return sc * pick - sc * (sc * pick).sum(1, keepdim=True)
    n = s["slot"].long()
    at = torch.where(n < 0, ~n, n)
    row = torch.div(at, k, rounding_mode="floor")
    if case["op"] == "combine":
        w = torch.where(n < 0, 0.0, s["weight"].reshape(-1)[at].to(D))
        if not case["back"]:
            o = torch.zeros(case["rows"], case["n_out"], dtype=D, device=n.device)
            return o.index_add_(0, row, w[:, None] * s["y"].to(D))
        d = s["dout"].to(D)
        dw = torch.zeros(case["rows"] * k, dtype=D, device=n.device)
        dw[at] = torch.einsum("ij,ij->i", d[row], s["y"].to(D)) * (n >= 0)
        return dict(dy=d[row] * w[:, None], dweight=dw.reshape(case["rows"], k))
    if not case["gather"]:
        row = torch.arange(n.numel(), device=n.device)
    of = torch.bucketize(torch.arange(n.numel(), device=n.device), s["off"][1:].long(), right=True)     # every position's expert
    outs = {} if case["back"] else torch.zeros(n.numel(), case["n_out"], dtype=D, device=n.device)
    if case["back"]:
        dz = s["dy"].to(D)
        if case["relu"]:
            dz = dz * (s["y"] > 0)
            outs["dz"] = dz
        outs.update(dx=torch.zeros(n.numel(), case["n_in"], dtype=D, device=n.device),
                    dw=torch.zeros(s["w"].shape, dtype=D, device=n.device), db=torch.zeros(s["b"].shape, dtype=D, device=n.device))
    for e in range(case["experts"]):
        mine = torch.nonzero(of == e).flatten()
        if mine.numel() == 0:
            continue
        x, w = s["x"][row[mine]].to(D), s["w"][e].to(D)
        if case["back"]:
            d = dz[mine]
            outs["dx"][mine] = torch.mm(d, w)
            outs["dw"][e] = torch.mm(d.t().contiguous(), x)
            outs["db"][e] = torch.mv(d.t().contiguous(), torch.ones(mine.numel(), dtype=D, device=n.device))
        else:
            z = torch.addmm(s["b"][e].to(D), x, w.t())
            outs[mine] = torch.relu(z) if case["relu"] else z
    return outs
