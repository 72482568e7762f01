"""The operators that read a request's tokens, as cases that can be timed.

A length predictor takes features of requests; these make them: rows of a table by token, a gated recurrence over
the tokens of every request, and dropout.  A case is one call of one operator, inputs and outputs in device memory.

Plain values of a case:

  op        "embed"    tokens -> rows of a table, scaled
            "scan"     h_t = f_t h_{t-1} + (1 - f_t) x_t along every sequence, f = sigmoid of a gate
            "dropout"  elements set to 0 at random, the rest scaled, added to a residual or not
  back      False: forward; True: the gradient of the forward (dropout's is the call itself)
  dtype     "float32", "bfloat16" or "float16": what tables, gates, values and gradients are held in

  embed     tokens, vocab, width; padded (True: some tokens are -1, which have no row)
  scan      tokens (of all sequences together), sequences, width; single (True: every token is a sequence of its own);
            start (True: sequences start from given states, else from 0); all (True: the states after every token,
            else the last ones only; backward: whether there is a gradient of those after every token)
  dropout   n, rate, residual
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
MOST_BYTES = 1.6e9      # of a drawn case


def _embed(name, dtype, tokens, vocab, width, padded=False, back=False):
    return dict(name=name, op="embed", back=back, dtype=dtype, tokens=tokens, vocab=vocab, width=width, padded=padded)


def _scan(name, dtype, tokens, sequences, width, single=False, start=False, all=True, back=False):
    return dict(name=name, op="scan", back=back, dtype=dtype, tokens=tokens, sequences=sequences, width=width, single=single,
                start=start, all=all)


def _dropout(name, dtype, n, rate, residual=False):
    return dict(name=name, op="dropout", back=False, dtype=dtype, n=n, rate=rate, residual=residual)


def listed():
    return [
        # the first tokens of a moment's arrivals: launch and host time
        _embed("embed_arrivals", "float32", 512, 32000, 256),
        # the prompts of a large batch: the rows that are written
        _embed("embed_large", "bfloat16", 524288, 65536, 1024),
        # the gradient of a small training batch, odd sizes, padding between its prompts
        _embed("embed_back_odd", "float32", 49999, 32003, 511, padded=True, back=True),
        # a large training batch, few tokens very often, most hardly ever
        _embed("embed_back_large", "bfloat16", 524288, 65536, 1024, back=True),
        # one generated token of every running request: its state moves on by it
        _scan("scan_token", "bfloat16", 4096, 4096, 1024, single=True, start=True),
        # a moment's arrivals, read at once; only the last states are wanted
        _scan("scan_arrivals", "float32", 3000, 16, 256, all=False),
        # the prompts of a training batch, of all lengths
        _scan("scan_prompts", "bfloat16", 262144, 1024, 1024),
        # one very long request
        _scan("scan_long", "float16", 65536, 1, 1024, start=True),
        # the gradient of a few long requests, single precision, an odd width
        _scan("scan_back_odd", "float32", 20001, 5, 515, start=True, back=True),
        # the gradient of the training batch
        _scan("scan_back_prompts", "bfloat16", 262144, 1024, 1024, back=True),
        # the features of a moment's arrivals
        _dropout("dropout_arrivals", "float32", 4095, 0.1),
        # the states of a training batch, added to what went in
        _dropout("dropout_large", "bfloat16", 268435456, 0.1, residual=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    n = _log_int(rng, lo, hi)
    return n if rng.random() < 0.5 or n < 64 else n // 64 * 64


def draw(rng):
    op = rng.choice(["embed", "embed", "scan", "scan", "scan", "dropout"])
    dtype = rng.choice(["float32", "bfloat16", "bfloat16", "float16"])
    back = rng.random() < 0.5
    while True:
        if op == "dropout":
            case = _dropout("", dtype, _log_int(rng, 64, 300_000_000), rng.choice([0.05, 0.1, 0.2, 0.5]), rng.random() < 0.5)
        elif op == "embed":
            case = _embed("", dtype, _log_int(rng, 1, 1 << 20), _log_int(rng, 64, 262144), _width(rng, 16, 4096),
                          rng.random() < 0.4, back)
        else:
            single = rng.random() < 0.2
            tokens = _log_int(rng, 1, 8192) if single else _log_int(rng, 1, 1 << 19)
            sequences = tokens if single else _log_int(rng, 1, min(tokens, 4096))
            case = _scan("", dtype, tokens, sequences, _width(rng, 16, 4096), single, rng.random() < 0.5, rng.random() < 0.75, back)
        if work(case)["bytes"] <= MOST_BYTES:
            del case["name"]
            return case


def work(case):
    b = DTYPES[case["dtype"]].itemsize
    if case["op"] == "dropout":
        return {"bytes": (3 if case["residual"] else 2) * case["n"] * b, "flops": 2 * case["n"]}
    N, C = case["tokens"], case["width"]
    if case["op"] == "embed":
        V = case["vocab"]
        distinct = min(N, V) if not case["back"] else V
        # (forward: about as many different tokens as there are draws from all of them, by their shares)
        if not case["back"]:
            distinct = _distinct(N, V)
        return {"bytes": (N + distinct) * C * b + 4 * N, "flops": (1 if not case["back"] else 2) * N * C}
    S = case["sequences"]
    if case["back"]:
        arrays = 6 if case["all"] else 5      # gate, value, state, its gradient -> two gradients
        states = (2 if case["start"] else 0) + 1
        return {"bytes": arrays * N * C * b + 4 * S * C * states, "flops": 14 * N * C}
    arrays, states = (3 if case["all"] else 2), (2 if case["start"] else 1)
    return {"bytes": arrays * N * C * b + 4 * S * C * states, "flops": 10 * N * C}


def _distinct(n, vocab):
    """How many different tokens n draws have: shares fall with the rank, log(rank) is uniform."""
    top, got, at = math.log((vocab + 2) / 2), 0.0, 2.0
    while at < vocab + 2:
        to = min(vocab + 2.0, max(at + 1, at * 1.1))
        got += (to - at) * -math.expm1(-n * math.log(to / at) / (to - at) / top)
        at = to
    return int(min(n, vocab, max(1, got)))


# ---- inputs -----------------------------------------------------------------------------------


def _tokens(case, g, dev):
    """Tokens of texts: the frequency of a token falls with its rank; ranks are spread over the vocabulary."""
    N, V = case["tokens"], case["vocab"]
    u = torch.rand(N, generator=g, device=dev, dtype=torch.float64)
    rank = (2 * torch.exp(u * math.log((V + 2) / 2)) - 2).long().clamp(0, V - 1)
    step = next(s for s in range(int(V * 0.618) | 1, 2 * V + 3) if math.gcd(s, V) == 1)
    token = (rank * step + 7) % V
    if case["padded"]:
        token = torch.where(torch.rand(N, generator=g, device=dev) < 1 / 16, torch.full_like(token, -1), token)
    return token.int()


def _offsets(case, g, dev):
    """Where sequences of all lengths start in the list of all tokens; a few may be empty."""
    N, S = case["tokens"], case["sequences"]
    share = torch.exp(torch.randn(S, generator=g, device=dev, dtype=torch.float64))
    cut = torch.round(torch.cumsum(share, 0) / share.sum() * N).int()
    cut[-1] = N
    return torch.cat([torch.zeros(1, dtype=torch.int32, device=dev), cut]).contiguous()


def prepare(case, seed):
    dev = torch.device("cuda", torch.cuda.current_device())
    g = torch.Generator(device=dev)
    g.manual_seed(seed * 1000003 + 29)
    dt = DTYPES[case["dtype"]]
    s = dict(case)

    def randn(*shape, of=dt, scale=1.0):
        return torch.randn(*shape, generator=g, device=dev, dtype=of if of.itemsize > 2 else torch.float32).mul_(scale).to(of)

    def out(*shape, of=dt):
        return torch.empty(*shape, dtype=of, device=dev)

    if case["op"] == "dropout":
        s["x"] = randn(case["n"])
        s["residual"] = randn(case["n"]) if case["residual"] else None
        s["seed"], s["offset"] = seed * 7919 + 3, 5 * seed + (1 << 33)
        if own:
            s["out"] = out(case["n"])
    elif case["op"] == "embed":
        s["token"], s["scale"] = _tokens(case, g, dev), math.sqrt(case["width"])
        s["dout" if case["back"] else "table"] = randn(case["tokens"] if case["back"] else case["vocab"], case["width"],
                                                       scale=1.0 if case["back"] else 0.02)
        if own:
            s["out"] = out(case["vocab"] if case["back"] else case["tokens"], case["width"])
    else:
        N, S, C = case["tokens"], case["sequences"], case["width"]
        # gates and values as one product of features leaves them, side by side; channels remember 2 to 2 000 tokens
        s["both"] = randn(N, 2 * C, scale=0.7)
        far = torch.exp(torch.rand(C, generator=g, device=dev) * math.log(1000) + math.log(2))
        s["both"][:, :C] += torch.log(far - 1).to(dt)
        s["off"] = None if case["single"] else _offsets(case, g, dev)
        s["h0"] = randn(S, C, of=torch.float32) if case["start"] else None
        if case["back"]:
            s["y"] = _scan_plain(s, torch.float32)[0].to(dt)
            s["dy"] = randn(N, C) if case["all"] else None
            s["dh"] = randn(S, C, of=torch.float32)
        if own:
            f32 = torch.float32
            if case["back"]:
                s["out"] = dict(dboth=out(N, 2 * C), dh0=out(S, C, of=f32) if case["start"] else None)
            else:
                s["out"] = dict(y=out(N, C) if case["all"] else None, h=out(S, C, of=f32))
    if own:
        from paper_2605_16867_amd import binding
        s["h"] = binding.Tokens(case.get("tokens", 1), case.get("vocab", 1), case.get("width", 1))
    return s


# ---- one pass ---------------------------------------------------------------------------------


def run(s):
    if own:
        return _run_own(s)
    dt = DTYPES[s["dtype"]]
    if s["op"] == "dropout":
        return _dropout_plain(s).to(dt)
    if s["op"] == "embed":
        return (_embed_back(s, torch.float32) if s["back"] else _embed_plain(s, torch.float32)).to(dt)
    if s["back"]:
        dboth, dh0 = _scan_back(s, torch.float32)
        return dict(dboth=dboth.to(dt), dh0=dh0)
    y, h = _scan_plain(s, torch.float32)
    return dict(y=y.to(dt) if s["all"] else None, h=h)


def _run_own(s):
    h, o = s["h"], s["out"]
    if s["op"] == "dropout":
        h.gr_dropout(s["x"], o, s["rate"], s["seed"], offset=s["offset"], residual=s["residual"])
    elif s["op"] == "embed":
        if s["back"]:
            h.gr_token_embed_backward(s["token"], s["dout"], o, scale=s["scale"])
        else:
            h.gr_token_embed(s["token"], s["table"], o, scale=s["scale"])
    else:
        C, both = s["width"], s["both"]
        if s["back"]:
            d = o["dboth"]
            h.gr_gated_scan_backward(both[:, :C], both[:, C:], s["y"], d[:, :C], d[:, C:], off=s["off"], h0=s["h0"], dy=s["dy"],
                                     dh=s["dh"], out_dh0=o["dh0"])
        else:
            h.gr_gated_scan(both[:, :C], both[:, C:], out_y=o["y"], off=s["off"], h0=s["h0"], out_h=o["h"])
    return o


def _embed_plain(s, wide):
    t = s["token"].long()
    kept = (t >= 0) & (t < s["vocab"])
    rows = s["table"][t.clamp(0, s["vocab"] - 1)].to(wide) * s["scale"]
    return torch.where(kept[:, None], rows, torch.zeros_like(rows))


def _embed_back(s, wide):
    t = s["token"].long()
    kept = (t >= 0) & (t < s["vocab"])
    d = torch.where(kept[:, None], s["dout"].to(wide), torch.zeros((), dtype=wide, device=t.device))
    return torch.zeros(s["vocab"], s["width"], dtype=wide, device=t.device).index_add_(0, t.clamp(0, s["vocab"] - 1), d) * s["scale"]


def _ranges(s):
    """First and last row of every sequence, and which sequences have one."""
    if s["off"] is None:
        first = torch.arange(s["tokens"], device=s["both"].device)
        return first, first, torch.ones_like(first, dtype=torch.bool)
    off = s["off"].long()
    return off[:-1], off[1:] - 1, off[1:] > off[:-1]


def _chain(a, b):
    """h_t = a_t h_{t-1} + b_t down the rows, by joining ever longer stretches (a = 0 where a sequence starts)."""
    d = 1
    while d < a.shape[0]:
        b[d:] += a[d:] * b[:-d].clone()
        a[d:] *= a[:-d].clone()
        d *= 2
    return b


def _scan_plain(s, wide):
    C = s["width"]
    gate, x = s["both"][:, :C].to(wide), s["both"][:, C:].to(wide)
    first, last, there = _ranges(s)
    h0 = torch.zeros(s["sequences"], C, dtype=wide, device=x.device) if s["h0"] is None else s["h0"].to(wide)
    a = 1 / (1 + torch.exp(-gate))
    b = x / (1 + torch.exp(gate))
    b[first[there]] += a[first[there]] * h0[there]
    a[first[there]] = 0
    y = _chain(a, b)
    h = h0.clone()
    h[there] = y[last[there]]
    return y, h


def _scan_back(s, wide):
    C = s["width"]
    gate, x = s["both"][:, :C].to(wide), s["both"][:, C:].to(wide)
    first, last, there = _ranges(s)
    first, last = first[there], last[there]
    f, i = 1 / (1 + torch.exp(-gate)), 1 / (1 + torch.exp(gate))
    before = torch.roll(s["y"].to(wide), 1, 0)
    before[first] = 0 if s["h0"] is None else s["h0"][there].to(wide)
    d = torch.zeros_like(x) if s["dy"] is None else s["dy"].to(wide).clone()
    d[last] += s["dh"][there].to(wide)
    a = torch.roll(f, -1, 0)
    a[last] = 0
    d = _chain(a.flip(0), d.flip(0)).flip(0)
    dh0 = s["dh"].to(wide).clone()
    dh0[there] = f[first] * d[first]
    return torch.cat([d * f * i * (before - x), d * i], 1), dh0 if s["h0"] is not None else None


def _threshold(rate):
    return int(round(rate * 65536))


def _random16(n, seed, offset, dev):
    """16 random bits for each of n elements: Philox 4x32 with ten rounds, a block of four words for eight elements."""
    c = torch.arange((n + 7) // 8, device=dev)
    low = 0xFFFFFFFF
    words = [c & low, c >> 32, torch.full_like(c, offset & low), torch.full_like(c, offset >> 32 & low)]
    key = [seed & low, seed >> 32 & low]
    for _ in range(10):
        p, q = words[0] * 0xD2511F53, words[2] * 0xCD9E8D57      # (64 bits, whose sign does not matter)
        words = [(q >> 32 & low) ^ words[1] ^ key[0], q & low, (p >> 32 & low) ^ words[3] ^ key[1], p & low]
        key = [key[0] + 0x9E3779B9 & low, key[1] + 0xBB67AE85 & low]
    return torch.stack([h for w in words for h in (w & 0xFFFF, w >> 16)], 1).view(-1)[:n]


def _dropout_plain(s):
    limit = _threshold(s["rate"])
    x = s["x"].float() * (65536 / (65536 - limit))
    x = torch.where(_random16(s["n"], s["seed"], s["offset"], x.device) < limit, torch.zeros_like(x), x)
    return x if s["residual"] is None else x + s["residual"].float()


# ---- the definition in 64 bits ----------------------------------------------------------------


def exact(case, seed):
    """From the definitions, in double precision: tokens one after the other."""
    s = prepare(case, seed)
    D, dev = torch.float64, torch.device("cuda", torch.cuda.current_device())
    if case["op"] == "dropout":
        return _dropout_exact(s, dev)
    if case["op"] == "embed":
        t = s["token"].long()
        if not case["back"]:
            rows = torch.cat([s["table"].to(D), torch.zeros(1, case["width"], dtype=D, device=dev)])
            return rows[torch.where(t < 0, case["vocab"], t)] * s["scale"]
        order = torch.sort(torch.where(t < 0, case["vocab"], t), stable=True)
        out = torch.zeros(case["vocab"] + 1, case["width"], dtype=D, device=dev)
        step = max(1, (1 << 27) // case["width"])
        for lo in range(0, t.numel(), step):
            out.index_add_(0, order.values[lo:lo + step], s["dout"][order.indices[lo:lo + step]].to(D))
        return out[:-1] * s["scale"]
    C, N = case["width"], case["tokens"]
    if case["single"]:
        start, length = torch.arange(N, device=dev), torch.ones(N, dtype=torch.long, device=dev)
    else:
        start, length = s["off"][:-1].long(), (s["off"][1:] - s["off"][:-1]).long()
    by = torch.sort(length, descending=True)
    start, most = start[by.indices], int(by.values[0])
    if most > 200000:      # (a dozen launches a token)
        return None
    alive = torch.bincount(length, minlength=most + 2).flip(0).cumsum(0).flip(0).tolist()[1:]      # sequences with more than t tokens
    gate, x = s["both"][:, :C], s["both"][:, C:]
    h0 = torch.zeros(case["sequences"], C, dtype=D, device=dev) if s["h0"] is None else s["h0"].to(D)
    if not case["back"]:
        h = h0[by.indices].clone()
        y = torch.zeros(N, C, dtype=D, device=dev) if case["all"] else None
        for t in range(most):
            n = alive[t]
            at = start[:n] + t
            h[:n] += torch.sigmoid(-gate[at].to(D)) * (x[at].to(D) - h[:n])
            if case["all"]:
                y[at] = h[:n]
        last = torch.empty_like(h)
        last[by.indices] = h
        return dict(y=y, h=last)
    carried = s["dh"].to(D)[by.indices].clone()
    both = torch.zeros(N, 2 * C, dtype=D, device=dev)
    for t in range(most - 1, -1, -1):
        n = alive[t]
        at = start[:n] + t
        d = carried[:n] if s["dy"] is None else carried[:n] + s["dy"][at].to(D)
        i = torch.sigmoid(-gate[at].to(D))
        before = s["y"][at - 1].to(D) if t > 0 else h0[by.indices[:n]]
        both[at, :C] = d * i * torch.sigmoid(gate[at].to(D)) * (before - x[at].to(D))
        both[at, C:] = d * i
        carried[:n] = d * torch.sigmoid(gate[at].to(D))
    dh0 = torch.empty_like(carried)
    dh0[by.indices] = carried
    return dict(dboth=both, dh0=dh0 if s["h0"] is not None else None)


def _dropout_exact(s, dev):
    """Bit by bit as published: the products' upper halves from 16-bit parts, in pieces of 2^25 elements."""
    def product(m, v):
        a, b = m * (v & 0xFFFF), m * (v >> 16)
        upper = (b + (a >> 16)) >> 16
        return upper, (a + ((b & 0xFFFF) << 16)) & 0xFFFFFFFF

    n, limit = s["n"], _threshold(s["rate"])
    out = torch.empty(n, dtype=torch.float64, device=dev)
    for lo in range(0, n, 1 << 25):
        hi = min(n, lo + (1 << 25))
        block = torch.arange(lo // 8, (hi + 7) // 8, device=dev)
        c0, c1 = block % (1 << 32), torch.div(block, 1 << 32, rounding_mode="floor")
        c2, c3 = (torch.zeros_like(block) + v for v in (s["offset"] % (1 << 32), s["offset"] // (1 << 32) % (1 << 32)))
        for r in range(10):
            k0 = (s["seed"] + r * 0x9E3779B9) % (1 << 32)
            k1 = (s["seed"] // (1 << 32) + r * 0xBB67AE85) % (1 << 32)
            (h0, l0), (h1, l1) = product(0xD2511F53, c0), product(0xCD9E8D57, c2)
            c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        word = torch.stack([c0, c1, c2, c3], 1).reshape(-1, 1)
        u = torch.cat([word % 65536, word // 65536], 1).reshape(-1)[:hi - lo]
        kept = s["x"][lo:hi].double() * (u >= limit) * 65536 / (65536 - limit)
        out[lo:hi] = kept if s["residual"] is None else kept + s["residual"][lo:hi].double()
    return out
