"""The length predictor end to end: its forward pass against the same network in 64 bits, its gradients through all operators
against differences, training in two phases, and its lengths in a routing call."""
import numpy as np
import pytest
import torch

from paper_2605_16867_amd import binding, predictor, workloads
from tests import experts_reference as ref
from tests import parity

pytestmark = pytest.mark.gpu


def _network(p, x):
    """Logarithms of lengths from the predictor's weights, in 64 bits on the CPU."""
    x = ref.f64(x)
    w, b = [ref.f64(t) for t in p.w], [ref.f64(t) for t in p.b]
    (r0, r1), (s0, s1) = [ref.f64(t) for t in p.router_w], [ref.f64(t) for t in p.router_b]
    share, ids = ref.route(np.maximum(x @ r0.T + s0, 0) @ r1.T + s1, p.top_k, None, "softmax", 1, 1, True, 1.0)
    out = np.zeros((len(x), 1))
    for e in range(p.n_expert):
        v = x
        for i in range(len(w)):
            v = v @ w[i][e].T + b[i][e]
            v = np.maximum(v, 0) if i < len(w) - 1 else v
        out += (share * (ids == e)).sum(1)[:, None] * v
    return out


@pytest.mark.parametrize("top_k", [9, 2])
@pytest.mark.parametrize("rows", [1, 7, 130])
def test_forward(rows, top_k):
    p = predictor.LengthPredictor(40, hidden=(32, 24, 16), router_hidden=24, top_k=top_k, max_rows=130, dtype=torch.float32)
    x, _, _ = predictor.synthetic_requests(rows, 40, 9, seed=3, dtype=torch.float32)
    got = ref.f64(p.forward(x))
    # single precision through six products of some 40 terms of order 1: 1e-6 each of results of order 1 to 10
    assert np.abs(got - _network(p, x)).max() < 1e-4
    for max_len in (1, 50, 4096):
        n = p.predict(x, max_len)
        assert n.dtype == torch.int32 and n.shape == (rows,) and int(n.min()) >= 1 and int(n.max()) <= max_len


def test_gradients_through_all_operators():
    """A step with rate 1 and no clipping moves every weight by its gradient: against differences of the loss in 64 bits."""
    for phase in ("experts", "router"):
        p = predictor.LengthPredictor(10, n_expert=3, hidden=(9, 8, 6), router_hidden=7, max_rows=50, dtype=torch.float32, max_norm=float("inf"))
        x, target, kind = predictor.synthetic_requests(50, 10, 3, seed=8, dtype=torch.float32)
        t = ref.f64(target)

        def loss():
            if phase == "router":
                return ((_network(p, x).reshape(-1) - t) ** 2).mean()
            v, k = ref.f64(x), kind.cpu().numpy()
            for i in range(4):
                v = np.stack([ref.f64(p.w[i][e]) @ row + ref.f64(p.b[i][e]) for row, e in zip(v, k)])
                v = np.maximum(v, 0) if i < 3 else v
            return ((v.reshape(-1) - t) ** 2).mean()

        tensors = p.w + p.b if phase == "experts" else p.router_w + p.router_b
        before = [w.clone() for w in tensors]
        value = p.train_experts(x, target, kind, 1.0) if phase == "experts" else p.train_router(x, target, 1.0)
        moved = [b - w for b, w in zip(before, tensors)]
        for w, b in zip(tensors, before):
            w.copy_(b)
        assert abs(float(value) - loss()) < 1e-4 * loss()
        rng = np.random.default_rng(0)
        for w, m in zip(tensors, moved):
            flat, step = w.view(-1), 2.0 ** -9
            for i in rng.choice(flat.numel(), min(6, flat.numel()), replace=False):
                keep = float(flat[i])
                flat[i] = keep + step
                up_at, up = float(flat[i]), loss()
                flat[i] = keep - step
                diff = (up - loss()) / (up_at - float(flat[i]))
                flat[i] = keep
                # differences over 2^-8 of a loss whose kinks a step may cross: a few of a hundred of the largest gradient
                assert abs(float(m.view(-1)[i]) - diff) < 0.05 * max(1.0, float(m.abs().max())), (phase, w.shape, i)


def test_two_phases_and_a_routing_call():
    p = predictor.LengthPredictor(128, hidden=(64, 32, 16), router_hidden=32, max_rows=4096)
    first = last = None
    for phase, rate in (("experts", 0.05), ("router", 0.2)):
        losses = []
        for step in range(60):
            x, target, kind = predictor.synthetic_requests(1024, 128, 9, seed=step)
            losses.append(p.train_experts(x, target, kind, rate) if phase == "experts" else p.train_router(x, target, rate))
        losses = [float(v) for v in losses]
        assert all(np.isfinite(losses)) and np.mean(losses[-5:]) < 0.7 * np.mean(losses[:5]), (phase, losses)
    fl = workloads.make_fleet(workloads.spec("mid"))
    d, h = parity.upload(fl, "cuda:0"), parity.make_handle(fl)
    fin = torch.empty(len(fl.act_prompt), dtype=torch.float32, device="cuda:0")
    h.gr_build_status(d["act_off"], d["act_prompt"], d["act_gen"], d["act_rem"], d["q_off"], d["q_prompt"], d["q_len"], fin)
    x, _, _ = predictor.synthetic_requests(len(fl.in_prompt), 128, 9, seed=999)
    length = p.predict(x, int(fl.spec.max_len))
    inst, slack = torch.full_like(length, -7), torch.empty(len(length), dtype=torch.float32, device="cuda:0")
    h.gr_score_route(d["in_prompt"], length, d["in_budget"], inst, slack)
    assert int(inst.min()) >= 0 and int(inst.max()) < fl.n_inst and h.gr_device_status() == 0
    assert bool(torch.isfinite(slack).all())


def test_as_by_ctypes(monkeypatch):
    """The native marshalling and the binding's own give the same bits."""
    outs = []
    for native in (True, False):
        if not native:
            monkeypatch.setattr(binding, "_marshal", binding._Ctypes)
        p = predictor.LengthPredictor(64, hidden=(48, 32, 8), router_hidden=16, top_k=3, max_rows=200)
        for step in range(3):
            x, target, kind = predictor.synthetic_requests(200, 64, 9, seed=step)
            p.train_experts(x, target, kind, 0.05)
            p.train_router(x, target, 0.1)
        outs.append([t.clone() for t in (*p.w, *p.b, *p.router_w, *p.router_b, p.forward(x))])
    for a, b in zip(*outs):
        assert torch.equal(a, b)
