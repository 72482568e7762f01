"""Prompts to features to lengths: the reader's states against the same network in 64 bits, its gradients through all operators against
differences, a prompt read in parts and token by token, training steps, and its lengths in the routing calls."""
import numpy as np
import pytest
import torch

from paper_2605_16867_amd import binding, predictor, reader
from tests import experts_reference as ref
from tests import tokens_reference

pytestmark = pytest.mark.gpu


def _states(r, token, off, start=None):
    """States from the reader's weights, in 64 bits on the CPU."""
    table, w, b = ref.f64(r.table), ref.f64(r.w), ref.f64(r.b)
    t = token.cpu().numpy()
    ok = (t >= 0) & (t < r.n_vocab)
    rows = np.where(ok[:, None], table[np.clip(t, 0, r.n_vocab - 1)] * r.scale, 0)
    both = rows @ w.T + b
    return tokens_reference.scan(both[:, :r.n_out], both[:, r.n_out:], off.cpu().numpy(), start)[1]


def _small(dtype=torch.float32, drop=0.0, **more):
    return reader.PromptReader(60, 24, width=20, max_tokens=600, max_rows=40, drop=drop, dtype=dtype, **more)


def _prompts(rows, seed, n_vocab=60):
    return reader.synthetic_prompts(rows, n_vocab, 3, 9, seed=seed)


@pytest.mark.parametrize("rows", [1, 5, 30])
def test_states(rows):
    r = _small()
    token, off, _, _ = _prompts(rows, seed=rows)
    token[::7] = -1
    got = r.read(token, off)
    # single precision: sums of 20 terms of order 1 in a gate and a value, states that forget in up to 500 tokens
    assert np.abs(ref.f64(got) - _states(r, token, off)).max() < 1e-4
    # gone on from there
    more, more_off, _, _ = _prompts(rows, seed=rows + 50)
    again = r.read(more, more_off, start=got)
    assert np.abs(ref.f64(again) - _states(r, more, more_off, ref.f64(got))).max() < 1e-4


def test_token_by_token_as_at_once():
    """A request of 40 tokens read whole, and its first 30 read, then one after the other: the same states up to the roundings of a different order."""
    r = _small()
    g = torch.Generator().manual_seed(1)
    prompts = torch.randint(0, 60, (12, 40), generator=g, dtype=torch.int32).to(r.dev)
    off = torch.arange(13, dtype=torch.int32, device=r.dev)
    whole = r.read(prompts.view(-1), off * 40)
    state = r.read(prompts[:, :30].contiguous().view(-1), off * 30)
    for t in range(30, 40):
        r.advance(prompts[:, t].contiguous(), state)
    assert float((state - whole).abs().max()) < 1e-5


def test_reading_between_a_batch_and_its_gradient():
    """Arrivals are read, what runs moves on, while a batch waits for its gradient: the gradient is the batch's all the same."""
    token, off, _, _ = _prompts(12, seed=4)
    others, their_off, _, _ = _prompts(30, seed=77)
    grads = []
    for reads in (False, True):
        r = _small(drop=0.3)
        x = r.train_forward(token, off)
        kept = x.clone()
        if reads:
            state = r.read(others, their_off)
            r.advance(others[:30].contiguous(), state)
        assert torch.equal(x, kept)
        r.backward(token, off, torch.ones_like(x))
        grads.append([t.clone() for t in (r.dtable, r.dw, r.db)])
    for a, b in zip(*grads):
        assert torch.equal(a, b)


@pytest.mark.parametrize("drop", [0.0, 0.3])
def test_gradients_through_all_operators(drop):
    """The gradient of a loss by table, product and bias: against differences of the loss in 64 bits, the same elements dropped."""
    r = _small(drop=drop, max_norm=float("inf"))
    token, off, _, _ = _prompts(12, seed=4)
    token[5] = -1
    rng = np.random.default_rng(2)
    u = rng.normal(size=(12, r.n_out))
    x = r.train_forward(token, off)
    kept = np.ones(x.shape) if drop == 0 else (tokens_reference.random_bits(range(x.numel()), r.seed, 1) >= round(drop * 65536)).reshape(x.shape)
    scale = 65536 / (65536 - round(drop * 65536))
    assert np.array_equal(ref.f64(x) != 0, kept != 0)

    def loss():
        return (_states(r, token, off) * kept * scale * u).sum()

    d = torch.from_numpy(u).float().to(r.dev)
    r.backward(token, off, d)
    for p, g in ((r.table, r.dtable), (r.w, r.dw), (r.b, r.db)):
        flat, grad = p.view(-1), ref.f64(g).reshape(-1)
        most = np.abs(grad).max()
        for i in rng.choice(flat.numel(), min(12, flat.numel()), replace=False):
            keep, step, both = float(flat[i]), 2.0 ** -10, []
            for s in (step, -step):
                flat[i] = keep + s
                both.append((loss(), float(flat[i])))
            flat[i] = keep
            diff = (both[0][0] - both[1][0]) / (both[0][1] - both[1][1])
            # differences over 2^-9 of a smooth loss: third derivatives of order 100 at 1e-3 squared are 1e-4 of the largest
            assert abs(grad[i] - diff) < 2e-3 * max(1.0, most), (i, grad[i], diff)


def test_the_predictors_gradient_by_its_features():
    """What `train_experts` gives out beside its own step: against differences of its loss."""
    p = predictor.LengthPredictor(10, n_expert=3, hidden=(9, 8, 6), router_hidden=7, max_rows=40, dtype=torch.float32)
    x, target, kind = predictor.synthetic_requests(40, 10, 3, seed=8, dtype=torch.float32)
    kind[3], kind[9] = -1, 7
    t, v, e = ref.f64(target), ref.f64(x), kind.cpu().numpy()
    w, b = [ref.f64(a) for a in p.w], [ref.f64(a) for a in p.b]
    some = (e >= 0) & (e < 3)

    def loss():
        out = 0.0
        for row, k, y in zip(v[some], e[some], t[some]):
            for i in range(4):
                row = w[i][k] @ row + b[i][k]
                row = np.maximum(row, 0) if i < 3 else row
            out += (row[0] - y) ** 2
        return out / some.sum()

    dx = torch.full_like(x, 77)
    alone = predictor.LengthPredictor(10, n_expert=3, hidden=(9, 8, 6), router_hidden=7, max_rows=40, dtype=torch.float32)
    first = alone.train_experts(x, target, kind, 0.1)
    assert torch.equal(first, p.train_experts(x, target, kind, 0.1, out_dx=dx))
    for a, c in zip(alone.w + alone.b, p.w + p.b):      # (its own step is the same)
        assert torch.equal(a, c)
    g = ref.f64(dx)
    assert (g[~some] == 0).all()
    rng = np.random.default_rng(0)
    for r, c in zip(rng.integers(0, 40, 30), rng.integers(0, 10, 30)):
        keep, step, both = v[r, c], 2.0 ** -9, []
        for s in (step, -step):
            v[r, c] = keep + s
            both.append(loss())
        v[r, c] = keep
        # (as for the predictor's weights: kinks that a step may cross)
        assert abs((both[0] - both[1]) / (2 * step) - g[r, c]) < 0.05 * max(1.0, np.abs(g).max())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_training_steps_and_the_routing_calls(dtype, capsys, monkeypatch):
    """Steps run, leave every weight a number and move all of them; the same steps give the same bits."""
    seen = []
    for _ in range(2):
        r = reader.PromptReader(500, 64, width=48, max_tokens=1 << 14, max_rows=300, dtype=dtype)
        p = predictor.LengthPredictor(64, hidden=(32, 24, 16), router_hidden=24, max_rows=300, dtype=dtype)
        before = [t.clone() for t in (r.table, r.w, r.b)]
        for step in range(4):
            token, off, target, kind = reader.synthetic_prompts(256, 500, 9, 20, seed=step)
            loss = reader.train(r, p, token, off, target, kind, 0.05, 0.2)
            assert bool(torch.isfinite(loss)) and bool(torch.isfinite(r.norm))
        for b, t in zip(before, (r.table, r.w, r.b)):
            assert bool(torch.isfinite(t).all()) and not torch.equal(b, t)
        seen.append([t.clone() for t in (r.table, r.w, r.b, *p.w, *p.b)])
    for a, b in zip(*seen):
        assert torch.equal(a, b)


def test_the_command(capsys):
    reader.main()
    said = capsys.readouterr().out
    assert "arrivals of" in said and "running requests re-checked" in said and "nan" not in said
