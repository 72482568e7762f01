"""The choice of experts and its gradient where single precision has little left: scores far below a row's largest, sigmoids near one."""
import numpy as np
import pytest
import torch

from paper_2605_16867_amd import binding
from tests import experts_reference as ref
from tests.test_gpu_experts import TYPES, empty, f64_of, ints, put, run_route

pytestmark = pytest.mark.gpu


def faint_logits(rng, T, E, k, dtype, scoring):
    """Rows of which a bias chooses k experts whose scores are between the least numbers of single precision and its least ones of full
    precision; another expert has nearly all of a softmax."""
    x = rng.uniform(-103, -86, (T, E)) if scoring == "softmax" else rng.uniform(-103, -70, (T, E))
    bias = np.zeros(E)
    chosen = rng.permutation(E)[:k]
    bias[chosen] = 2.0 + np.arange(k)
    x[:, chosen[0]] = rng.uniform(-100, -85, T) if scoring == "softmax" else rng.uniform(-88, -60, T)
    if scoring == "softmax":
        x[:, np.setdiff1d(np.arange(E), chosen)[0]] = 0
    return f64_of(x, dtype), bias


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scale", [1.0, 2.5, 1e30])
@pytest.mark.parametrize("E,k", [(9, 2), (3, 2), (64, 8), (64, 1), (200, 5), (512, 16)])
@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
def test_shares_of_faint_scores(scoring, E, k, scale, dtype):
    """Weights of experts that a bias chose far below the row's largest logit are their shares all the same, and so is the gradient."""
    rng = np.random.default_rng(E + k)
    T = 70
    x, bias = faint_logits(rng, T, E, k, dtype, scoring)
    w, ids, _ = run_route(x, k, dtype, bias=bias, scoring=scoring, renorm=True, scale=scale)
    rw, rids = ref.route(x, k, bias, scoring, 1, 1, True, scale)
    assert np.array_equal(ids, rids)
    ref.close(w, rw, torch.float32, magnitude=rw, n=k + 8)
    u = f64_of(rng.normal(size=(T, k)), torch.float32)
    out, h = empty(T, E, dtype=torch.float32), binding.Experts(E, T, k)
    h.gr_expert_route_backward(put(x, torch.float32), ints(ids), put(u, torch.float32), out, scoring=scoring, renormalise=True, scale=scale)
    r = ref.route_backward(x, ids, u, scoring, True, scale)
    rows = np.arange(T)[:, None]
    size = np.zeros((T, E))
    size[rows, ids] = rw * (np.abs(u) + (np.abs(u) * rw / scale).sum(1, keepdims=True))
    ref.close(out, r, torch.float32, magnitude=size, n=k + 16)


@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
def test_a_large_scale_of_shares(scoring):
    """scale times a share, not the quotient of scale and the sum, is what has to be a number."""
    rng = np.random.default_rng(1)
    x = f64_of(rng.normal(size=(33, 512)) * 0.1, torch.float32)
    w, ids, _ = run_route(x, 2, torch.float32, scoring=scoring, renorm=True, scale=3e38)
    rw, rids = ref.route(x, 2, None, scoring, 1, 1, True, 3e38)
    assert np.array_equal(ids, rids)
    ref.close(w, rw, torch.float32, magnitude=rw, n=512)


@pytest.mark.parametrize("renorm", [False, True])
def test_gradient_of_sigmoids_near_one(renorm):
    """1 - s of a large logit is not what single precision leaves of the difference."""
    rng = np.random.default_rng(2)
    T, E, k = 50, 24, 5
    x = f64_of(rng.choice([-20, -16, -12, -3, 0, 3, 12, 16, 20, 30, 60], (T, E)) + rng.normal(size=(T, E)), torch.float32)
    ids = np.stack([rng.permutation(E)[:k] for _ in range(T)])
    u = f64_of(rng.normal(size=(T, k)), torch.float32)
    out, h = empty(T, E), binding.Experts(E, T, k)
    h.gr_expert_route_backward(put(x, torch.float32), ints(ids), put(u, torch.float32), out, scoring="sigmoid", renormalise=renorm)
    s = 1 / (1 + np.exp(-x))
    q = 1 / (1 + np.exp(x))
    rows = np.arange(T)[:, None]
    p, c = s[rows, ids], q[rows, ids]
    if renorm:
        p = p / p.sum(1, keepdims=True)
        d = p * c * (u - (u * p).sum(1, keepdims=True))
        size = p * c * (np.abs(u) + (np.abs(u) * p).sum(1, keepdims=True))
    else:
        d = p * c * u
        size = np.abs(d)
    r, m = np.zeros((T, E)), np.zeros((T, E))
    r[rows, ids], m[rows, ids] = d, size
    # (an exponent of up to 60 magnifies the rounding of x log2(e): 60 units more)
    ref.close(out, r, torch.float32, magnitude=m, n=k + 64)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("with_bias", [False, True])
def test_masks_of_the_types_lowest_value(with_bias, scoring, dtype):
    """They are logits like others: chosen where nothing else is left, with a score of 0 beside any other, and equal among themselves."""
    rng = np.random.default_rng(11)
    T, E, k = 60, 24, 6
    x = (np.stack([rng.permutation(E) for _ in range(T)]) - E / 2) * 0.125
    low = float(torch.finfo(dtype).min)
    x[rng.random((T, E)) < 0.5] = low
    x[3], x[4, 1:], x[5], x[6, :4] = low, low, low, -np.inf
    x[5, 7] = -np.inf
    x = f64_of(x, dtype)
    bias = 2.0 * rng.permutation(E) if with_bias else None
    for renorm in (False, True):
        w, ids, _ = run_route(x, k, dtype, bias=bias, scoring=scoring, renorm=renorm)
        rw, rids = ref.route(x, k, bias, scoring, 1, 1, renorm, 1.0)
        assert np.array_equal(ids, rids)
        ref.close(w, rw, torch.float32, magnitude=rw, n=E + 8)
        u = f64_of(rng.normal(size=(T, k)), torch.float32)
        out, h = empty(T, E, dtype=torch.float32), binding.Experts(E, T, k)
        h.gr_expert_route_backward(put(x, dtype).float(), ints(ids), put(u, torch.float32), out, scoring=scoring, renormalise=renorm)
        with np.errstate(over="ignore"):
            r = ref.route_backward(x, ids, u, scoring, renorm, 1.0)
            s = ref.scores(x, scoring)
        big = np.abs(u).sum(1, keepdims=True)
        if scoring == "softmax" and renorm:      # (chosen of nothing but the lowest value beside others: a sum of 0 in single precision has no shares)
            total = np.array([s[t, ids[t][ids[t] >= 0]].sum() for t in range(T)])
            r[total == 0], s = 0, np.ones_like(s)
        elif renorm:
            s = np.ones_like(s)
        ref.close(out, r, torch.float32, magnitude=np.abs(s) * 2 * big, n=E + 16)
