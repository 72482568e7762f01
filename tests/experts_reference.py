"""The operators of a length predictor from their definitions, in 64 bits on the CPU (numpy), and how far a result in fewer bits may be
off.  Shares no code with the library.

Tolerances.  A result of type t is rounded once: u(t) times itself (2^-24, 2^-8, 2^-11), or half the smallest number of the type.  Before
that it is a sum of n products in single precision: at most (n + 8) roundings (or truncations: 2^-23 each) of the sum of their
magnitudes, the eight for what an element passes through besides (a bias, a weight, a quotient, an exponential)."""
import numpy as np
import torch

UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
LEAST = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -25}


def f64(t):
    return t.detach().double().cpu().numpy()


def close(got, ref, dtype, magnitude=0.0, n=0, where=""):
    """|got - ref| within what n products whose magnitudes add up to `magnitude` and one rounding allow."""
    g = f64(got)
    assert g.shape == np.shape(ref), (where, g.shape, np.shape(ref))
    tol = (n + 8) * 2.0 ** -23 * np.asarray(magnitude) + UNIT[dtype] * np.abs(ref) * (1 + 1e-3) + LEAST[dtype]
    with np.errstate(invalid="ignore"):
        bad = ~(np.abs(g - ref) <= tol) & ~(np.isnan(g) & np.isnan(ref)) & ~(g == ref)
    assert not bad.any(), (where, int(bad.sum()), np.argwhere(bad)[:3].tolist(), g[bad][:3], np.asarray(ref)[bad][:3])


def scores(x, scoring):
    """Scores of every row of logits x."""
    with np.errstate(over="ignore", invalid="ignore"):
        if scoring == "sigmoid":
            return 1 / (1 + np.exp(-x))
        m = x.max(1, keepdims=True)
        e = np.where(np.isneginf(x), 0, np.exp(x - np.where(np.isneginf(m), 0, m)))
        s = e.sum(1, keepdims=True)
        return np.divide(e, s, out=np.zeros_like(e), where=s != 0)


def route(x, k, bias, scoring, n_group, kept, renorm, scale):
    """Weights and experts, row by row, by sorting in Python (first by score, then by index)."""
    s_all = scores(x, scoring)
    T, E = x.shape
    w, ids = np.zeros((T, k)), np.full((T, k), -1)
    size = E // n_group
    for t in range(T):
        s = s_all[t]
        c = [-np.inf if np.isneginf(x[t, e]) else s[e] + (0 if bias is None else bias[e]) for e in range(E)]
        groups = []
        for g in range(n_group):
            best = sorted((v for v in c[g * size:(g + 1) * size] if v > -np.inf), reverse=True)[:2]
            if best:
                groups.append((-sum(best), g))
        allowed = {g for _, g in sorted(groups)[:kept]}
        order = sorted((-c[e], e) for e in range(E) if c[e] > -np.inf and e // size in allowed)[:k]
        for j, (_, e) in enumerate(order):
            ids[t, j], w[t, j] = e, s[e]
        if renorm and w[t].sum() != 0:
            w[t] /= w[t].sum()
    return w * scale, ids


def route_backward(x, ids, u, scoring, renorm, scale):
    """By the matrix of derivatives of the weights, built up row by row.  (Shares of a softmax among the chosen are the softmax of the
    chosen: taken as that, experts that are not chosen have a gradient of 0 here too, and not what is left of 1 - 1.)"""
    if scoring == "softmax" and renorm:
        chosen = np.zeros(x.shape, dtype=bool)
        for t, j in zip(*np.nonzero((ids >= 0) & (ids < x.shape[1]))):
            chosen[t, ids[t, j]] = True
        x, renorm = np.where(chosen, x, -np.inf), False
    s_all = scores(x, scoring)
    out = np.zeros_like(x)
    for t in range(x.shape[0]):
        s = s_all[t]
        js = [j for j in range(ids.shape[1]) if 0 <= ids[t, j] < x.shape[1]]
        ds = np.zeros_like(s)                      # by the scores
        r = sum(s[ids[t, j]] for j in js)
        for j in js:
            e = ids[t, j]
            if not renorm:
                ds[e] += scale * u[t, j]
            elif r != 0:
                ds[e] += scale * u[t, j] / r
                for i in js:
                    ds[ids[t, i]] -= scale * u[t, j] * s[e] / r ** 2
        jac = np.diag(s * (1 - s)) if scoring == "sigmoid" else np.diag(s) - np.outer(s, s)
        out[t] = jac @ ds
    return out


def plan(ids, n_expert):
    flat = ids.reshape(-1)
    e = np.where((flat >= 0) & (flat < n_expert), flat, n_expert)
    order = np.argsort(e, kind="stable")
    off = np.concatenate([[0], np.cumsum(np.bincount(e, minlength=n_expert + 1)[:n_expert])])
    kept = np.arange(len(flat)) < off[-1]
    pos = np.full(len(flat), -1)
    pos[order[kept]] = np.arange(off[-1])
    return off, np.where(kept, order, -1 - order), pos.reshape(ids.shape)


def row_of(slot, top_k, n):
    if slot is None:
        return np.arange(n)
    return np.where(slot < 0, -1 - slot, slot) // top_k


def linear(x, w, b, off, slot, top_k, relu, n):
    """y and the sums of the magnitudes behind it."""
    row = row_of(slot, top_k, n)
    y, size = np.zeros((n, w.shape[1])), np.zeros((n, w.shape[1]))
    for e in range(len(off) - 1):
        p = slice(off[e], off[e + 1])
        y[p] = x[row[p]] @ w[e].T + b[e]
        size[p] = np.abs(x[row[p]]) @ np.abs(w[e]).T + np.abs(b[e])
    return np.where(y < 0, 0, y) if relu else y, size


def linear_backward(x, w, dz, off, slot, top_k):
    """dx, dW, db, each with the sums of the magnitudes behind it."""
    n = dz.shape[0]
    row = row_of(slot, top_k, n)
    dx, dw, db = np.zeros((n, w.shape[2])), np.zeros(w.shape), np.zeros(w.shape[:2])
    m_dx, m_dw, m_db = np.zeros_like(dx), np.zeros_like(dw), np.zeros_like(db)
    for e in range(len(off) - 1):
        p = slice(off[e], off[e + 1])
        dx[p], m_dx[p] = dz[p] @ w[e], np.abs(dz[p]) @ np.abs(w[e])
        dw[e], m_dw[e] = dz[p].T @ x[row[p]], np.abs(dz[p]).T @ np.abs(x[row[p]])
        db[e], m_db[e] = dz[p].sum(0), np.abs(dz[p]).sum(0)
    return (dx, m_dx), (dw, m_dw), (db, m_db)
