"""The operators that read a request's tokens from their definitions, in 64 bits on the CPU (numpy), and how far results in fewer bits may be
off.  Shares no code with the library.

Tolerances of the recurrence.  A gate's smaller sigmoid is off by at most 4 units of 2^-23, relative (an exponential's unit and its
correction's half, the sum's half, a reciprocal's unit, a product's half), the larger one, what it leaves of 1, by no more.  A step adds two
roundings.  With M_t = f_t M_{t-1} + i_t |x_t| the sum of magnitudes behind a state, a step
puts an error of at most k M_t there, and it goes on as the state does: in all k E_t with E_t = f_t E_{t-1} + M_t.  Stretches that are joined (a state
times a product of f) have the roundings of the product besides, one a step and one a join: twice as many at most.  k = 2 * (4 + 4 + 2) * 2^-23, which is 20 units.
Gradients likewise, backward, with one more product or three."""
import numpy as np

from tests.experts_reference import LEAST, UNIT, f64

K = 20


def sigmoids(g):
    with np.errstate(over="ignore"):
        return 1 / (1 + np.exp(-g)), 1 / (1 + np.exp(g))


def ranges(off, n):
    return [(t, t + 1) for t in range(n)] if off is None else list(zip(off[:-1], off[1:]))


def scan(gate, x, off, h0):
    """y, last states, and E of each."""
    f, i = sigmoids(gate)
    n, W = gate.shape
    seqs = ranges(off, n)
    y, E_y = np.full((n, W), np.nan), np.zeros((n, W))
    last, E_last = np.zeros((len(seqs), W)), np.zeros((len(seqs), W))
    for s, (a, b) in enumerate(seqs):
        h = np.zeros(W) if h0 is None else h0[s].copy()
        M, E = np.abs(h), np.zeros(W)
        for t in range(a, b):
            h = f[t] * h + i[t] * x[t]
            M = f[t] * M + i[t] * np.abs(x[t])
            E = f[t] * E + M
            y[t], E_y[t] = h, E
        last[s], E_last[s] = h, E
    return y, last, E_y, E_last


def scan_backward(gate, x, y, off, h0, dy, dh):
    """dgate, dx, dh0, and E of each."""
    f, i = sigmoids(gate)
    n, W = gate.shape
    seqs = ranges(off, n)
    dgate, dx, E_dgate, E_dx = (np.zeros((n, W)) for _ in range(4))
    dh0, E_dh0 = np.zeros((len(seqs), W)), np.zeros((len(seqs), W))
    for s, (a, b) in enumerate(seqs):
        c = np.zeros(W) if dh is None else dh[s].copy()
        M, E = np.abs(c), np.zeros(W)
        for t in range(b - 1, a - 1, -1):
            up = np.zeros(W) if dy is None else dy[t]
            d, M = c + up, M + np.abs(up)
            E = E + M
            before = y[t - 1] if t > a else np.zeros(W) if h0 is None else h0[s]
            dx[t], E_dx[t] = i[t] * d, i[t] * E
            dgate[t] = f[t] * i[t] * d * (before - x[t])
            E_dgate[t] = 2 * f[t] * i[t] * E * (np.abs(before) + np.abs(x[t]))
            c, M, E = f[t] * d, f[t] * M, f[t] * E
        dh0[s], E_dh0[s] = c, E
    return (dgate, E_dgate), (dx, E_dx), (dh0, E_dh0)


def near(got, ref, E, dtype, what):
    """|got - ref| within k E and one rounding; the same places not finite."""
    import torch
    g = f64(got)
    assert g.shape == ref.shape, (what, g.shape, ref.shape)
    out = torch.float32 if got.dtype == torch.float32 else dtype
    # (behind a gate of 87 the smaller sigmoid is past single precision's range of full digits, 2^-126)
    tol = K * 2.0 ** -23 * E + UNIT[out] * np.abs(ref) * (1 + 1e-3) + LEAST[out] + 2.0 ** -120
    bad = ~(np.abs(g - ref) <= tol)
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[:3].tolist(), g[bad][:3], ref[bad][:3], tol[bad][:3])


def embed_backward(token, dout, vocab, scale):
    """The sums, those of the magnitudes, and how many rows each token has."""
    ok = (token >= 0) & (token < vocab)
    out, size = np.zeros((vocab, dout.shape[1])), np.zeros((vocab, dout.shape[1]))
    np.add.at(out, token[ok], dout[ok])
    np.add.at(size, token[ok], np.abs(dout[ok]))
    return out * scale, size * abs(scale), np.bincount(token[ok], minlength=vocab)


def philox(counter, key):
    """Four words from a counter of four words and a key of two, arrays of whole numbers in Python's own arithmetic's range."""
    c, k = [np.asarray(v, dtype=object) for v in counter], [int(v) for v in key]
    for _ in range(10):
        p, q = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [q >> 32 ^ c[1] ^ k[0], q & 0xFFFFFFFF, p >> 32 ^ c[3] ^ k[1], p & 0xFFFFFFFF]
        k = [k[0] + 0x9E3779B9 & 0xFFFFFFFF, k[1] + 0xBB67AE85 & 0xFFFFFFFF]
    return c


def random_bits(index, seed, offset):
    """The 16 random bits of elements `index`."""
    low = 0xFFFFFFFF
    block, part = [int(i) >> 3 for i in index], np.asarray([int(i) & 7 for i in index])
    full = lambda v: np.full(len(index), v, dtype=object)
    words = philox([np.array([b & low for b in block], dtype=object), np.array([b >> 32 for b in block], dtype=object), full(offset & low),
                    full(offset >> 32)], (seed & low, seed >> 32))
    word = np.stack([w.astype(np.int64) for w in words])[part // 2, np.arange(len(index))]
    return word >> (16 * (part % 2)) & 0xFFFF
