"""The operators of a length predictor (choice of experts, layers of all experts, weighted sum, clipping) against their definitions in 64
bits: sizes around the edges of tiles and units, masks, ties, rows and experts with nothing, values that are no numbers, the largest
offsets; gradients against the formulas and against differences; refusals."""
import numpy as np
import pytest
import torch

from paper_2605_16867_amd import binding
from tests import experts_reference as ref

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]
INF, NAN = float("inf"), float("nan")


def put(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV).to(dtype).contiguous()


def ints(a):
    return put(np.asarray(a, dtype=np.int32), torch.int32)


def empty(*shape, dtype=torch.float32):
    """Outputs start as something that no result is."""
    return torch.full(shape, 77, dtype=dtype, device=DEV)


def shifted(t, by=1):
    """The same values at an address `by` elements off a boundary of 16 bytes."""
    buf = torch.empty(t.numel() + by, dtype=t.dtype, device=t.device)
    buf[by:] = t.reshape(-1)
    return buf[by:].view(t.shape)


# ---- choice -----------------------------------------------------------------------------------


def spread_logits(rng, T, E, dtype):
    """Rows whose scores are well apart: a row's logits are multiples of 1/8 in random order (exact in every type), in
    a window that softmax and sigmoid still tell apart in single precision."""
    step = 0.125 if E <= 64 else 6.0 / E
    x = (np.stack([rng.permutation(E) for _ in range(T)]) - E / 2) * step if T else np.zeros((0, E))
    return f64_of(x, dtype)


def f64_of(x, dtype):
    return torch.from_numpy(x).to(dtype).double().numpy()


def run_route(x, k, dtype, bias=None, scoring="softmax", n_group=1, kept=1, renorm=False, scale=1.0, shift=False):
    T, E = x.shape
    h = binding.Experts(E, max(T, 1), k)
    w, ids = empty(T, k), empty(T, k, dtype=torch.int32)
    off, slot, pos = empty(E + 1, dtype=torch.int32), empty(T * k, dtype=torch.int32), empty(T, k, dtype=torch.int32)
    logits = put(x, dtype)
    h.gr_expert_route(shifted(logits) if shift else logits, w, ids, off, slot, pos, bias=None if bias is None else put(bias, torch.float32),
                      scoring=scoring, n_group=n_group, n_group_kept=kept, renormalise=renorm, scale=scale)
    return w, ids.cpu().numpy(), (off, slot, pos)


def check_plan(ids, E, got):
    for g, r in zip(got, ref.plan(ids, E)):
        assert np.array_equal(g.cpu().numpy(), r)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 9, 9), (16, 9, 2), (65, 16, 16), (3, 17, 5), (257, 64, 8), (5, 33, 16), (130, 128, 1),
                                   (40, 256, 8), (7, 511, 3), (9, 512, 16)])
def test_choice(T, E, k, dtype):
    rng = np.random.default_rng(T * 1000 + E)
    if dtype != torch.float32 and E > 128:
        pytest.skip("that many scores well apart are not to be had in 16 bits")
    x = spread_logits(rng, T, E, dtype)
    for scoring in ("softmax", "sigmoid"):
        for renorm in (False, True):
            w, ids, order = run_route(x, k, dtype, scoring=scoring, renorm=renorm, scale=1.5, shift=renorm)
            rw, rids = ref.route(x, k, None, scoring, 1, 1, renorm, 1.5)
            assert np.array_equal(ids, rids)
            # (exponents of up to 6 magnify the rounding of x - max)
            ref.close(w, rw, torch.float32, magnitude=rw, n=E + 8)
            check_plan(ids, E, order)


@pytest.mark.parametrize("E,n_group,kept,k", [(64, 8, 3, 6), (16, 16, 2, 2), (16, 4, 1, 3), (33, 3, 2, 16), (512, 32, 5, 16), (9, 9, 4, 4),
                                              (12, 2, 1, 8)])
@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
def test_choice_by_groups_and_bias(E, n_group, kept, k, scoring):
    rng = np.random.default_rng(E + n_group)
    T = 77
    x = spread_logits(rng, T, E, torch.float32)
    x[rng.random((T, E)) < 0.3] = -INF
    x[5] = -INF
    x[6, 1:] = -INF
    bias = f64_of(rng.permutation(E) * 0.37 + 0.01, torch.float32)       # (larger than any difference of scores: these order the experts)
    w, ids, order = run_route(x, k, torch.float32, bias=bias, scoring=scoring, n_group=n_group, kept=kept, renorm=True)
    rw, rids = ref.route(x, k, bias, scoring, n_group, kept, True, 1.0)
    assert np.array_equal(ids, rids)
    assert (ids[5] == -1).all() and ids[6, 0] == (-1 if np.isneginf(x[6, 0]) else 0) and (ids[6, 1:] == -1).all()
    ref.close(w, rw, torch.float32, magnitude=rw, n=E + 8)
    check_plan(ids, E, order)


@pytest.mark.parametrize("E,n_group", [(9, 1), (64, 8), (200, 1)])
def test_equal_scores_go_to_the_lowest_index(E, n_group):
    x = np.zeros((70, E))
    x[1::2, E // 2:] = 1.0
    x[2, :] = -0.0
    for bias in (None, np.zeros(E)):
        for scoring in ("softmax", "sigmoid"):
            _, ids, order = run_route(x, 5, torch.bfloat16, bias=bias, scoring=scoring, n_group=n_group, kept=max(1, n_group // 2))
            assert np.array_equal(ids, ref.route(x, 5, bias, scoring, n_group, max(1, n_group // 2), False, 1.0)[1])
            check_plan(ids, E, order)


def test_scores_that_are_no_numbers():
    x = np.zeros((6, 9))
    x[0, 3] = NAN
    x[1, 4] = INF
    x[2, :] = [-INF, 5, -INF, 1, -INF, -INF, -INF, -INF, -INF]
    x[3, :] = 88.0
    x[4, :] = [-200, 0, 200, -90, 90, 1, 2, 3, 4]
    w, ids, order = run_route(x, 3, torch.float32, scoring="sigmoid", renorm=False)
    assert ids[0].tolist() == [0, 1, 2] and ids[1].tolist() == [4, 0, 1] and ids[2].tolist() == [1, 3, -1]
    assert ids[4].tolist()[:2] in ([2, 4], [2, 8]) and float(w[4, 0]) == 1.0 and float(w[2, 2]) == 0
    w, ids, order = run_route(x, 9, torch.float32, scoring="sigmoid")
    assert ids[0].tolist() == [0, 1, 2, 4, 5, 6, 7, 8, 3] and np.isnan(float(w[0, 8])) and not np.isnan(ref.f64(w[0, :8])).any()
    w, ids, order = run_route(x, 3, torch.float32, renorm=True)
    # a row without a softmax says so, and takes the first experts
    assert np.isnan(ref.f64(w[0])).all() and ids[0].tolist() == [0, 1, 2] and np.isnan(ref.f64(w[1])).all()
    assert ids[2].tolist() == [1, 3, -1] and float(w[2, 2]) == 0
    assert float(w[4, 0]) == 1.0 and ids[4, 0] == 2
    # chosen by the bias, with scores that are zero in single precision: no share of nothing
    bias = np.zeros(9)
    bias[[0, 3]] = 5
    w, ids, _ = run_route(x[4:5], 2, torch.float32, bias=bias, renorm=True)
    assert ids[0].tolist() == [0, 3] and ref.f64(w).tolist() == [[0.0, 0.0]]
    bias[0] = -INF
    _, ids, _ = run_route(x[4:5], 9, torch.float32, bias=bias)
    assert ids[0, 8] == -1 and 0 not in ids[0]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,E,k", [(1, 4, 2), (19, 9, 9), (65, 64, 8), (33, 40, 5), (5, 512, 16)])
@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [False, True])
def test_gradient_of_the_choice(T, E, k, scoring, renorm, dtype):
    rng = np.random.default_rng(E * 7 + k)
    x = f64_of(rng.normal(size=(T, E)) * 1.5, dtype)
    x[rng.random((T, E)) < 0.1] = -INF
    _, ids = ref.route(x, k, None, scoring, 1, 1, renorm, 0.75)
    if T > 2:
        x[2], ids[2] = -INF, -1
    u = f64_of(rng.normal(size=(T, k)), torch.float32)
    given = u.copy()
    given[ids < 0] = NAN
    h = binding.Experts(E, T, k)
    for shift in (False, True):
        out = empty(T, E, dtype=dtype)
        lg = put(x, dtype)
        h.gr_expert_route_backward(shifted(lg) if shift else lg, ints(ids), put(given, torch.float32), out, scoring=scoring,
                                   renormalise=renorm, scale=0.75)
        r = ref.route_backward(x, ids, u, scoring, renorm, 0.75)
        s = ref.scores(x, scoring)
        # the sums it is a difference of: s (|u| + sum |u| s), or the same of shares
        hot = np.zeros((T, E))
        for j in range(k):
            hot[np.arange(T)[ids[:, j] >= 0], ids[ids[:, j] >= 0, j]] = np.abs(u[ids[:, j] >= 0, j])
        if renorm:
            chosen = np.zeros((T, E))
            for j in range(k):
                chosen[np.arange(T)[ids[:, j] >= 0], ids[ids[:, j] >= 0, j]] = 1
            tot = (chosen * s).sum(1, keepdims=True)
            p = np.divide(chosen * s, tot, out=np.zeros_like(s), where=tot > 0)
        else:
            p = s
        ref.close(out, r, dtype, magnitude=0.75 * p * (hot + (hot * p).sum(1, keepdims=True)), n=E + 16)


@pytest.mark.parametrize("E", [1, 2, 9, 64, 65, 512])
@pytest.mark.parametrize("T,k", [(0, 1), (1, 1), (63, 1), (341, 3), (1024, 1), (1025, 1), (5000, 7), (20011, 2)])
def test_order_of_given_experts(T, k, E):
    if k > E:
        pytest.skip("more choices than experts")
    rng = np.random.default_rng(T + E)
    ids = rng.integers(-2, E + 2, (T, k))
    if T > 100:
        ids[50:] = np.where(rng.random((T - 50, k)) < 0.5, E - 1, ids[50:])
    h = binding.Experts(E, max(T, 1), k)
    off, slot, pos = empty(E + 1, dtype=torch.int32), empty(T * k, dtype=torch.int32), empty(T, k, dtype=torch.int32)
    for _ in range(2):
        h.gr_expert_plan(ints(ids).reshape(T, k), off, slot, pos)
        check_plan(ids, E, (off, slot, pos))


# ---- layers -----------------------------------------------------------------------------------


def ranges(rng, n, E, dropped, skew):
    """Offsets of E experts over n positions of which the last `dropped` belong to none; some experts may have none."""
    share = rng.random(E) ** skew
    share[rng.random(E) < 0.25] = 0
    if E == 1 or share.sum() == 0:
        share[:] = 1
    off = np.concatenate([[0], np.round(np.cumsum(share) / share.sum() * (n - dropped))]).astype(int)
    return off


def slots(rng, n, dropped):
    s = rng.permutation(n)
    s[n - dropped:] = -1 - s[n - dropped:]
    return s


LAYERS = [  # positions, experts, in, out, top_k (0: rows are positions)
    (1, 1, 1, 1, 0), (1, 9, 64, 32, 1), (9, 9, 4096, 40, 9), (17, 4, 16, 8, 1), (64, 1, 64, 64, 2), (130, 3, 128, 128, 0),
    (257, 5, 72, 136, 2), (300, 9, 33, 65, 3), (129, 2, 129, 127, 0), (511, 16, 520, 24, 1), (1000, 64, 40, 48, 8),
    (700, 3, 264, 300, 2), (1500, 2, 192, 1, 3), (90, 9, 7, 513, 9), (2000, 2, 1, 3, 0), (513, 9, 256, 264, 9), (3000, 4, 96, 520, 2)]


def layer(rng, n, E, I, O, k, dtype, scale=1.0):
    dropped = n // 7
    off = ranges(rng, n, E, dropped, 2.0)
    slot = slots(rng, n, dropped) if k else None
    rows = -(-n // k) if k else n
    x = f64_of(rng.normal(size=(rows, I)) * scale, dtype)
    w = f64_of(rng.normal(size=(E, O, I)) / I ** 0.5, dtype)
    b = f64_of(rng.normal(size=(E, O)) * 0.1, dtype)
    return off, slot, x, w, b


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,E,I,O,k", LAYERS)
def test_layer(n, E, I, O, k, dtype):
    rng = np.random.default_rng(n + I)
    off, slot, x, w, b = layer(rng, n, E, I, O, k, dtype)
    h = binding.Experts(E, n, 1)
    tx, tw, tb = put(x, dtype), put(w, dtype), put(b, dtype)
    plan = dict(off=ints(off), slot=None if slot is None else ints(slot), top_k=max(k, 1))
    for relu, shift in ((True, False), (False, True)):
        y = empty(n, O, dtype=dtype)
        h.gr_expert_linear(shifted(tx) if shift else tx, shifted(tw) if shift else tw, y, bias=tb if relu else None, relu=relu, **plan)
        r, size = ref.linear(x, w, b if relu else 0 * b, off, slot, max(k, 1), relu, n)
        ref.close(y, r, dtype, size, I)
        again = empty(n, O, dtype=dtype)
        h.gr_expert_linear(tx, tw, again, bias=tb if relu else None, relu=relu, **plan)
        if relu:
            assert torch.equal(y, again)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,E,I,O,k", LAYERS)
def test_gradients_of_a_layer(n, E, I, O, k, dtype):
    rng = np.random.default_rng(n + I + 1)
    off, slot, x, w, b = layer(rng, n, E, I, O, k, dtype)
    dy, y = f64_of(rng.normal(size=(n, O)), dtype), f64_of(np.maximum(rng.normal(size=(n, O)), 0), dtype)
    h = binding.Experts(E, n, 1)
    tx, tw, tdy, ty = (put(a, dtype) for a in (x, w, dy, y))
    plan = dict(off=ints(off), slot=None if slot is None else ints(slot), top_k=max(k, 1))
    for relu, shift in ((True, False), (False, True)):
        dx, dw, db = empty(n, I, dtype=dtype), empty(E, O, I, dtype=dtype), empty(E, O, dtype=dtype)
        dz = empty(n, O, dtype=dtype) if relu else None
        given = [shifted(t) if shift else t for t in (tx, tw, tdy)]
        h.gr_expert_linear_backward(*given, out_dx=dx, out_dw=dw, out_db=db, y=ty if relu else None, out_dz=dz, **plan)
        z = np.where(y > 0, dy, 0) if relu else dy
        if relu:
            assert np.array_equal(ref.f64(dz), z)
        (rx, mx), (rw, mw), (rb, mb) = ref.linear_backward(x, w, z, off, slot, max(k, 1))
        ref.close(dx, rx, dtype, mx, O, "dx")
        ref.close(dw, rw, dtype, mw, n, "dw")
        ref.close(db, rb, dtype, mb, n, "db")
        if relu:      # each alone, the same bits; dz in the place of dy
            for name in ("out_dx", "out_dw", "out_db"):
                full = dict(out_dx=dx, out_dw=dw, out_db=db)[name]
                only = torch.full_like(full, 5)
                d = tdy.clone()
                h.gr_expert_linear_backward(tx, tw, d, y=ty, out_dz=d, **{name: only}, **plan)
                assert torch.equal(only, full) and torch.equal(d, dz)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,E,I,O,k", [  # few features out; rows that are no whole 16 bytes, or shorter than that
    (1, 3, 5, 16, 1), (200, 3, 9, 4, 2), (4099, 9, 100, 1, 9), (333, 5, 2703, 8, 2), (70, 1, 4101, 16, 0), (2500, 64, 31, 2, 4), (129, 7, 33, 12, 1),
    (1000, 2, 8192, 8, 1)])
def test_layers_of_few_features(n, E, I, O, k, dtype):
    test_layer(n, E, I, O, k, dtype)
    test_gradients_of_a_layer(n, E, I, O, k, dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_layers_of_many_tiles(dtype):
    """More large tiles than rounds of them are whole: forward and by input 1 295 to 1 310, by weight 530 (a round is 256)."""
    test_layer(66100, 3, 72, 1032, 2, dtype)
    test_gradients_of_a_layer(66100, 3, 1032, 72, 2, dtype)
    test_gradients_of_a_layer(300, 2, 13320, 1032, 1, dtype)


def test_gradients_of_many_weights():
    """1 060 large tiles by weight."""
    test_gradients_of_a_layer(40, 4, 13320, 1032, 1, torch.bfloat16)


def test_gradients_of_many_weights():
    """1 060 large tiles by weight."""
    test_gradients_of_a_layer(40, 4, 13320, 1032, 1, torch.bfloat16)


def test_one_matrix_for_all_rows():
    rng = np.random.default_rng(3)
    n, I, O = 333, 80, 72
    x, w, b = (f64_of(rng.normal(size=s), torch.bfloat16) for s in ((n, I), (O, I), (O,)))
    h = binding.Experts(9, n, 2)
    y, dx, dw, db = empty(n, O, dtype=torch.bfloat16), empty(n, I, dtype=torch.bfloat16), empty(O, I, dtype=torch.bfloat16), empty(O, dtype=torch.bfloat16)
    tx, tw, tb = (put(a, torch.bfloat16) for a in (x, w, b))
    h.gr_expert_linear(tx, tw, y, bias=tb)
    r, size = ref.linear(x, w[None], b[None], [0, n], None, 1, False, n)
    ref.close(y, r, torch.bfloat16, size, I)
    h.gr_expert_linear_backward(tx, tw, y, out_dx=dx, out_dw=dw, out_db=db)
    (rx, mx), (rw, mw), (rb, mb) = ref.linear_backward(x, w[None], ref.f64(y), [0, n], None, 1)
    ref.close(dx, rx, torch.bfloat16, mx, O)
    ref.close(dw, rw[0], torch.bfloat16, mw[0], n)
    ref.close(db, rb[0], torch.bfloat16, mb[0], n)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("I,O", [(64, 64), (33, 40)])
def test_what_is_no_number_stays_where_it_belongs(I, O, dtype):
    """Rows without an expert are not read as rows of one; a row or weight that is no number spoils what depends on it and no more."""
    rng = np.random.default_rng(8)
    n, E = 200, 3
    off = np.array([0, 70, 70, 190])
    x, w = f64_of(rng.normal(size=(n, I)), dtype), f64_of(rng.normal(size=(E, O, I)), dtype)
    dz = f64_of(rng.normal(size=(n, O)), dtype)
    x[5], x[190:], w[1], dz[190:] = NAN, NAN, NAN, INF
    h = binding.Experts(E, n, 1)
    y, dx, dw, db = empty(n, O, dtype=dtype), empty(n, I, dtype=dtype), empty(E, O, I, dtype=dtype), empty(E, O, dtype=dtype)
    plan = dict(off=ints(off))
    tx, tw, tdz = put(x, dtype), put(w, dtype), put(dz, dtype)
    for relu in (False, True):
        h.gr_expert_linear(tx, tw, y, relu=relu, **plan)
        bad = np.isnan(ref.f64(y)).any(1)
        assert bad[5] and np.isnan(ref.f64(y)[5]).all() and bad.sum() == 1 and (ref.f64(y)[190:] == 0).all()
    h.gr_expert_linear_backward(tx, tw, tdz, out_dx=dx, out_dw=dw, out_db=db, **plan)
    assert np.isfinite(ref.f64(dx)).all() and (ref.f64(dx)[190:] == 0).all()
    assert np.isnan(ref.f64(dw)[0]).all() and (ref.f64(dw)[1] == 0).all() and np.isfinite(ref.f64(dw)[2]).all()
    assert np.isfinite(ref.f64(db)).all() and (ref.f64(db)[1] == 0).all()


def test_no_rows():
    h = binding.Experts(4, 8, 2)
    off = ints(np.zeros(5))
    x, w = torch.zeros(0, 16, device=DEV), torch.ones(4, 8, 16, device=DEV)
    dw, db = empty(4, 8, 16), empty(4, 8)
    h.gr_expert_linear(x, w, torch.zeros(0, 8, device=DEV), off=off)
    h.gr_expert_linear_backward(x, w, torch.zeros(0, 8, device=DEV), out_dw=dw, out_db=db, off=off)
    assert float(dw.abs().sum()) == 0 and float(db.abs().sum()) == 0
    h.gr_expert_route(torch.zeros(0, 4, device=DEV), empty(0, 2), empty(0, 2, dtype=torch.int32), off, empty(0, dtype=torch.int32),
                      empty(0, 2, dtype=torch.int32))
    assert off.tolist() == [0] * 5
    h.gr_expert_combine(torch.zeros(0, 8, device=DEV), empty(0, 2, dtype=torch.int32), empty(0, 8))
    norm = empty(1)
    h.gr_clip_gradients([], 1.0, norm)
    assert float(norm) == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_offsets_beyond_32_bits(dtype):
    """More than 2^31 elements of y (and of dz and dx): the last rows are as right as the first."""
    n, E, I, O, k = 540_000, 3, 32, 4096, 2
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.randn(n // k, I, generator=g, device=DEV).to(dtype)
    w = torch.randn(E, O, I, generator=g, device=DEV).to(dtype)
    off = torch.tensor([0, 1000, 300_001, n - 5], dtype=torch.int32, device=DEV)
    slot = torch.randperm(n, generator=g, device=DEV).int()
    slot[n - 5:] = -1 - slot[n - 5:]
    h = binding.Experts(E, n // k, k)
    y = torch.empty(n, O, dtype=dtype, device=DEV)
    h.gr_expert_linear(x, w, y, off=off, slot=slot, top_k=k)
    at = torch.tensor([0, 999, 1000, 300_000, 300_001, n - 7, n - 6], device=DEV)
    e = [0, 0, 1, 1, 2, 2, 2]
    for p, ex in zip(at.tolist(), e):
        r = ref.f64(x[int(slot[p]) // k]) @ ref.f64(w[ex]).T
        ref.close(y[p], r, dtype, np.abs(ref.f64(x[int(slot[p]) // k])) @ np.abs(ref.f64(w[ex])).T, I)
    assert float(y[n - 5:].abs().max()) == 0
    out = torch.empty(n // k, O, dtype=dtype, device=DEV)
    pos = torch.empty(n, dtype=torch.int32, device=DEV)
    live = slot[:n - 5].long()
    pos.fill_(-1)
    pos[live] = torch.arange(n - 5, dtype=torch.int32, device=DEV)
    pos = pos.view(n // k, k)
    h.gr_expert_combine(y, pos, out)
    for r_ in (0, 77, n // k - 1):
        want = sum(ref.f64(y[p]) for p in pos[r_].tolist() if p >= 0)
        ref.close(out[r_], want, dtype, np.abs(want) + 64, k)
    del out
    dx = torch.empty(n, I, dtype=dtype, device=DEV)
    dw = torch.empty_like(w)
    h.gr_expert_linear_backward(x, w, y, out_dx=dx, out_dw=dw, off=off, slot=slot, top_k=k)
    for p, ex in ((n - 6, 2), (300_000, 1)):
        r = ref.f64(y[p]) @ ref.f64(w[ex])
        ref.close(dx[p], r, dtype, np.abs(ref.f64(y[p])) @ np.abs(ref.f64(w[ex])), O)
    # a weight's gradient reaches to the last rows
    rows = slot[300_001:n - 5].long() // k
    col = y[300_001:n - 5, O - 1].double() @ x[rows].double()
    size = y[300_001:n - 5, O - 1].double().abs() @ x[rows].double().abs()
    ref.close(dw[2, O - 1], ref.f64(col), dtype, ref.f64(size), 240_000)


# ---- weighted sum -----------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,k,O", [(1, 1, 1), (16, 9, 1), (300, 2, 64), (77, 9, 33), (1000, 1, 7), (129, 16, 520), (5, 3, 2048), (64, 2, 24)])
def test_weighted_sum_and_its_gradient(T, k, O, dtype):
    rng = np.random.default_rng(T + O)
    S, E = T * k, 16
    ids = rng.integers(-1, E, (T, k))
    off, slot, pos = ref.plan(ids, E)
    y, w, dout = f64_of(rng.normal(size=(S, O)), dtype), f64_of(rng.normal(size=(T, k)), torch.float32), f64_of(rng.normal(size=(T, O)), dtype)
    given_w, given_y = np.where(ids < 0, NAN, w), y.copy()
    given_y[off[-1]:] = NAN                        # what has no expert is not read
    h = binding.Experts(E, T, k)
    ty, tw, td = put(given_y, dtype), put(given_w, torch.float32), put(dout, dtype)
    live = (pos >= 0)[:, :, None]
    parts = np.where(live, y[pos], 0)
    for weight, ww in ((tw, np.where(ids < 0, 0, w)), (None, np.where(ids < 0, 0, 1.0))):
        out = empty(T, O, dtype=dtype)
        h.gr_expert_combine(shifted(ty) if weight is None else ty, ints(pos), out, weight=weight)
        ref.close(out, (parts * ww[:, :, None]).sum(1), dtype, np.abs(parts * ww[:, :, None]).sum(1), k)
        dy, dw = empty(S, O, dtype=dtype), empty(T, k)
        h.gr_expert_combine_backward(shifted(td) if weight is None else td, ty, ints(slot), dy, weight=weight, out_dweight=dw)
        flat = np.where(slot < 0, -1 - slot, slot)
        rdy = dout[flat // k] * ww.reshape(-1)[flat, None]
        ref.close(dy, rdy, dtype, np.abs(rdy), 1)
        prod = parts * dout[:, None, :]
        ref.close(dw, prod.sum(2), torch.float32, np.abs(prod).sum(2), O)
    only = empty(S, O, dtype=dtype)
    h.gr_expert_combine_backward(td, None, ints(slot), only)
    assert torch.equal(only, dy)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,k,O", [(1, 2, 3), (61, 3, 9), (200, 2, 17), (33, 9, 511), (40, 1, 1021), (7, 4, 2050)])
def test_weighted_sums_of_odd_widths(T, k, O, dtype):
    test_weighted_sum_and_its_gradient(T, k, O, dtype)


# ---- clipping ---------------------------------------------------------------------------------


@pytest.mark.parametrize("lengths", [[1], [0, 5, 0], [4096, 1, 8191], [60000, 7], list(range(1, 403)), [3_000_001, 17, 1_000_000]])
@pytest.mark.parametrize("limit", [0.5, 2.0, 0.0, INF])
def test_clipping(lengths, limit):
    rng = np.random.default_rng(len(lengths))
    types = [TYPES[i % 3] for i in range(len(lengths))]
    g = [f64_of(rng.normal(size=n), t) for n, t in zip(lengths, types)]
    t = [shifted(put(a, ty), i % 3) if len(a) else put(a, ty) for i, (a, ty) in enumerate(zip(g, types))]
    norm = np.sqrt(sum((a * a).sum() for a in g))
    h = binding.Experts(1, 1, 1)
    got, out = empty(1), [torch.full_like(x, 3) for x in t]
    h.gr_clip_gradients(t, limit * norm, got, out=out)
    ref.close(got, np.array([norm]), torch.float32, norm)
    by = min(1.0, float(np.float32(limit * norm)) / norm) if norm else 1.0
    for a, o, x, ty in zip(g, out, t, types):
        ref.close(o, a * by, ty, np.abs(a * by), 0)
        assert np.array_equal(ref.f64(x), a)
        if by == 1.0:
            assert torch.equal(o, x)
    h.gr_clip_gradients(t, limit * norm, got)
    for o, x in zip(out, t):
        assert torch.equal(o, x)


def test_norms_at_the_ends_of_the_range():
    h = binding.Experts(1, 1, 1)
    norm = empty(1)
    for value, n in ((3e38, 1), (1e30, 100), (1e-40, 1000), (2.0 ** -149, 4), (0.0, 10)):
        t = torch.full((n,), value, device=DEV)
        v = float(t[0])
        h.gr_clip_gradients([t], 1.0, norm)
        ref.close(norm, np.array([v * n ** 0.5]), torch.float32, v * n ** 0.5)
        ref.close(t, np.full(n, v * min(1.0, 1 / (v * n ** 0.5)) if v else 0.0), torch.float32, 1.0 if v > 1 else v)
    huge = torch.full((4,), 3e38, device=DEV)      # the norm is past what single precision holds, the gradients are not
    h.gr_clip_gradients([huge], 8.0, norm)
    assert float(norm) == INF
    ref.close(huge, np.full(4, 4.0), torch.float32, 4.0)
    for bad in (INF, -INF, NAN):
        a, b = torch.ones(1000, device=DEV), torch.ones(7, dtype=torch.float16, device=DEV)
        b[3] = bad
        keep = b.clone()
        h.gr_clip_gradients([a, b], 0.1, norm)
        assert not np.isfinite(float(norm)) and bool((a == 1).all()) and torch.equal(b.isnan(), keep.isnan()) and float(b[0]) == 1


# ---- all of it --------------------------------------------------------------------------------


def test_gradients_against_differences():
    """A mixture of two-layer experts in single precision: every gradient against central differences of the same mixture in 64 bits."""
    rng = np.random.default_rng(4)
    T, E, k, F, H = 11, 5, 3, 6, 7
    x, lg = (f64_of(rng.normal(size=s), torch.float32) for s in ((T, F), (T, E)))
    w1, b1, w2, b2 = (f64_of(rng.normal(size=s) * 0.6, torch.float32) for s in ((E, H, F), (E, H), (E, 1, H), (E, 1)))
    goal = f64_of(rng.normal(size=(T, 1)), torch.float32)
    _, ids = ref.route(lg, k, None, "softmax", 1, 1, True, 1.0)

    def loss(x, lg, w1, b1, w2, b2):
        s = ref.scores(lg, "softmax")
        total = 0.0
        for t in range(T):
            share = s[t, ids[t]] / s[t, ids[t]].sum()
            out = sum(p * (w2[e] @ np.maximum(w1[e] @ x[t] + b1[e], 0) + b2[e]) for p, e in zip(share, ids[t]))
            total += 0.5 * ((out - goal[t]) ** 2).sum()
        return total

    h = binding.Experts(E, T, k)
    S, f32 = T * k, torch.float32
    t = {n: put(a, f32) for n, a in dict(x=x, lg=lg, w1=w1, b1=b1, w2=w2, b2=b2, goal=goal).items()}
    weight, chosen = empty(T, k), empty(T, k, dtype=torch.int32)
    off, slot, pos = empty(E + 1, dtype=torch.int32), empty(S, dtype=torch.int32), empty(T, k, dtype=torch.int32)
    h.gr_expert_route(t["lg"], weight, chosen, off, slot, pos, renormalise=True)
    assert np.array_equal(chosen.cpu().numpy(), ids)
    y1, y2, out = empty(S, H), empty(S, 1), empty(T, 1)
    h.gr_expert_linear(t["x"], t["w1"], y1, bias=t["b1"], off=off, slot=slot, top_k=k, relu=True)
    h.gr_expert_linear(y1, t["w2"], y2, bias=t["b2"], off=off)
    h.gr_expert_combine(y2, pos, out, weight=weight)
    dout = out - t["goal"]
    g = {n: torch.full_like(t[n], 9) for n in ("lg", "w1", "b1", "w2", "b2", "x")}
    dy2, dweight, dy1, dz1, dxs = empty(S, 1), empty(T, k), empty(S, H), empty(S, H), empty(S, F)
    h.gr_expert_combine_backward(dout, y2, slot, dy2, weight=weight, out_dweight=dweight)
    h.gr_expert_route_backward(t["lg"], chosen, dweight, g["lg"], renormalise=True)
    h.gr_expert_linear_backward(y1, t["w2"], dy2, out_dx=dy1, out_dw=g["w2"], out_db=g["b2"], off=off)
    h.gr_expert_linear_backward(t["x"], t["w1"], dy1, out_dx=dxs, out_dw=g["w1"], out_db=g["b1"], y=y1, out_dz=dz1, off=off, slot=slot, top_k=k)
    h.gr_expert_combine(dxs, pos, g["x"])
    at = dict(x=x, lg=lg, w1=w1, b1=b1, w2=w2, b2=b2)
    step = 1e-6
    for name in g:
        diff = np.zeros_like(at[name])
        for i in np.ndindex(*at[name].shape):
            up, down = at[name].copy(), at[name].copy()
            up[i] += step
            down[i] -= step
            diff[i] = (loss(**{**at, name: up}) - loss(**{**at, name: down})) / (2 * step)
        # differences of 1e-6 in sums of order 10: 1e-16 * 10 / 1e-6 = 1e-9, and step^2 = 1e-12 times third derivatives; single
        # precision through five products: 1e-6 of the largest gradients
        assert np.abs(ref.f64(g[name]) - diff).max() < 1e-5 * max(1.0, np.abs(diff).max()), name


def test_another_stream_and_a_recorded_sequence():
    rng = np.random.default_rng(5)
    T, E, k, I, O = 100, 9, 3, 64, 40
    h = binding.Experts(E, T, k)
    bf = torch.bfloat16
    lg, x, w = put(rng.normal(size=(T, E)), torch.float32), put(rng.normal(size=(T, I)), bf), put(rng.normal(size=(E, O, I)), bf)
    S = T * k
    weight, chosen = empty(T, k), empty(T, k, dtype=torch.int32)
    off, slot, pos = empty(E + 1, dtype=torch.int32), empty(S, dtype=torch.int32), empty(T, k, dtype=torch.int32)
    y, out, dw, dx, dweight, dlg, norm, db = empty(S, O, dtype=bf), empty(T, O, dtype=bf), empty(E, O, I, dtype=bf), empty(S, I, dtype=bf), empty(T, k), empty(T, E), empty(1), empty(E, O, dtype=bf)
    dz, dy = empty(S, O, dtype=bf), empty(S, O, dtype=bf)
    clipped = [torch.empty_like(dw), torch.empty_like(db)]
    results = [weight, chosen, off, slot, pos, y, out, dw, dx, dweight, dlg, norm, db, dz, dy, *clipped]

    def step():
        h.gr_expert_route(lg, weight, chosen, off, slot, pos, renormalise=True)
        h.gr_expert_linear(x, w, y, off=off, slot=slot, top_k=k, relu=True)
        h.gr_expert_combine(y, pos, out, weight=weight)
        h.gr_expert_combine_backward(out, y, slot, dy, weight=weight, out_dweight=dweight)
        h.gr_expert_route_backward(lg, chosen, dweight, dlg, renormalise=True)
        h.gr_expert_linear_backward(x, w, dy, out_dx=dx, out_dw=dw, out_db=db, y=y, out_dz=dz, off=off, slot=slot, top_k=k)
        h.gr_clip_gradients([dw, db], 0.5, norm, out=clipped)

    def wipe():
        for r in results:
            r.fill_(55)

    step()
    torch.cuda.synchronize()
    want = [r.clone() for r in results]
    wipe()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(2_000_000)
        step()
    side.synchronize()
    for r, v in zip(results, want):
        assert torch.equal(r, v)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for scale in (1.0, -1.0, 0.5):
        lg.mul_(scale)
        x.mul_(scale)
        step()
        torch.cuda.synchronize()
        want = [r.clone() for r in results]
        wipe()
        graph.replay()
        torch.cuda.synchronize()
        for r, v in zip(results, want):
            assert torch.equal(r, v)


# ---- refusals ---------------------------------------------------------------------------------


def refused(code, call, *a, **k):
    with pytest.raises(binding.GoodRouteError) as e:
        call(*a, **k)
    assert e.value.code == code


def test_refusals():
    E, T, k, I, O = 6, 10, 2, 8, 4
    for args, code in (((0, 1, 1), -1), ((4, -1, 1), -1), ((4, 1, 0), -1), ((4, 1, 5), -1), ((513, 1, 1), -2), ((64, 1, 17), -2), ((4, 2 ** 30, 2), -2)):
        refused(code, binding.Experts, *args)
    h = binding.Experts(E, T, k)
    lg, w, ids = torch.zeros(T, E, device=DEV), empty(T, k), empty(T, k, dtype=torch.int32)
    refused(-1, h.gr_expert_route, lg, w, ids, n_group=4)
    refused(-1, h.gr_expert_route, lg, w, ids, n_group=2, n_group_kept=3)
    refused(-1, h.gr_expert_route, lg, w, ids, n_group=2, n_group_kept=0)
    refused(-1, h.gr_expert_route, lg, w, ids, scale=INF)
    refused(-1, h.gr_expert_route, lg, w, ids, out_off=empty(E + 1, dtype=torch.int32))
    refused(-2, h.gr_expert_route, torch.zeros(T + 1, E, device=DEV), empty(T + 1, k), empty(T + 1, k, dtype=torch.int32))
    refused(-2, h.gr_expert_route, lg, empty(T, 3), empty(T, 3, dtype=torch.int32))
    refused(-2, h.gr_expert_plan, empty(T, 3, dtype=torch.int32), empty(E + 1, dtype=torch.int32), empty(3 * T, dtype=torch.int32), empty(T, 3, dtype=torch.int32))
    with pytest.raises(ValueError, match="logits"):
        h.gr_expert_route(torch.zeros(T, E + 1, device=DEV), w, ids)
    with pytest.raises(TypeError, match="logits"):
        h.gr_expert_route(lg.double(), w, ids)
    with pytest.raises(TypeError, match="out_weight"):
        h.gr_expert_route(lg, w.half(), ids)
    with pytest.raises(TypeError, match="logits"):
        h.gr_expert_route(torch.zeros(T, 2 * E, device=DEV)[:, ::2], w, ids)
    with pytest.raises(ValueError, match="out_slot"):
        h.gr_expert_plan(ids, empty(E + 1, dtype=torch.int32), empty(3, dtype=torch.int32), empty(T, k, dtype=torch.int32))
    with pytest.raises(KeyError):
        h.gr_expert_route(lg, w, ids, scoring="softplus")
    x, wt, off = torch.zeros(T, I, device=DEV), torch.zeros(E, O, I, device=DEV), ints(np.zeros(E + 1))
    with pytest.raises(ValueError, match="x: shape"):
        h.gr_expert_linear(torch.zeros(T, I + 1, device=DEV), wt, empty(T, O), off=off)
    with pytest.raises(ValueError, match="w: shape"):
        h.gr_expert_linear(x, wt[:-1], empty(T, O), off=off)
    with pytest.raises(TypeError, match="w: need"):
        h.gr_expert_linear(x, wt.half(), empty(T, O), off=off)
    with pytest.raises(ValueError, match="x: shape"):
        h.gr_expert_linear(x, wt, empty(T, O), off=off, slot=ints(np.zeros(T)), top_k=2)
    refused(-2, h.gr_expert_linear, torch.zeros(T * k + 1, I, device=DEV), wt, empty(T * k + 1, O), off=off)
    refused(-2, h.gr_expert_linear, torch.zeros(1, 65537, device=DEV), torch.zeros(1, 65537, device=DEV), empty(1, 1))
    refused(-1, h.gr_expert_linear_backward, x, wt, empty(T, O), out_dx=empty(T, I), y=empty(T, O), off=off)
    refused(-1, h.gr_expert_linear_backward, x, wt, empty(T, O), out_dx=empty(T, I), out_dz=empty(T, O), off=off)
    refused(-2, h.gr_expert_combine, empty(T * 3, O), empty(T, 3, dtype=torch.int32), empty(T, O))
    refused(-1, h.gr_expert_combine_backward, empty(T, O), None, empty(T * k, dtype=torch.int32), out_dweight=empty(T, k))
    with pytest.raises(ValueError, match="y: "):
        h.gr_expert_combine(empty(T, O), ids, empty(T, O))
    refused(-1, h.gr_clip_gradients, [x], -1.0)
    refused(-1, h.gr_clip_gradients, [x], NAN)
    refused(-2, h.gr_clip_gradients, [x] * 4097, 1.0)
    with pytest.raises(ValueError, match="out: "):
        h.gr_clip_gradients([x], 1.0, out=[])
    with pytest.raises(TypeError, match="grads"):
        h.gr_clip_gradients([x.int()], 1.0)
    h.close()
    refused(-1, h.gr_expert_route, lg, w, ids)
    assert binding.lib().gr_experts_destroy(None) == 0
