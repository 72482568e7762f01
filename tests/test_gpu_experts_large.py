"""The forms that the operators of a length predictor take for many rows, many experts and many elements: more units of slots than one
workgroup adds up, several batches of rows a workgroup, large tiles of 64 experts and more, results past 2^31 elements."""
import numpy as np
import pytest
import torch

from paper_2605_16867_amd import binding
from tests import experts_reference as ref
from tests.test_gpu_experts import (DEV, INF, check_plan, empty, f64_of, ints, run_route, test_gradients_of_a_layer as gradients_of_a_layer,
                                    test_layer as forward_of_a_layer)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("E", [2, 9, 64, 512])
@pytest.mark.parametrize("T,k", [(65_536, 2), (65_537, 2), (70_001, 2), (600_001, 2), (149_800, 7), (2_200_003, 1)])
def test_order_of_many_slots(T, k, E):
    """128 units of 1 024 slots, 129, 137; 1 172, 1 025 and 2 149, past one and two steps of the sums over units, with remainders."""
    if k > E:
        pytest.skip("more choices than experts")
    rng = np.random.default_rng(T + E)
    ids = rng.integers(-2, E + 2, (T, k))
    ids[T // 3:T // 2] = E - 1                    # (many of one expert in a row)
    h = binding.Experts(E, T, k)
    off, slot, pos = empty(E + 1, dtype=torch.int32), empty(T * k, dtype=torch.int32), empty(T, k, dtype=torch.int32)
    h.gr_expert_plan(ints(ids), off, slot, pos)
    check_plan(ids, E, (off, slot, pos))


def _route_reference(x, k, bias, n_group, kept):
    """Softmax and the choice of many rows at once, in 64 bits: weights as shares of the chosen, experts."""
    T, E = x.shape
    masked = x == -INF
    m = x.max(1, keepdim=True).values.clamp(min=-1e300)
    s = torch.where(masked, 0.0, torch.exp(x - m))
    s = s / s.sum(1, keepdim=True).clamp(min=1e-300)
    c = s if bias is None else s + bias
    c = torch.where(masked, -INF, c)
    if n_group > 1:
        two = c.view(T, n_group, -1).sort(dim=2, descending=True).values[:, :, :2]
        group = torch.where(two == -INF, 0.0, two).sum(2)
        group = torch.where(two[:, :, 0] == -INF, -INF, group)
        best = group.sort(dim=1, descending=True, stable=True).indices[:, :kept]
        keep = torch.zeros(T, n_group, dtype=torch.bool, device=x.device).scatter_(1, best, True)
        c = torch.where(keep.repeat_interleave(E // n_group, 1), c, -INF)
    v, ids = c.sort(dim=1, descending=True, stable=True)
    none = v[:, :k] == -INF
    ids = torch.where(none, -1, ids[:, :k])
    w = torch.where(none, 0.0, s.gather(1, ids.clamp(min=0)))
    total = w.sum(1, keepdim=True)
    return torch.where(total > 0, w / total.clamp(min=1e-300), 0.0), ids


@pytest.mark.parametrize("form", ["plain", "bias", "groups"])
@pytest.mark.parametrize("T,E,k,dtype", [  # rows of a batch: 256, 64, 8; from 2 048 batches on two a workgroup, from 4 096 on four
    (524_288 - 100, 9, 2, torch.float32), (524_288 + 77, 9, 9, torch.float32), (1_048_576 + 300, 9, 2, torch.bfloat16),
    (131_072 + 33, 64, 8, torch.bfloat16), (262_144 + 65, 64, 9, torch.float32), (32_768 + 9, 512, 16, torch.float32)])
def test_choice_in_several_batches(T, E, k, dtype, form):
    g = torch.Generator(device=DEV).manual_seed(T)
    order = torch.rand(T, E, generator=g, device=DEV).argsort(1)
    x = (order - E // 2) * (0.125 if E <= 64 else 6.0 / E)         # (well apart, and exact in every type up to 64 experts)
    n_group, kept, bias = 1, 1, None
    if form != "plain":
        x = torch.where(torch.rand(T, E, generator=g, device=DEV) < 0.2, -INF, x)
        x[5], x[T - 1], x[T // 2, 1:] = -INF, -INF, -INF
        bias = 2.0 * torch.randperm(E, generator=g, device=DEV)        # (further apart than scores are: these order the experts)
    if form == "groups":
        n_group, kept = (3, 2) if E == 9 else (8, 3)
        # groups of which no two have the same sum, of two experts or of one
        bias += 5000.0 * 3.0 ** torch.randperm(n_group, generator=g, device=DEV).repeat_interleave(E // n_group)
    x, bias = x.to(dtype).double(), None if bias is None else bias.float().double()
    h = binding.Experts(E, T, k)
    w, ids = empty(T, k), empty(T, k, dtype=torch.int32)
    off, slot, pos = empty(E + 1, dtype=torch.int32), empty(T * k, dtype=torch.int32), empty(T, k, dtype=torch.int32)
    h.gr_expert_route(x.to(dtype), w, ids, off, slot, pos, bias=None if bias is None else bias.float(), n_group=n_group, n_group_kept=kept,
                      renormalise=True)
    rw, rids = _route_reference(x, k, bias, n_group, kept)
    assert torch.equal(ids.long(), rids)
    assert bool(((w.double() - rw).abs() <= (E + 16) * 2.0 ** -23 * rw + 2.0 ** -149).all())
    check_plan(ids.cpu().numpy(), E, (off, slot, pos))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("E,k", [(129, 4), (256, 8), (511, 16), (512, 2)])
def test_choice_of_many_experts_in_16_bits(E, k, dtype):
    """A few experts of each row well apart, all others equal behind them."""
    rng = np.random.default_rng(E)
    T, few = 90, k - 1
    x = np.full((T, E), -4.0)
    for t in range(T):
        x[t, rng.permutation(E)[:few]] = rng.permutation(few) * 0.25
    for scoring in ("softmax", "sigmoid"):
        w, ids, order = run_route(x, k, dtype, scoring=scoring, renorm=True)
        rw, rids = ref.route(x, k, None, scoring, 1, 1, True, 1.0)
        assert np.array_equal(ids, rids)
        ref.close(w, rw, torch.float32, magnitude=rw, n=E + 8)
        check_plan(ids, E, order)


@pytest.mark.parametrize("E", [63, 64, 65, 200])
def test_large_tiles_of_many_experts(E):
    """1 600 tiles of 256 by 256 and more forward, by input and by weight, of as many experts as a wave has lanes and more."""
    forward_of_a_layer(66_100, E, 72, 1032, 2, torch.bfloat16)
    gradients_of_a_layer(66_100, E, 1032, 72, 2, torch.float16)


def test_large_tiles_by_weight_of_many_experts():
    gradients_of_a_layer(700, 70, 1544, 520, 1, torch.bfloat16)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("I,O", [(32, 4096), (4096, 32)])
def test_gradients_past_32_bits(I, O, dtype):
    """More than 2^31 elements of y, dy and dz, or of dx and x: the last rows are as right as the first."""
    n, E = 540_000, 3
    g = torch.Generator(device=DEV).manual_seed(1)
    x, w = torch.randn(n, I, generator=g, device=DEV).to(dtype), torch.randn(E, O, I, generator=g, device=DEV).to(dtype)
    y, dy = torch.randn(n, O, generator=g, device=DEV).to(dtype), torch.randn(n, O, generator=g, device=DEV).to(dtype)
    off = torch.tensor([0, 1000, 300_001, n - 5], dtype=torch.int32, device=DEV)
    h = binding.Experts(E, n, 1)
    dz, dx = torch.full_like(dy, 77), torch.full_like(x, 77)
    dw, db = torch.full_like(w, 77), empty(E, O, dtype=dtype)
    h.gr_expert_linear_backward(x, w, dy, out_dx=dx, out_dw=dw, out_db=db, y=y, out_dz=dz, off=off)
    for p in range(0, n, 90_000):       # (whole, some rows at a time)
        part = slice(p, p + 90_000)
        assert torch.equal(dz[part], torch.where(y[part] > 0, dy[part], torch.zeros_like(dy[part])))
    del y, dy
    for p, e in ((0, 0), (999, 0), (1000, 1), (300_000, 1), (300_001, 2), (n - 7, 2), (n - 6, 2)):
        z, we = ref.f64(dz[p]), ref.f64(w[e])
        ref.close(dx[p], z @ we, dtype, np.abs(z) @ np.abs(we), O)
    assert float(dx[n - 5:].abs().max()) == 0
    for e, (lo, hi) in enumerate(((0, 1000), (1000, 300_001), (300_001, n - 5))):
        z = dz[lo:hi, O - 3:].double()
        ref.close(db[e, O - 3:], ref.f64(z.sum(0)), dtype, ref.f64(z.abs().sum(0)), hi - lo)
        total, size = torch.zeros(3, 8, dtype=torch.float64, device=DEV), torch.zeros(3, 8, dtype=torch.float64, device=DEV)
        for at in (slice(0, 4), slice(I - 4, I)):
            to = slice(0, 4) if at.start == 0 else slice(4, 8)
            total[:, to] = z.t().contiguous() @ x[lo:hi, at].double().contiguous()
            size[:, to] = z.t().abs().contiguous() @ x[lo:hi, at].double().abs().contiguous()
        got = torch.cat([dw[e, O - 3:, :4], dw[e, O - 3:, I - 4:]], 1)
        ref.close(got, ref.f64(total), dtype, ref.f64(size), hi - lo)
