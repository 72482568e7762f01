"""Layers at the ends of what their arguments may be: how many slots share a row, how many rows a launch takes, where a bias lies."""
import numpy as np
import pytest
import torch

from paper_2605_16867_amd import binding
from tests import experts_reference as ref
from tests.test_gpu_experts import DEV, TYPES, empty, f64_of, ints, layer, put, shifted

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("top_k", [(1 << 29) - 1, 1 << 30, (1 << 30) + 1, (1 << 31) - 1])
def test_one_row_for_all_slots(top_k):
    """More slots share a row than there may be slots: all are of the first."""
    rng = np.random.default_rng(7)
    n, I, O = 40, 24, 8
    x, w = f64_of(rng.normal(size=(1, I)), torch.float32), f64_of(rng.normal(size=(2, O, I)), torch.float32)
    off, slot = np.array([0, 17, 38]), rng.permutation(n)
    slot[38:] = -1 - slot[38:]
    h = binding.Experts(2, n, 1)
    y, dw = empty(n, O), empty(2, O, I)
    plan = dict(off=ints(off), slot=ints(slot), top_k=top_k)
    h.gr_expert_linear(put(x, torch.float32), put(w, torch.float32), y, **plan)
    r, size = ref.linear(x, w, np.zeros((2, O)), off, slot, top_k, False, n)
    ref.close(y, r, torch.float32, size, I)
    h.gr_expert_linear_backward(put(x, torch.float32), put(w, torch.float32), y, out_dw=dw, **plan)
    _, (rw, mw), _ = ref.linear_backward(x, w, ref.f64(y), off, slot, top_k)
    ref.close(dw, rw, torch.float32, mw, n)


def test_many_rows_of_few_features():
    """What a launch may have is asked of the results' tiles, not of the features that go in."""
    n, I = (1 << 20) + 1, 65536
    g = torch.Generator(device=DEV).manual_seed(0)
    x, w = torch.randn(2, I, generator=g, device=DEV).bfloat16(), torch.randn(1, I, generator=g, device=DEV).bfloat16()
    h = binding.Experts(1, n, 1)
    slot = torch.arange(n, dtype=torch.int32, device=DEV)
    y = empty(n, 1, dtype=torch.bfloat16)
    h.gr_expert_linear(x, w, y, slot=slot, top_k=1 << 20)
    want = ref.f64(x) @ ref.f64(w).T
    size = np.abs(ref.f64(x)) @ np.abs(ref.f64(w)).T
    ref.close(y[:1], want[:1], torch.bfloat16, size[:1], I)
    ref.close(y[-1:], want[1:], torch.bfloat16, size[1:], I)
    assert bool((y[:-1] == y[0]).all())
    # by weight the features that go in count, in tiles of them alone
    dw = empty(1, I, dtype=torch.bfloat16)
    h.gr_expert_linear_backward(x, w, y, out_dw=dw, slot=slot, top_k=1 << 20)
    first = float(ref.f64(y[:-1]).sum())
    r = first * ref.f64(x)[0] + float(y[-1]) * ref.f64(x)[1]
    ref.close(dw[0], r, torch.bfloat16, np.abs(first * ref.f64(x)[0]) + np.abs(float(y[-1]) * ref.f64(x)[1]), n)


def test_more_tiles_than_a_launch_may_have():
    """Results of which there would be more are refused, before anything is read."""
    n, I = (1 << 24) - 64, 65536
    h = binding.Experts(1, n, 1)
    few = empty(8)
    at, none = few.data_ptr(), None
    lib, stream = binding.lib(), torch.cuda.current_stream().cuda_stream
    layer = lambda i, o: lib.gr_expert_linear(h._h, n, i, o, 0, none, at, 1 << 30, at, at, none, 0, at, stream)
    assert layer(I, I) == -2 and layer(1, I) == -2
    assert lib.gr_expert_linear_backward(h._h, n, I, 1, 0, none, at, 1 << 30, at, at, none, at, none, at, none, none, stream) == -2


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,E,I,O", [(9, 3, 64, 40), (700, 3, 264, 304), (300, 2, 96, 8), (33_000, 2, 40, 2056), (400, 3, 33, 65)])
@pytest.mark.parametrize("by", [1, 2, 3])
def test_a_bias_at_any_address(n, E, I, O, by, dtype):
    """Only the bias off its boundary of 16 bytes: few rows, tiles of 128 and of 256, few features, odd widths."""
    rng = np.random.default_rng(n + O)
    off, slot, x, w, b = layer(rng, n, E, I, O, 1, dtype)
    h = binding.Experts(E, n, 1)
    y = empty(n, O, dtype=dtype)
    h.gr_expert_linear(put(x, dtype), put(w, dtype), y, bias=shifted(put(b, dtype), by), off=ints(off), slot=ints(slot), top_k=1)
    if n * O <= 1 << 20:
        r, size = ref.linear(x, w, b, off, slot, 1, False, n)
        ref.close(y, r, dtype, size, I)
    plain = empty(n, O, dtype=dtype)
    h.gr_expert_linear(put(x, dtype), put(w, dtype), plain, bias=put(b, dtype), off=ints(off), slot=ints(slot), top_k=1)
    assert torch.equal(y, plain)
