"""Layers at the ends of what their arguments may be: how many slots share a row, how many rows a launch takes, where a bias lies."""
import numpy as np
import pytest
import torch

from paper_2605_16867_amd import binding
from tests import experts_reference as ref
from tests.test_gpu_experts import DEV, empty, f64_of, ints, put

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
