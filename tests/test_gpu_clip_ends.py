"""Clipping at the end of the range of single precision."""
import numpy as np
import pytest
import torch

from paper_2605_16867_amd import binding
from tests import experts_reference as ref
from tests.test_gpu_experts import empty, f64_of, put

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("value,n,limit", [(3e38, 4, 1e-3), (3e38, 4, 1e-6), (1e38, 300_000, 1e-5), (1e35, 40, 1e-7), (2e38, 9000, 30.0)])
def test_clipping_by_very_much(value, n, limit):
    """Factors below the least number of full precision: results keep theirs."""
    rng = np.random.default_rng(n)
    a = f64_of(value * rng.uniform(0.5, 1.0, n), torch.float32)
    b = f64_of(rng.normal(size=n), torch.bfloat16)
    h = binding.Experts(1, 1, 1)
    t, norm = [put(a, torch.float32), put(b, torch.bfloat16)], np.sqrt((a * a).sum() + (b * b).sum())
    h.gr_clip_gradients(t, limit)
    by = float(np.float32(limit)) / norm
    # (the factor and two products: three roundings)
    ref.close(t[0], a * by, torch.float32, np.abs(a * by), 0)
    ref.close(t[1], b * by, torch.bfloat16, np.abs(b * by), 0)
    out = [torch.full_like(x, 3) for x in t]      # (and apart)
    t = [put(a, torch.float32), put(b, torch.bfloat16)]
    got = empty(1)
    h.gr_clip_gradients(t, limit, got, out=out)
    ref.close(out[0], a * by, torch.float32, np.abs(a * by), 0)
    # the norm itself as single precision holds it
    assert float(got) == float("inf") if norm > 3.41e38 else abs(float(got) - norm) <= 2.0 ** -22 * norm
