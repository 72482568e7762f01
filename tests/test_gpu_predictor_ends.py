"""The length predictor on what is not the ordinary: requests that belong to no expert, results that are no lengths."""
import pytest
import torch

from paper_2605_16867_amd import predictor

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_requests_of_no_expert_are_left_out(dtype):
    """A step on requests of which some are given to experts that there are not is the step on the others; with none, nothing moves."""
    def trained(x, target, kind):
        p = predictor.LengthPredictor(24, n_expert=4, hidden=(16, 16, 8), router_hidden=8, max_rows=200, dtype=dtype)
        loss = p.train_experts(x, target, kind, 0.1)
        return float(loss), float(p.norm), [t.clone() for t in p.w + p.b]

    x, target, kind = predictor.synthetic_requests(200, 24, 4, seed=5, dtype=dtype)
    out = torch.arange(200, device=x.device) % 3 == 1
    target[out] = 1e6
    given = kind.clone()
    given[out] = torch.where(torch.arange(200, device=x.device)[out] % 2 == 0, -1, 4).to(torch.int32)
    loss, norm, moved = trained(x, target, given)
    want, want_norm, want_moved = trained(x[~out].contiguous(), target[~out], kind[~out].contiguous())
    # the mean's factor and sums in another order: some roundings of single precision, then one of the type
    assert abs(loss - want) < 1e-5 * want and abs(norm - want_norm) < (1e-5 if dtype == torch.float32 else 0.02) * want_norm
    for a, b in zip(moved, want_moved):
        assert torch.allclose(a.float(), b.float(), rtol=2.0 ** -20 if dtype == torch.float32 else 2.0 ** -7, atol=1e-6 if dtype == torch.float32 else 1e-3)
    loss, norm, moved = trained(x, target, torch.full_like(kind, -1))
    start = predictor.LengthPredictor(24, n_expert=4, hidden=(16, 16, 8), router_hidden=8, max_rows=200, dtype=dtype)
    assert loss == 0 and norm == 0 and all(torch.equal(a, b) for a, b in zip(moved, start.w + start.b))


@pytest.mark.parametrize("max_len", [1, 4096, (1 << 24) + 1, (1 << 31) - 1])
@pytest.mark.parametrize("bias,least", [(float("nan"), False), (float("inf"), False), (80.0, False), (float("-inf"), True)])
def test_lengths_are_in_their_range(bias, least, max_len):
    """Whatever the experts come to; what is no number is taken for the longest."""
    p = predictor.LengthPredictor(24, n_expert=4, hidden=(16, 16, 8), router_hidden=8, max_rows=50)
    p.b[-1].fill_(bias)
    x, _, _ = predictor.synthetic_requests(50, 24, 4, seed=5)
    n = p.predict(x, max_len)
    assert n.dtype == torch.int32 and n.tolist() == [1 if least else max_len] * 50
