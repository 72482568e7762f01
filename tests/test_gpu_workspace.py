"""Device memory of a handle: parts that only some handles can use are not reserved by the others."""
import numpy as np
import pytest
import torch

from paper_2605_16867_amd import binding
from tests.fleets import CLASSES

pytestmark = pytest.mark.gpu


def _held(n_inst, n_class, entries, max_len, max_requests, handles=1):
    """Bytes that a handle takes (of several, as small allocations share a block)."""
    coef = [np.array([CLASSES[c % 3][i] for c in range(n_class)]) for i in range(4)]

    def make():
        return binding.Fleet(*coef, np.arange(n_inst, dtype=np.int32) % n_class, entries, max_len, max_requests)

    make().close()      # (what the runtime itself takes for the first one)
    before = torch.cuda.mem_get_info()[0]
    hs = [make() for _ in range(handles)]
    held = before - torch.cuda.mem_get_info()[0]
    for h in hs:
        h.close()
    return held / handles


def test_minima_by_row_only_where_classes_may_come_first():
    """4 096 instances of six classes, a row for each of 16 385 lengths either way: 16 640 rows of 272 minima more from 131 072 requests on, and none for more classes than a group has lanes."""
    rows, runs = 16640, 272
    few, many = (_held(4096, 6, 64, 16384, n) for n in (131071, 131072))
    assert many - few >= 0.9 * rows * runs * 4
    few, many = (_held(4096, 17, 64, 16384, n) for n in (131071, 131072))
    assert many - few < 0.1 * rows * runs * 4


def test_feedback_sums_only_where_waves_share_an_instance():
    """512 instances: 65 to 128 entries take (50 * 128 + 1 200) * 512 bytes that up to 64 entries do not, besides the tables,
    whose 18 bytes an entry and 8 a request double."""
    small, large = _held(512, 3, 64, 64, 1, 32), _held(512, 3, 128, 64, 1, 32)
    assert large - small >= 0.9 * 512 * ((50 * 128 + 1200) + 64 * 26)


@pytest.mark.parametrize("tokens,vocab,width", [(1 << 20, 1 << 24, 4096), (32768, 100, 65536), (1 << 22, 1, 1), (1 << 23, 1 << 20, 130), (1, 1, 64)])
def test_a_handle_of_tokens_holds_what_its_header_says(tokens, vocab, width):
    up = lambda a, b: -(-a // b)
    p, t = up(tokens + vocab, 1024), max(up(tokens, 96), min(up(tokens, 64), 512))
    channels = up(width, 128) * 128 if width > 128 else width + 3
    parts = [16 * tokens, 2048 * (up(tokens, 2048) + 1), max(8 * width * p, 1 << 24), max(8 * p, 16384), 8 * (2 * t + up(t, 16)) * channels, 2 * width + 400]
    binding.Tokens(1, 1, 1).close()
    before = torch.cuda.mem_get_info()[0]
    h = binding.Tokens(tokens, vocab, width)
    held = before - torch.cuda.mem_get_info()[0]
    h.close()
    # an allocation is of whole blocks of 2 MB, or shares one
    assert abs(held - sum(parts)) <= len(parts) * (2 << 20), (held, parts)


def test_a_handle_that_does_not_fit_leaves_no_error_behind():
    """Refused for its 12 TB of words between tiles, it changes nothing for the next calls: another handle's, or torch's own."""
    h, table = binding.Tokens(16, 4, 8), torch.arange(32.0, device="cuda").view(4, 8)
    token, out = torch.tensor([1, 3], dtype=torch.int32, device="cuda"), torch.empty(2, 8, device="cuda")
    torch.cuda.synchronize()
    for after in (lambda: h.gr_token_embed(token, table, out), lambda: torch.index_select(table, 0, token, out=out)):
        out.fill_(77)
        with pytest.raises(binding.GoodRouteError) as e:
            binding.Tokens(1 << 30, 1, 65536)
        assert e.value.code == -5
        after()
        torch.cuda.synchronize()
        assert torch.equal(out, table[[1, 3]])
