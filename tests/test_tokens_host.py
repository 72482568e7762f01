"""What the entry points of the operators that read a request's tokens refuse before they look at the device (CPU only)."""
import ctypes as C

import pytest

from paper_2605_16867_amd import binding


@pytest.mark.parametrize("sizes,code", [((-1, 1, 1), -1), ((1, 0, 1), -1), ((1, 1, 0), -1), (((1 << 30) + 1, 1, 1), -2), ((1, (1 << 24) + 1, 1), -2),
                                        ((1, 1, 65537), -2)])
def test_sizes_of_a_handle(sizes, code):
    at = C.c_void_p(5)
    assert binding.lib().gr_tokens_create(C.byref(at), *sizes) == code and at.value is None
    with pytest.raises(binding.GoodRouteError):
        binding.Tokens(*sizes)


def test_no_handle():
    l, p = binding.lib(), None
    assert l.gr_tokens_create(None, 1, 1, 1) == -1 and l.gr_tokens_destroy(None) == 0
    assert l.gr_token_embed(p, 0, 1, 1, 0, p, p, 1.0, p, p) == -1
    assert l.gr_token_embed_backward(p, 0, 1, 1, 0, p, p, 1.0, p, p) == -1
    assert l.gr_gated_scan(p, 0, 0, 1, 0, p, p, 1, p, 1, p, p, p, p) == -1
    assert l.gr_gated_scan_backward(p, 0, 0, 1, 0, p, p, 1, p, 1, p, p, p, p, p, 1, p, 1, p, p) == -1
    assert l.gr_dropout(p, 0, 0, p, p, 0.1, 0, 0, p, p, p) == -1
