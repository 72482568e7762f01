"""What the entry points of the operators that read a request's tokens refuse before they look at the device (CPU only)."""
import ctypes as C

import pytest

from paper_2605_16867_amd import binding, build


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


def test_a_build_with_spilled_states_fails():
    scan, other = "_ZN2gr12k_scan_tilesIfLi4ELi8ELb0EEEvNS0_8TileArgsE", "_ZN2gr7k_routeIfEEvNS_9RouteArgsE"

    def remarks(*kernels):
        return "".join(f"scan.hip:479:1: remark: {line} [-Rpass-analysis=kernel-resource-usage]\n" for name, scalar, vector, scratch in kernels for line in (
            f"Function Name: {name}", "    VGPRs: 105", f"    ScratchSize [bytes/lane]: {scratch}", f"    SGPRs Spill: {scalar}", f"    VGPRs Spill: {vector}"))

    build.check_held(remarks((other, 9, 4, 16), (scan, 0, 0, 0), (scan, 0, 0, 0)))
    for bad in (((scan, 0, 0, 0), (scan, 1, 0, 0)), ((scan, 0, 1, 0),), ((scan, 0, 0, 8), (other, 0, 0, 0)), ((other, 0, 0, 0),), ()):
        with pytest.raises(RuntimeError, match="k_scan_tiles"):
            build.check_held(remarks(*bad))
    with pytest.raises(RuntimeError, match="no word of"):
        build.check_held(remarks((scan, 0, 0, 0)).replace("SGPRs Spill", "spilled"))
