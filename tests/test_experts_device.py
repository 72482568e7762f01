"""The calls of a length predictor are on one device: the handle's, its tensors' and the current one."""
import pytest
import torch

from paper_2605_16867_amd import binding


class _Elsewhere:
    """As much of a tensor on another device as the check of an argument asks for."""
    is_cuda, dtype, device = True, torch.float32, torch.device("cuda", 1)

    def is_contiguous(self):
        return True

    def numel(self):
        return 4

    def data_ptr(self):
        return 16


def test_a_tensor_of_another_device_is_refused():
    h = object.__new__(binding.Experts)
    h._h, h._device = binding.C.c_void_p(), 0
    with pytest.raises(ValueError, match="logits: on cuda:1, need the handle's device, cuda:0"):
        h._dev(_Elsewhere(), torch.float32, "logits", 4)
    h._device = 1
    assert h._dev(_Elsewhere(), torch.float32, "logits", 4).value == 16 and h._dev(None, torch.float32, "bias") is None


@pytest.mark.gpu
@pytest.mark.parametrize("native", [True, False])
def test_a_handle_of_another_device_is_refused(native, monkeypatch):
    """By every call, natively marshalled or not, and nothing is queued."""
    if not native:
        monkeypatch.setattr(binding, "_marshal", binding._Ctypes)
    T, E, k, O = 4, 3, 2, 8
    f = lambda *s: torch.zeros(*s, device="cuda:0")
    i = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda:0")
    h = binding.Experts(E, T, k)
    calls = (lambda: h.gr_expert_route(f(T, E), weight, i(T, k)), lambda: h.gr_expert_route_backward(f(T, E), i(T, k), f(T, k), f(T, E)),
             lambda: h.gr_expert_plan(i(T, k), i(E + 1), i(T * k), i(T, k)), lambda: h.gr_expert_linear(f(T, O), f(E, O, O), f(T, O), off=i(E + 1)),
             lambda: h.gr_expert_linear_backward(f(T, O), f(E, O, O), f(T, O), out_dx=f(T, O), off=i(E + 1)),
             lambda: h.gr_expert_combine(f(T * k, O), i(T, k), f(T, O)), lambda: h.gr_expert_combine_backward(f(T, O), None, i(T * k), f(T * k, O)),
             lambda: h.gr_clip_gradients([f(3)], 1.0), lambda: h.gr_clip_gradients([], 1.0))
    weight = f(T, k)
    for call in calls:
        call()
    assert bool((weight > 0).all())
    weight.zero_()
    h._device, h._at = 1, (h._at[0], 1)
    for call in calls:
        with pytest.raises(ValueError, match="need the handle's"):
            call()
    torch.cuda.synchronize()
    assert bool((weight == 0).all())
    h._device = 0
    h.close()
    for call in calls:
        with pytest.raises(binding.GoodRouteError):
            call()


@pytest.mark.gpu
@pytest.mark.parametrize("native", [True, False])
def test_slots_without_a_row_are_the_librarys_to_refuse(native, monkeypatch):
    if not native:
        monkeypatch.setattr(binding, "_marshal", binding._Ctypes)
    h = binding.Experts(2, 8, 1)
    x, w, y, slot = (torch.zeros(*s, device="cuda:0") for s in ((8, 4), (4, 4), (8, 4), (8,)))
    for top_k in (0, -1):
        for call in (lambda: h.gr_expert_linear(x, w, y, slot=slot.int(), top_k=top_k),
                     lambda: h.gr_expert_linear_backward(x, w, y, out_dx=torch.zeros_like(x), slot=slot.int(), top_k=top_k)):
            with pytest.raises(binding.GoodRouteError) as e:
                call()
            assert e.value.code == -1
