"""The extension behind rms_norm, route and AdapterBank.forward: calls that it has to turn away, without a GPU."""
import pytest

from paper_2308_15030_b200 import binding


@pytest.mark.parametrize("name,n", [("rms_norm", 10), ("route", 8), ("adapters_forward", 11)])
def test_the_number_of_arguments_comes_first(name, n):
    call = getattr(binding.marshal(), name)
    for have in list(range(n)) + [n + 1, n + 7]:
        with pytest.raises(TypeError, match="arguments expected"):
            call(*([None] * have))


def test_things_that_are_no_tensors_and_no_gate():
    import torch
    t = torch.zeros(2, 8)
    with pytest.raises(AttributeError):
        binding.rms_norm(None, t, 1e-6, out=t)
    with pytest.raises(AttributeError):
        binding.route(binding.Gate(), [1.0] * 8, t, t)
    for gate in (None, b"gate", 7):
        with pytest.raises(TypeError):
            binding.route(gate, t, t, t)


def test_streams_and_devices_without_the_bare_functions(monkeypatch):
    """Where torch lacks its bare functions the ones of torch.cuda stand in; each can be called."""
    import types
    import torch
    assert binding._device_functions()[2] is torch._C._cuda_getCurrentRawStream
    monkeypatch.setattr(torch, "_C", types.SimpleNamespace())
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device: types.SimpleNamespace(cuda_stream=100 + device))
    now, put, stream = binding._device_functions()
    assert now() == 3 and callable(put) and stream(2) == 102
