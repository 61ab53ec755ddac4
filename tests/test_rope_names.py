"""Names that rotary positions do not know are bad arguments like any other: ValueError, with what is known."""
import pytest
import torch

from paper_2604_15408_amd import binding


@pytest.mark.parametrize("given", ["cubic", "", None, 3, ["linear"]])
def test_scaling(given):
    with pytest.raises(ValueError, match="scaling is .* expected one of none, linear, base, parts"):
        binding.rope_frequencies(8, scaling=given)


@pytest.mark.parametrize("given", ["halves", "Half", None, 0, {}])
def test_layout(given, monkeypatch):
    monkeypatch.setattr(binding, "_native", lambda: binding._Ctypes)
    monkeypatch.setattr(binding, "_marshal", binding._Ctypes)
    monkeypatch.setattr(binding, "_raw_device", lambda: None)
    monkeypatch.setattr(binding, "_dev", lambda t, *rest: t.data_ptr())
    monkeypatch.setattr(binding, "_token_rows", lambda t, *rest: (t.data_ptr(), t.stride(0)))
    q = torch.zeros(4, 2, 64).half()
    call = lambda layout: binding._rope_args(q, None, q, None, torch.zeros(4, 1), torch.zeros(32, dtype=torch.float64), None, layout, 1.0, False, None, 0)
    with pytest.raises(ValueError, match="layout is .* expected one of half, interleaved"):
        call(given)
    assert call("half")[19] == 0 and call("interleaved")[19] == 1
