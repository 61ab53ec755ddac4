"""ragged_grad_clip where the factor leaves fp32's normal range though gradients and outputs are ordinary numbers.  Bounds as for the other
tests of clipping: factor and product are rounded to fp32 (2^-24 each), then to the output's type."""
import math

import pytest
import torch

from paper_2604_15408_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("out", [torch.float32, None], ids=["f32", "norm only besides"])
@pytest.mark.parametrize("times,max_norm,scale", [(1e38, 1.0, 1.0), (3e38, 1.0, 1.0), (1e38, 1e-7, 1.0), (1e30, 1e-20, 1.0), (1e20, 1e-30, 1.0),
                                                  (1e38, 1.0, 1e-9), (1e37, 1.0, -1e30), (1e-30, 1e-38, 1.0), (2.0, 1e9, 1e-39)])
def test_small_factors(times, max_norm, scale, out):
    gen = torch.Generator(device=DEV).manual_seed(61)
    g = [(torch.rand(1000, generator=gen, device=DEV) + 0.1) * times, -torch.rand(77, generator=gen, device=DEV) * times * 1e-3]
    outs = [torch.full_like(g[0], 7.0), None if out is None else torch.full_like(g[1], 7.0)]
    norm = torch.zeros(1, dtype=torch.float64, device=DEV)
    scale = torch.tensor(scale).item()                         # (an fp32 number, as the call takes it)
    binding.ragged_grad_clip(binding.GradPlan(g, outs), norm, max_norm, scale)
    want = abs(scale) * math.sqrt(math.fsum(float(t.double().square().sum()) for t in g))
    assert abs(float(norm) - want) <= 1e-12 * want
    factor = scale * min(1.0, torch.tensor(max_norm).item() / (want + 1e-6))
    for t, o in zip(g, outs):
        if o is not None:
            w = t.double() * factor
            assert torch.all((o.double() - w).abs() <= (2.0 ** -24 + 2.0 ** -22) * w.abs() + 2.0 ** -149), float(((o.double() - w) / w).abs().max())


def test_half_gradients_and_small_factors():
    """In place and into fp32: 60 000 with a largest norm of 1e-40, which is below fp32's normal range itself."""
    for dtype in (torch.float16, torch.bfloat16):
        g = [torch.full((500,), 60000.0, device=DEV).to(dtype)]
        out, norm = [torch.empty(500, device=DEV)], torch.zeros(1, dtype=torch.float64, device=DEV)
        most = torch.tensor(1e-36).item()
        binding.ragged_grad_clip(binding.GradPlan(g, out), norm, most)
        want = float(g[0][0]) * (most / (float(norm) + 1e-6))
        assert torch.all((out[0].double() - want).abs() <= 2.0 ** -22 * want + 2.0 ** -149)
