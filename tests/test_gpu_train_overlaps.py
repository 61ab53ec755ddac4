"""On the GPU: outputs over what is still read are refused before anything is launched, views between each other's rows are not."""
import pytest
import torch

from paper_2604_15408_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_shifted_by_a_row():
    T, H, D = 40, 2, 64
    fused = torch.randn(T + 1, 3, H, D, device=DEV).half()
    kept = fused.clone()
    q, k, v = fused[:T].unbind(1)
    down = fused[1:].unbind(1)
    cu = torch.tensor([0, T], dtype=torch.int32, device=DEV)
    o, lse, freqs = torch.zeros(T, H, D, device=DEV).half(), torch.zeros(T, H, device=DEV), binding.rope_frequencies(32).to(DEV)
    coords = torch.arange(T, dtype=torch.float32, device=DEV).reshape(-1, 1)
    with pytest.raises(ValueError, match="overlaps"):
        binding.ragged_attn_backward(q, k, v, o, o.clone(), lse, *down, cu, T, 0.125)
    with pytest.raises(ValueError, match="overlaps"):
        binding.ragged_rope(q, k, down[0], down[1], coords, freqs)
    with pytest.raises(ValueError, match="overlaps"):
        binding.prepare_attn_lse(q, k, v, o, o.view(torch.float32)[..., 0], cu, T, 0.125)
    flat = torch.randn(T + 1, 64, device=DEV).half()
    workspace = torch.empty(binding.layernorm_backward_workspace(T, 64), dtype=torch.uint8, device=DEV)
    gamma, sums = torch.ones(64, device=DEV).half(), torch.zeros(2, 64, device=DEV)
    with pytest.raises(ValueError, match="overlaps"):
        binding.ragged_layernorm_backward(flat[:T], gamma, flat[:T].clone(), flat[1:], sums[0], sums[1], workspace)
    torch.cuda.synchronize()
    assert torch.equal(fused, kept) and not sums.any()


def test_gradients_between_the_rows_of_their_inputs():
    """q, k, v and dq, dk, dv as the six slices of one buffer: the same bits as in buffers of their own."""
    T, H, D = 100, 2, 64
    gen = torch.Generator(device=DEV).manual_seed(1)
    six = torch.randn(T, 6, H, D, generator=gen, device=DEV).half()
    q, k, v, *grads = six.unbind(1)
    cu = torch.tensor([0, 30, T], dtype=torch.int32, device=DEV)
    do, o, lse = torch.randn(T, H, D, generator=gen, device=DEV).half(), torch.empty(T, H, D, device=DEV).half(), torch.empty(T, H, device=DEV)
    binding.ragged_attn_lse(q, k, v, o, lse, cu, T, 0.125)
    own = [torch.empty_like(o) for _ in range(3)]
    binding.ragged_attn_backward(q, k, v, o, do, lse, *own, cu, T, 0.125)
    binding.ragged_attn_backward(q, k, v, o, do, lse, *grads, cu, T, 0.125)
    assert all(torch.equal(a, b) for a, b in zip(own, grads))
