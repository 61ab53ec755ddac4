"""Outputs that lie over what is still read, and those that only look like it (no GPU: the check takes any tensor's address)."""
import random

import pytest
import torch

from paper_2604_15408_amd import binding


@pytest.fixture(scope="module", params=["native", "ctypes"])
def placed(request):
    if not binding.LIB_PATH.exists():
        from paper_2604_15408_amd import build
        build.build()
    if request.param == "ctypes":
        return lambda written, *tensors: binding._Ctypes.placed(None, written, *tensors)
    native = binding._native()
    return lambda written, *tensors: native.placed(-1, written, *tensors)


def _bytes(t, most=None):
    """Every byte of a tensor, one by one."""
    if t.numel() == 0:
        return set()
    at = torch.zeros(1, dtype=torch.int64)
    for size, stride in zip(t.shape, t.stride()):
        at = (at[:, None] + torch.arange(size) * stride).reshape(-1)
    all_bytes = {t.data_ptr() + int(i) * t.element_size() + b for i in at for b in range(t.element_size())}
    return {b for b in all_bytes if most is None or b < t.data_ptr() + most}


def test_against_every_byte(placed):
    """Views of one buffer as the calls take them: contiguous ones, slices of rows at the same distance, ranges of rows of those."""
    rng = random.Random(1)
    for _ in range(400):
        width = rng.choice((12, 20))
        buffer = torch.zeros(width * 40, dtype=torch.float16)
        grid = buffer.view(40, width)

        def view():
            if rng.random() < 0.4:
                lo = rng.randrange(len(buffer))
                return buffer[lo:lo + rng.randrange(0, 60)]
            row, col = rng.randrange(40), rng.randrange(width)
            t = grid[row:row + rng.randrange(1, 12), col:col + 4 * rng.randrange(1, 4)]
            return t.unflatten(1, (-1, 4)) if t.shape[1] % 4 == 0 else t
        a, b, c = view(), view(), view()
        meet = lambda x, y: bool(_bytes(x) & _bytes(y))
        assert placed(1, a, b) == placed(1, b, a) == (2 if meet(a, b) else 0)
        assert placed(1, a, None, b, c) == (2 if meet(a, b) or meet(a, c) else 0)
        assert placed(2, a, b, c) == (2 if meet(a, b) or meet(a, c) or meet(b, c) else 0)
        assert placed(0, a, b, c) == 0


def test_rows_at_different_distances(placed):
    buffer = torch.zeros(1000, dtype=torch.float16)
    a, b = buffer[:400].view(20, 20)[:, :8], buffer[208:].as_strided((10, 4), (24, 1))
    assert placed(1, a, b) == 2
    assert placed(1, a, buffer[400:].as_strided((10, 4), (24, 1))) == 0


def test_a_workspace_is_as_long_as_it_is_used(placed):
    buffer = torch.zeros(100, dtype=torch.uint8)
    assert placed(1, (buffer, 60), buffer[60:]) == 0 and placed(1, (buffer, 61), buffer[60:]) == 2


def test_devices(placed):
    t = torch.zeros(4)
    assert placed(1, t, None) == 0 and binding._native().placed(0, 1, t) == 1 and binding._Ctypes.placed(0, 1, t) == 1
    assert binding._native().placed(-1, 1, t, "x") == 1
    with pytest.raises(TypeError):
        binding._native().placed(-1)


@pytest.fixture
def on_cpu(monkeypatch):
    """The calls' argument functions over CPU tensors: their checks of place are what is tested."""
    monkeypatch.setattr(binding, "_raw_device", lambda: None)
    monkeypatch.setattr(binding, "_native", lambda: binding._Ctypes)
    monkeypatch.setattr(binding, "_marshal", binding._Ctypes)
    monkeypatch.setattr(binding, "_dev", lambda t, *rest: t.data_ptr())
    monkeypatch.setattr(binding, "_rows_dev", lambda t: t.data_ptr())
    monkeypatch.setattr(binding, "_token_rows", lambda t, *rest: (t.data_ptr(), t.stride(0)))


T, H, D = 6, 2, 64


def _qkv(*shape, dtype=torch.float16):
    return torch.zeros(*shape, dtype=dtype)


def test_rope(on_cpu):
    fused, coords, freqs = _qkv(T + 1, 3, H, D), torch.zeros(8, 1), torch.zeros(32, dtype=torch.float64)
    q, k, v = fused[:T].unbind(1)
    call = lambda q, k, q_out, k_out, coords=coords: binding._rope_args(q, k, q_out, k_out, coords, freqs, None, "half", 1.0, False, None, 0)
    apart = _qkv(T, H, D), _qkv(T, H, D)
    for fine in ((q, k, q, k), (q, k, *apart), (q, None, q, None), (q, k, q, apart[0]), (q, k, v, apart[0])):
        call(*fine)
    down = fused[1:].unbind(1)
    for bad in ((q, k, down[0], apart[0]), (q, k, q, down[1]), (q, k, k, apart[0]), (q, k, apart[0], apart[0]), (q, k, apart[0], q),
                (q, None, down[0], None)):
        with pytest.raises(ValueError, match="overlaps"):
            call(*bad)
    with pytest.raises(ValueError, match="overlaps"):
        call(q, None, apart[0], None, apart[0].view(torch.float32).view(-1, 1)[:8])


def test_attention(on_cpu):
    fused, out, grads, cu = _qkv(T + 1, 3, H, D), _qkv(4, T + 1, H, D), _qkv(T + 1, 3, H, D), torch.zeros(2, dtype=torch.int32)
    q, k, v = fused[:T].unbind(1)
    o, d_o, lse = out[0, :T], out[1, :T], torch.zeros(T, H)
    forward = lambda o, lse: binding._attn_lse_args(q, k, v, o, lse, cu, T, 0.125, 0)
    backward = lambda dq, dk, dv: binding._attn_backward_args(q, k, v, o, d_o, lse, dq, dk, dv, cu, T, 0.125, 0)
    forward(o, lse)
    backward(*grads[:T].unbind(1))
    for bad in ((fused[1:].unbind(1)[2], lse), (o, o.view(torch.float32)[:, :, 0]), (o, k.view(torch.float32)[..., 0])):
        with pytest.raises(ValueError, match="overlaps"):
            forward(*bad)
    dq, dk, dv = grads[:T].unbind(1)
    for bad in ((fused[1:].unbind(1)[0], fused[1:].unbind(1)[1], fused[1:].unbind(1)[2]), (dq, dk, grads[1:].unbind(1)[1]), (dq, dq, dv)):
        with pytest.raises(ValueError, match="overlaps"):
            backward(*bad)
    shifted = out.view(-1)[H * D:].as_strided((T, H, D), (3 * H * D, D, 1))              # over o and its gradient, at another distance
    with pytest.raises(ValueError, match="overlaps"):
        backward(shifted, dk, dv)


def test_layernorm(on_cpu):
    C = 64
    flat = _qkv(4 * (T + 1), C)
    x, dy, res, dx = (flat[i * (T + 1):i * (T + 1) + T] for i in range(4))
    gamma, sums = _qkv(C), torch.zeros(2, C)
    workspace = torch.zeros(binding.layernorm_backward_workspace(T, C) + 4 * C, dtype=torch.uint8)
    call = lambda dx=dx, dgamma=sums[0], dbeta=sums[1], workspace=workspace, res=res: binding._layernorm_backward_args(
        x, gamma, dy, dx, dgamma, dbeta, workspace, res, None, 1e-6, 0)
    call()
    call(dx=dy)
    call(dx=res)
    call(dx=dx, res=None)
    call(dgamma=workspace[-4 * C:].view(torch.float32))        # behind what the call uses of the workspace
    for bad in (dict(dx=x), dict(dx=flat[T + 2:2 * T + 2]), dict(dx=flat[1:T + 1]), dict(dbeta=sums[0]), dict(dgamma=gamma.repeat(2).view(torch.float32),
                dbeta=workspace[:4 * C].view(torch.float32)), dict(workspace=flat.view(-1).view(torch.uint8))):
        with pytest.raises(ValueError, match="overlaps"):
            call(**bad)
