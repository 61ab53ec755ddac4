"""A whole training step (harness.AttentionTraining: pack, LayerNorm, linear, rotary positions, attention, and all of it back, then the clipping)
against differentiation of the same network in fp64.

Bound: a gradient's path rounds some twenty tensors to 16 bits, each off by at most half a step of its own size (u), and everything between
is a product with weights or features of size one: 40 u of the gradient's norm, twice what twenty roundings add up to at worst.  What
this test is for (an operator in the wrong place, a gradient added twice or not at all) is off by about the whole norm."""
import pytest
import torch

from paper_2604_15408_amd import harness
from paper_2604_15408_amd import workloads as wl

pytestmark = pytest.mark.gpu


def _rope(x, coords, freqs):
    at = coords.double()
    pairs = freqs.numel()
    angle = torch.cat([at[:, a:a + 1] * freqs[a * pairs // 2:(a + 1) * pairs // 2] for a in range(2)], dim=1)[:, None, :]
    p, q = x[..., :pairs], x[..., pairs:]
    return torch.cat((p * angle.cos() - q * angle.sin(), p * angle.sin() + q * angle.cos()), dim=-1)


def _reference(tr, d_last, T):
    """Gradients of sum(x_last * d_last) with respect to every parameter, in fp64 on the CPU."""
    w = tr.w
    names = ("ln1_g", "ln1_b", "w_qkv", "b_qkv", "w_o", "b_o")
    params = [{n: p[n].cpu().double().requires_grad_() for n in names} for p in tr.params]
    x = w.features().reshape(-1, w.C)[w.keep.reshape(-1).bool()].double()
    coords, freqs = tr.coords.cpu()[tr.gidx[:T].cpu().long() % w.N], tr.freqs.cpu()
    ends = tr.cu.cpu().tolist()
    for p in params:
        h = torch.nn.functional.layer_norm(x, (w.C,), p["ln1_g"], p["ln1_b"], harness.LN_EPS)
        q, k, v = (h @ p["w_qkv"].t() + p["b_qkv"]).reshape(T, 3, w.H, w.D).unbind(1)
        q, k = _rope(q, coords, freqs), _rope(k, coords, freqs)
        parts = []
        for lo, hi in zip(ends[:-1], ends[1:]):
            s = torch.einsum("ihd,jhd->hij", q[lo:hi], k[lo:hi]) * w.scale
            parts.append(torch.einsum("hij,jhd->ihd", torch.softmax(s, -1), v[lo:hi]))
        x = x + torch.cat(parts).reshape(T, w.C) @ p["w_o"].t() + p["b_o"]
    flat = [p[n] for p in params for n in names]
    return x.detach(), torch.autograd.grad((x * d_last).sum(), flat)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_training_step(dtype):
    B, N, H = 3, 50, 2
    keep = wl.keep_bernoulli(B, N, 0.6, 41)
    keep[1] = 0                                                # an image of which nothing is left
    w = wl.Workload("training", B, N, H, 64, dtype, 42, keep)
    tr = harness.AttentionTraining(w, depth=2, max_norm=1.0)
    T = w.T
    gen = torch.Generator().manual_seed(43)
    d_last = torch.zeros(B * N, w.C)
    d_last[:T] = torch.randn(T, w.C, generator=gen)
    d_last = d_last.to(tr.x_in.dtype)
    tr.forward()
    tr.backward(d_last.to("cuda:0"))
    tr.b.ragged_grad_clip(tr.plan, tr.norm, tr.max_norm)
    torch.cuda.synchronize()
    last, want = _reference(tr, d_last[:T].double(), T)
    u = torch.finfo(tr.x_in.dtype).eps / 2
    assert (tr.x[2][:T].cpu().double() - last).norm() <= 40 * u * last.norm()
    assert not tr.x[2][T:].any() and not tr.d_x[T:].any() and not tr.d_qkv[T:].any()
    got = [g for block in tr.grads for g in block.values()]
    for g, r in zip(got, want):
        off, size = (g.cpu().double().reshape(r.shape) - r).norm(), r.norm()
        assert off <= 40 * u * size, (tuple(r.shape), float(off / size))
    norm = torch.cat([g.double().reshape(-1) for g in got]).norm()
    assert abs(float(tr.norm) - float(norm)) <= 1e-12 * float(norm)
    clipped = torch.cat([g.double().reshape(-1) for g in got]) / (norm + 1e-6)
    assert torch.allclose(tr.clipped.double(), clipped, rtol=3e-7, atol=1e-30)


def test_steps_repeat():
    """Two steps of the same input give the same bits: nothing is added up in an order that changes, nothing is left from the first."""
    w = wl.Workload("training", 4, 197, 3, 64, "bf16", 44, wl.keep_bernoulli(4, 197, 0.5, 45))
    tr = harness.AttentionTraining(w, depth=2)
    tr.run()
    first = tr.clipped.clone(), tr.norm.clone()
    tr.run()
    torch.cuda.synchronize()
    assert torch.equal(first[0], tr.clipped) and torch.equal(first[1], tr.norm)
