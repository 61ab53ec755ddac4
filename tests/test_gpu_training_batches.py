"""harness.AttentionTraining over steps that differ: another mask with fewer tokens, other features, weights that an optimiser has changed.  Every
step is the same bits as on a fresh object."""
import pytest
import torch

from paper_2604_15408_amd import harness
from paper_2604_15408_amd import workloads as wl

pytestmark = pytest.mark.gpu
B, N, H = 4, 50, 2


def _training(keep, seed, dtype):
    return harness.AttentionTraining(wl.Workload("training", B, N, H, 64, dtype, seed, keep), depth=2)


def _results(tr):
    torch.cuda.synchronize()
    return [g.clone() for block in tr.grads for g in block.values()] + [tr.clipped.clone(), tr.norm.clone()]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_a_step_with_fewer_tokens_after_a_dense_one(dtype):
    dense, sparse = wl.keep_bernoulli(B, N, 1.0, 51), wl.keep_bernoulli(B, N, 0.3, 52)
    sparse[2] = 0
    tr, fresh = _training(dense, 53, dtype), _training(sparse, 54, dtype)
    tr.x_in[1, 7, 3] = float("nan")                            # a batch that went wrong leaves nothing behind either
    tr.run()
    tr.keep.copy_(fresh.keep)
    tr.x_in.copy_(fresh.x_in)
    tr.run()
    fresh.run()
    assert all(torch.equal(a, b) for a, b in zip(_results(tr), _results(fresh)))


def test_a_step_after_an_update_of_the_weights():
    keep = wl.keep_bernoulli(B, N, 0.5, 55)
    tr, fresh = _training(keep, 56, "bf16"), _training(keep, 56, "bf16")
    tr.run()
    before = _results(tr)
    for ours, theirs in zip(tr.params, fresh.params):          # (an update as large as the weights, so that the old ones would show)
        for name, times in (("w_qkv", -2.0), ("w_o", 2.0)):
            ours[name].mul_(times)
            theirs[name].copy_(ours[name])
    tr.run()
    fresh.run()
    assert all(torch.equal(a, b) for a, b in zip(_results(tr), _results(fresh)))
    assert not torch.equal(before[0], _results(tr)[0])
    # against differentiation: what reaches the first block's LayerNorm has gone through both transposed weights
    params = [{n: p[n].cpu().double().requires_grad_() for n in ("ln1_g", "ln1_b", "w_qkv", "b_qkv", "w_o", "b_o")} for p in tr.params]
    T, w = tr.w.T, tr.w
    x = tr.x[0][:T].cpu().double()
    at = tr.coords.cpu()[tr.gidx[:T].cpu().long() % N].double()
    freqs, ends = tr.freqs.cpu(), tr.cu.cpu().tolist()
    angle = torch.cat([at[:, a:a + 1] * freqs[a * 16:(a + 1) * 16] for a in range(2)], dim=1)[:, None, :]
    turned = lambda t: torch.cat((t[..., :32] * angle.cos() - t[..., 32:] * angle.sin(), t[..., :32] * angle.sin() + t[..., 32:] * angle.cos()), dim=-1)
    for p in params:
        q, k, v = (torch.nn.functional.layer_norm(x, (w.C,), p["ln1_g"], p["ln1_b"], harness.LN_EPS) @ p["w_qkv"].t() + p["b_qkv"]).reshape(T, 3, H, 64).unbind(1)
        q, k = turned(q).transpose(0, 1), turned(k).transpose(0, 1)
        parts = [torch.softmax(q[:, lo:hi] @ k[:, lo:hi].transpose(1, 2) * w.scale, -1) @ v.transpose(0, 1)[:, lo:hi] for lo, hi in zip(ends[:-1], ends[1:])]
        x = x + torch.cat(parts, dim=1).transpose(0, 1).reshape(T, w.C) @ p["w_o"].t() + p["b_o"]
    names = [(i, n) for i in range(2) for n in ("ln1_g", "ln1_b")]
    want = torch.autograd.grad((x * x).sum() / 2, [params[i][n] for i, n in names])
    for (i, n), g in zip(names, want):                         # (40 roundings of half a step, as for the whole step; d_last is the rounded x)
        assert (tr.grads[i][n].cpu().double() - g).norm() <= 40 * 2.0 ** -8 * g.norm(), (i, n)
