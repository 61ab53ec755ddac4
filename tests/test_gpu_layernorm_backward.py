"""ragged_layernorm_backward against the formulas in fp64.

Bounds: sums over a row in fp32 (at most 40 roundings on the way of a value) leave mean, w's mean and the mean of w xh off by 40 * 2^-24 of the
mean size of what is added, xh by 3e-6 of 1 + |xh| and of the mean: 1e-5 of the terms of dx, and half a step of the output.  A column's
sums have at most 120 roundings on a value's way: 120 * 2^-24 = 7e-6 of the sum of sizes, and the error of xh: 2e-5."""
import pytest
import torch

from paper_2604_15408_amd import binding, harness

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
_TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


def _reference(x, gamma, dy, res, eps):
    x, gamma, dy = x.double(), gamma.double(), dy.double()
    mean = x.mean(1, keepdim=True)
    rstd = 1 / ((x - mean).square().mean(1, keepdim=True) + eps).sqrt()
    xh, w = (x - mean) * rstd, dy * gamma
    dx = rstd * (w - w.mean(1, keepdim=True) - xh * (w * xh).mean(1, keepdim=True))
    spread = 1 + rstd * x.abs().mean(1, keepdim=True)          # of what xh is made, relative to xh
    size = rstd * (w.abs() + w.abs().mean(1, keepdim=True) + xh.abs() * (w * xh).abs().mean(1, keepdim=True)) * spread
    if res is not None:
        dx = dx + res.double()
    return dx, size, (dy * xh).sum(0), (dy.abs() * (xh.abs() + spread)).sum(0), dy.sum(0), dy.abs().sum(0)


def _check(x, gamma, dy, res, rows, eps, dx, dgamma, dbeta):
    want, size, wg, sg, wb, sb = _reference(x[:rows], gamma, dy[:rows], None if res is None else res[:rows], eps)
    u = torch.finfo(x.dtype).eps / 2
    err = (dx[:rows].double() - want).abs()
    assert torch.all(err <= u * want.abs() + 1e-5 * size + 2.0 ** -25), float((err - u * want.abs() - 1e-5 * size).max())
    assert torch.all((dgamma.double() - wg).abs() <= 2e-5 * sg)
    assert torch.all((dbeta.double() - wb).abs() <= 1e-5 * sb)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("C", [8, 64, 128, 192, 256, 264, 384, 512, 520, 768, 776, 1000, 1024, 1032, 1536, 2040, 2048])
def test_layernorm_backward(C, dtype):
    tdt = _TYPES[dtype]
    gen = torch.Generator(device=DEV).manual_seed(C)
    gamma = (torch.randn(C, generator=gen, device=DEV) * 0.5 + 1).to(tdt)
    for cap, rows in ((1, 1), (3, 2), (33, 33), (70, 5), (197, 196), (8200, 8195)):
        x, dy, res = (torch.randn(cap, C, generator=gen, device=DEV).mul(s).add(m).to(tdt) for s, m in ((2, 0.75), (1, 0), (1, 0.5)))
        workspace = torch.full((binding.layernorm_backward_workspace(cap, C),), 255, dtype=torch.uint8, device=DEV)    # NaN words
        valid = torch.tensor([rows], dtype=torch.int32, device=DEV)
        dgamma, dbeta = torch.full((2, C), 7.0, device=DEV)
        dx = torch.full_like(x, 7.0)
        binding.ragged_layernorm_backward(x, gamma, dy, dx, dgamma, dbeta, workspace, rows_dev=valid)
        _check(x, gamma, dy, None, rows, 1e-6, dx, dgamma, dbeta)
        assert torch.all(dx[rows:] == 7)
        # the residual's gradient, in place of it; then in place of dy: the same bits; the same sums again
        sums = dgamma.clone(), dbeta.clone()
        both = res.clone()
        binding.ragged_layernorm_backward(x, gamma, dy, both, dgamma, dbeta, workspace, residual_grad=both, rows_dev=valid)
        _check(x, gamma, dy, res, rows, 1e-6, both, dgamma, dbeta)
        assert torch.equal(both[rows:], res[rows:]) and torch.equal(dgamma, sums[0]) and torch.equal(dbeta, sums[1])
        own = dy.clone()
        binding.prepare_layernorm_backward(x, gamma, own, own, dgamma, dbeta, workspace, residual_grad=res, rows_dev=valid)()
        assert torch.equal(own[:rows], both[:rows]) and torch.equal(own[rows:], dy[rows:]) and torch.equal(dgamma, sums[0])


def test_no_rows():
    x = torch.randn(9, 64, device=DEV).half()
    gamma, dx = torch.ones(64, dtype=torch.float16, device=DEV), torch.full_like(x, 7.0)
    workspace = torch.full((binding.layernorm_backward_workspace(9, 64),), 255, dtype=torch.uint8, device=DEV)
    for none in (0, -4):
        dgamma, dbeta = torch.full((2, 64), 7.0, device=DEV)
        binding.ragged_layernorm_backward(x, gamma, x, dx, dgamma, dbeta, workspace, rows_dev=torch.tensor([none], dtype=torch.int32, device=DEV))
        assert torch.all(dx == 7) and not dgamma.any() and not dbeta.any()


def test_eps_zero_and_rows_behind_the_last():
    """Without eps a lane behind the last row (three of four rows of a wavefront) would divide by zero into the sums."""
    x, dy = torch.randn(2, 5, 64, device=DEV).half()
    gamma, dx = torch.ones(64, dtype=torch.float16, device=DEV), torch.empty_like(x)
    dgamma, dbeta = torch.empty(2, 64, device=DEV)
    workspace = torch.empty(binding.layernorm_backward_workspace(5, 64), dtype=torch.uint8, device=DEV)
    binding.ragged_layernorm_backward(x, gamma, dy, dx, dgamma, dbeta, workspace, eps=0.0)
    _check(x, gamma, dy, None, 5, 0.0, dx, dgamma, dbeta)


def test_infinity_stays_in_its_row():
    x, dy = torch.randn(2, 40, 768, device=DEV).bfloat16()
    x[7, 3] = float("inf")
    gamma, dx = torch.ones(768, dtype=torch.bfloat16, device=DEV), torch.empty_like(x)
    dgamma, dbeta = torch.empty(2, 768, device=DEV)
    workspace = torch.empty(binding.layernorm_backward_workspace(40, 768), dtype=torch.uint8, device=DEV)
    binding.ragged_layernorm_backward(x, gamma, dy, dx, dgamma, dbeta, workspace)
    fine = torch.isfinite(dx).all(dim=1)
    assert not fine[7] and fine[:7].all() and fine[8:].all() and torch.isfinite(dbeta).all()


def test_differences():
    """Against central differences of the fp64 forward pass along random directions."""
    gen = torch.Generator().manual_seed(2)
    x, dy = torch.randn(2, 6, 192, generator=gen).half()
    gamma = torch.randn(192, generator=gen).half()
    dx, (dgamma, dbeta) = torch.empty(6, 192, dtype=torch.float16, device=DEV), torch.empty(2, 192, device=DEV)
    workspace = torch.empty(binding.layernorm_backward_workspace(6, 192), dtype=torch.uint8, device=DEV)
    binding.ragged_layernorm_backward(x.to(DEV), gamma.to(DEV), dy.to(DEV), dx, dgamma, dbeta, workspace)

    def loss(x, gamma, beta):
        return (torch.nn.functional.layer_norm(x, (192,), gamma, beta, 1e-6) * dy.double()).sum()
    at = [x.double(), gamma.double(), torch.zeros(192, dtype=torch.float64)]
    for i, grad in enumerate((dx, dgamma, dbeta)):
        way, h = torch.randn(at[i].shape, generator=gen, dtype=torch.float64), 1e-5
        plus, minus = ([t + s * h * way if j == i else t for j, t in enumerate(at)] for s in (1, -1))
        want, got = (loss(*plus) - loss(*minus)) / (2 * h), (grad.cpu().double() * way).sum()
        step = 2.0 ** -11 if i == 0 else 2e-5
        assert abs(got - want) <= step * float((grad.cpu().double() * way).abs().sum()) + 1e-6


def test_graph():
    x, dy = torch.randn(2, 500, 384, device=DEV).bfloat16()
    gamma, dx = torch.randn(384, device=DEV).bfloat16(), torch.empty_like(x)
    dgamma, dbeta = torch.empty(2, 384, device=DEV)
    workspace = torch.empty(binding.layernorm_backward_workspace(500, 384), dtype=torch.uint8, device=DEV)
    call = lambda: binding.ragged_layernorm_backward(x, gamma, dy, dx, dgamma, dbeta, workspace)
    graph = harness.capture(torch, call)
    for _ in range(3):
        x.normal_()
        call()
        want = dx.clone(), dgamma.clone(), dbeta.clone()
        for t in (dx, dgamma, dbeta):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((dx, dgamma, dbeta), want))


@pytest.mark.parametrize("C,rows", [(128, 140001), (256, 70003), (512, 33001), (768, 22003), (1024, 17001), (1536, 11003)])
def test_tensors_larger_than_the_caches(C, rows):
    """More than 32 MB a tensor: the same bits of dx as in pieces, and the sums of the formulas."""
    gen = torch.Generator(device=DEV).manual_seed(C + 1)
    x, dy, res = (torch.randn(rows, C, generator=gen, device=DEV).add(0.5).half() for _ in range(3))
    gamma = torch.randn(C, generator=gen, device=DEV).half()
    dx, want = torch.empty_like(x), torch.empty_like(x)
    (dgamma, dbeta), spare = torch.empty(2, C, device=DEV), torch.empty(C, device=DEV)
    workspace = torch.empty(binding.layernorm_backward_workspace(rows, C), dtype=torch.uint8, device=DEV)
    binding.ragged_layernorm_backward(x, gamma, dy, dx, dgamma, dbeta, workspace, residual_grad=res)
    for lo in range(0, rows, 7000):
        s = slice(lo, min(lo + 7000, rows))
        binding.ragged_layernorm_backward(x[s], gamma, dy[s], want[s], spare, spare.clone(), workspace, residual_grad=res[s])
    assert torch.equal(dx, want)
    _, _, wg, sg, wb, sb = _reference(x, gamma, dy, None, 1e-6)
    # (a column's values pass up to 500 additions here: 500 * 2^-24 = 3e-5 of the sum of sizes, and the error of xh)
    assert torch.all((dgamma.double() - wg).abs() <= 5e-5 * sg) and torch.all((dbeta.double() - wb).abs() <= 4e-5 * sb)


def test_more_than_four_gigabytes():
    """The last rows lie beyond 2^32 bytes; they are what they are in a call of their own."""
    rows, C, last = 1060003, 2048, 1001
    x = torch.zeros(rows, C, dtype=torch.bfloat16, device=DEV)
    dy = torch.zeros_like(x)
    x[-last:].normal_()
    dy[-last:].normal_()
    gamma, sums = torch.ones(C, dtype=torch.bfloat16, device=DEV), torch.empty(4, C, device=DEV)
    workspace = torch.empty(binding.layernorm_backward_workspace(rows, C), dtype=torch.uint8, device=DEV)
    want, dx = torch.empty_like(x[-last:]), torch.full_like(x, 7.0)
    binding.ragged_layernorm_backward(x[-last:], gamma, dy[-last:], want, sums[0], sums[1], workspace)
    binding.ragged_layernorm_backward(x, gamma, dy, dx, sums[2], sums[3], workspace)
    assert torch.equal(dx[-last:], want) and not dx[:-last].any()
    size = dy[-last:].double().abs().sum(0)
    assert torch.all((sums[3].double() - sums[1].double()).abs() <= 2e-5 * size)      # (both off by 1e-5 of it at most)
