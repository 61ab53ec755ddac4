"""A bound below the length of a sequence, given to the forward and the backward call alike: what of that sequence's gradients is still right, and
that nothing else is touched by it.  (The keys' gradients of such a sequence are sums over queries whose o and lse were never written.)"""
import numpy as np
import pytest
import torch

from paper_2604_15408_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
H, D = 2, 64


def _forward(q, k, v, cu, bound):
    o, lse = torch.full_like(q, float("nan")), torch.full(q.shape[:2], float("nan"), device=DEV)
    binding.ragged_attn_lse(q, k, v, o, lse, cu, bound, 0.125)
    return o, lse


def _backward(q, k, v, do, cu, bound, o, lse):
    grads = [torch.full_like(q, 7.0) for _ in range(3)]
    binding.ragged_attn_backward(q, k, v, o, do, lse, *grads, cu, bound, 0.125)
    return grads


# few sequences (64 rows a work-group) and many (128)
@pytest.mark.parametrize("times", [1, 150])
@pytest.mark.parametrize("bound", [1, 70, 149])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_one_bound_too_small_for_a_sequence(dtype, bound, times):
    lengths = [150] + [min(bound, 40), min(bound, 70)] * times + [300]
    gen = torch.Generator().manual_seed(bound + times)
    q, k, v, do = (torch.randn(sum(lengths), H, D, generator=gen).to(dtype).to(DEV) for _ in range(4))
    ends = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    cu = torch.from_numpy(ends).to(DEV)
    o, lse = _forward(q, k, v, cu, bound)
    # (o of a long sequence may differ in its last place from launch to launch: what this one has written is taken over)
    all_o, all_lse = (torch.where(torch.isnan(a), b, a) for a, b in zip((o, lse), _forward(q, k, v, cu, 300)))
    want = _backward(q, k, v, do, cu, 300, all_o, all_lse)
    got = _backward(q, k, v, do, cu, bound, o, lse)
    inside = slice(150, int(ends[-2]))                         # sequences that the bound holds for
    for a, b in zip(want, got):
        assert torch.equal(a[inside], b[inside])
    for lo, n in ((0, 150), (int(ends[-2]), 300)):
        assert torch.equal(want[0][lo:lo + bound], got[0][lo:lo + bound])          # dq of the rows below the bound
        for a, b in zip(want, got):                            # a row past the last tile of 128 below the bound is as it was
            first = lo + (bound + 127) // 128 * 128
            assert torch.all(b[first:lo + n] == 7)
    # o and lse of all rows: the keys' gradients below the bound are right as well
    grads = _backward(q, k, v, do, cu, bound, all_o, all_lse)
    for a, b in zip(want, grads):
        assert torch.equal(a[inside], b[inside])
        for lo in (0, int(ends[-2])):
            assert torch.equal(a[lo:lo + bound], b[lo:lo + bound])
