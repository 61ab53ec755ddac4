"""harness.AttentionTraining over steps that differ: another mask with fewer tokens, other features.  Every step is the same bits as on a fresh
object."""
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
