"""ragged_attn_lse and ragged_attn_backward against the formulas in fp64 on the CPU.

Bounds, element by element.  u = half a step of the input type.  Scores: 64 products summed in fp32, off by 2^-18 |c| sum|q k| at most, and
with the exponential and the row statistics (2^-23 |L|) a probability is off by e = 2^-18 |c| max sum|q k| + 2^-22 (4 + |L|) of itself.
P and dS are rounded once (u), dP is a sum of 64 products (2^-18 sum|dO v|), delta carries the rounding of o (u sum|dO o|):
    dV: sum_i P |dO| (u + e);   dS: |dS| (u + e) + P (2^-17 sum|dO v| + u sum|dO o|) + |P dP| e;   dQ, dK: c sum of that |K|, |Q|
each with the last rounding (u) and, for fp16, values below its normal range (2^-25 each)."""
import numpy as np
import pytest
import torch

from paper_2604_15408_amd import binding, harness

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
D = 64
_TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


def _inputs(lengths, H, dtype, seed, fused=False, extra=3, times=1.0):
    gen = torch.Generator().manual_seed(seed)
    rows = int(sum(lengths))
    make = lambda *shape: (torch.randn(rows + extra, *shape, generator=gen) * times).to(_TYPES[dtype])
    if fused:
        qkv = make(3, H, D)
        qkv[rows:] = float("nan")                              # rows behind the last sequence are never read
        q, k, v = qkv.to(DEV).unbind(1)
    else:
        q, k, v = (make(H, D) for _ in range(3))
        for t in (q, k, v):
            t[rows:] = float("nan")
        q, k, v = (t.to(DEV) for t in (q, k, v))
    do = make(H, D)
    do[rows:] = float("nan")
    cu = torch.from_numpy(np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)).to(DEV)
    return rows, q, k, v, do.to(DEV), cu


def _run(q, k, v, do, cu, bound, scale, fused=False):
    rows, H, _ = q.shape
    o = torch.full((rows, H, D), 7.0, dtype=q.dtype, device=DEV)
    lse = torch.full((rows, H), 7.0, device=DEV)
    binding.ragged_attn_lse(q, k, v, o, lse, cu, bound, scale)
    if fused:
        dq, dk, dv = torch.full((rows, 3, H, D), 7.0, dtype=q.dtype, device=DEV).unbind(1)
    else:
        dq, dk, dv = (torch.full((rows, H, D), 7.0, dtype=q.dtype, device=DEV) for _ in range(3))
    binding.ragged_attn_backward(q, k, v, o, do, lse, dq, dk, dv, cu, bound, scale)
    return o, lse, dq, dk, dv


def _compare(q, k, v, do, cu, scale, out):
    o, lse, dq, dk, dv = (t.cpu().double() for t in out)
    u = torch.finfo(q.dtype).eps / 2
    tiny = 2.0 ** -25 if q.dtype == torch.float16 else 0.0
    c = abs(scale)
    ends = cu.tolist()
    for lo, hi in zip(ends[:-1], ends[1:]):
        if lo == hi:
            continue
        Q, K, V, dO, O = (t[lo:hi].cpu().double().transpose(0, 1) for t in (q, k, v, do, out[0]))
        T = lambda t: t.transpose(1, 2)
        S = scale * (Q @ T(K))
        L = torch.logsumexp(S, dim=-1)
        P = torch.exp(S - L[..., None])
        dP = dO @ T(V)
        exact_o = P @ V
        dS = P * (dP - (dO * exact_o).sum(-1, keepdim=True))
        size = c * (Q.abs() @ T(K.abs()))
        e = 2.0 ** -18 * size.amax(dim=-1, keepdim=True) + 2.0 ** -22 * (4 + L.abs()[..., None])
        assert torch.all((lse[lo:hi].transpose(0, 1) - L).abs() <= e[..., 0])
        b = dS.abs() * (u + e) + P * (2.0 ** -17 * (dO.abs() @ T(V.abs())) + u * (dO * O).abs().sum(-1, keepdim=True)) + (P * dP).abs() * e + tiny
        for got, want, bound in ((dv, T(P) @ dO, T(P * (u + e) + tiny) @ dO.abs()), (dq, scale * (dS @ K), c * (b @ K.abs())),
                                 (dk, scale * (T(dS) @ Q), c * (T(b) @ Q.abs()))):
            err = (got[lo:hi].transpose(0, 1) - want).abs()
            worst = (err - bound - u * want.abs() - tiny).max()
            assert worst <= 0, (lo, hi, float(worst), float(err.max()))


LENGTHS = [[1], [2, 1, 15], [0, 5, 0], [16, 17, 31, 32, 33], [63, 64, 65, 0], [40, 39, 41, 12], [96, 97, 127, 128, 129], [197, 40, 1, 0, 191],
           [577], [320, 3]]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("lengths", LENGTHS, ids=str)
def test_gradients(lengths, dtype):
    H, fused = (3, True) if len(lengths) % 2 else (2, False)
    rows, q, k, v, do, cu = _inputs(lengths, H, dtype, 5 + sum(lengths), fused)
    scale = 0.125
    out = _run(q, k, v, do, cu, max(lengths), scale, fused)
    _compare(q, k, v, do, cu, scale, out)
    for t in out:
        assert torch.all(t[rows:] == 7)                        # rows behind the last sequence as they were
    o = torch.full_like(out[0], 7.0)
    binding.ragged_attn_strided(q, k, v, o, cu, max(lengths), scale)
    assert torch.equal(o, out[0])
    # a larger bound and another pass: the same gradients, bit for bit
    o, lse = out[0], out[1]
    for bound in (max(lengths), max(lengths) + 1000):
        dq, dk, dv = (torch.full((q.shape[0], H, D), 7.0, dtype=q.dtype, device=DEV) for _ in range(3))
        binding.prepare_attn_backward(q, k, v, o, do, lse, dq, dk, dv, cu, bound, scale)()
        for a, b in zip((dq, dk, dv), out[2:]):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_few_keys(dtype):
    """Up to 32 keys delta is sum P dP in fp32 and carries no rounding of o: each dP is off by 2^-18 sum|dO v| and each P by e of itself, their
    sum over 32 keys by 2^-21 more.  One key has P = 1 whatever q and k are: dq and dk are zeros."""
    lengths, scale = [1, 2, 3, 1, 15, 16, 17, 31, 32, 8], 0.125
    rows, q, k, v, do, cu = _inputs(lengths, 3, dtype, 21)
    do[:rows] = do[:rows] * 0.1 + 1.0                          # delta well beside dP, as where the rounding of o would tell
    o, lse, dq, dk, dv = _run(q, k, v, do, cu, 32, scale)
    u, tiny = torch.finfo(q.dtype).eps / 2, 2.0 ** -25 if dtype == "f16" else 0.0
    ends = cu.tolist()
    for lo, hi in zip(ends[:-1], ends[1:]):
        if hi - lo == 1:
            assert torch.all(dq[lo] == 0) and torch.all(dk[lo] == 0) and torch.equal(dv[lo], do[lo])
            continue
        Q, K, V, dO = (t[lo:hi].cpu().double().transpose(0, 1) for t in (q, k, v, do))
        T = lambda t: t.transpose(1, 2)
        S = scale * (Q @ T(K))
        L = torch.logsumexp(S, dim=-1)
        P, dP = torch.exp(S - L[..., None]), dO @ T(V)
        dS = P * (dP - (P * dP).sum(-1, keepdim=True))
        e = 2.0 ** -18 * (scale * (Q.abs() @ T(K.abs()))).amax(dim=-1, keepdim=True) + 2.0 ** -22 * (4 + L.abs()[..., None])
        off = 2.0 ** -18 * (dO.abs() @ T(V.abs()))
        delta_off = (P * (dP.abs() * (e + 2.0 ** -21) + off)).sum(-1, keepdim=True)
        b = dS.abs() * (u + e) + P * (off + delta_off) + (P * dP).abs() * 2.0 ** -22 + tiny
        for got, want, bound in ((dq, scale * (dS @ K), scale * (b @ K.abs())), (dk, scale * (T(dS) @ Q), scale * (T(b) @ Q.abs()))):
            err = (got[lo:hi].cpu().double().transpose(0, 1) - want).abs()
            assert torch.all(err <= bound + u * want.abs() + tiny), (lo, hi, float((err - bound).max()))


@pytest.mark.parametrize("scale", [-0.25, 0.0, 1.0])
def test_scales(scale):
    rows, q, k, v, do, cu = _inputs([70, 20], 2, "f16", 11)
    _compare(q, k, v, do, cu, scale, _run(q, k, v, do, cu, 70, scale))


def test_large_scores_and_many_small_groups():
    """Scores of some hundred: most probabilities vanish; and a launch far larger than the small one's key-split form."""
    rows, q, k, v, do, cu = _inputs([130, 66], 2, "bf16", 12, times=6.0)
    _compare(q, k, v, do, cu, 0.125, _run(q, k, v, do, cu, 130, 0.125))
    lengths = [(7 * i) % 150 for i in range(90)]
    rows, q, k, v, do, cu = _inputs(lengths, 7, "f16", 13)
    _compare(q, k, v, do, cu, 0.125, _run(q, k, v, do, cu, 149, 0.125))


def test_sequences_do_not_reach_each_other():
    """A sequence's gradients are the same bits alone and among others, one of which holds NaN and infinities."""
    rows, q, k, v, do, cu = _inputs([50, 100, 9], 3, "f16", 14)
    alone = _run(*(t[50:150].contiguous() for t in (q, k, v, do)), torch.tensor([0, 100], dtype=torch.int32, device=DEV), 100, 0.125)
    for t in (q, k, v, do):
        t[:50] = float("nan")
        t[150:] = float("inf")
    among = _run(q, k, v, do, cu, 100, 0.125)
    for a, b in zip(alone[2:], among[2:]):
        assert torch.equal(a, b[50:150])


def test_differences():
    """The gradients against central differences of the fp64 forward pass along random directions."""
    rows, q, k, v, do, cu = _inputs([37], 2, "f16", 15, extra=0)
    _, _, dq, dk, dv = _run(q, k, v, do, cu, 37, 0.125)
    x = [t.cpu().double().transpose(0, 1) for t in (q, k, v, do)]
    loss = lambda q, k, v: ((torch.softmax(0.125 * (q @ k.transpose(1, 2)), -1) @ v) * x[3]).sum()
    gen = torch.Generator().manual_seed(16)
    for i, grad in enumerate((dq, dk, dv)):
        way = torch.randn(x[i].shape, generator=gen, dtype=torch.float64)
        h = 1e-5
        plus, minus = ([t + s * h * way if j == i else t for j, t in enumerate(x[:3])] for s in (1, -1))
        want = (loss(*plus) - loss(*minus)) / (2 * h)
        got = grad.cpu().double().transpose(0, 1)
        # each gradient is off by some steps of 2^-11 of its own size, with independent signs: four standard deviations of three steps
        sigma = 3 * 2.0 ** -11 * float((got.square().mean() * way.square().sum()).sqrt())
        assert abs((got * way).sum() - want) <= 4 * sigma + 1e-6 * abs(want)


def test_graph_and_streams():
    rows, q, k, v, do, cu = _inputs([197, 33, 64], 3, "bf16", 17, extra=0)
    want = _run(q, k, v, do, cu, 197, 0.125)
    o, lse, dq, dk, dv = (torch.zeros_like(t) for t in want)

    def step():
        binding.ragged_attn_lse(q, k, v, o, lse, cu, 197, 0.125)
        binding.ragged_attn_backward(q, k, v, o, do, lse, dq, dk, dv, cu, 197, 0.125)
    graph = harness.capture(torch, step)
    for _ in range(3):
        for t in (o, lse, dq, dk, dv):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((o, lse, dq, dk, dv), want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for t in (dq, dk, dv):
        t.zero_()
    torch.cuda.synchronize()
    binding.ragged_attn_backward(q, k, v, o, do, lse, dq, dk, dv, cu, 197, 0.125, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((dq, dk, dv), want[2:]))


def test_a_bound_that_is_too_small_leaves_rows():
    """Rows in 64-row tiles past the bound are left as they were; the others are right."""
    rows, q, k, v, do, cu = _inputs([150], 2, "f16", 18, extra=0)
    o, lse, *want = _run(q, k, v, do, cu, 150, 0.125)
    dq, dk, dv = (torch.full_like(t, 7.0) for t in want)
    binding.ragged_attn_backward(q, k, v, o, do, lse, dq, dk, dv, cu, 70, 0.125)
    for a, b in zip((dq, dk, dv), want):
        assert torch.equal(a[:128], b[:128]) and torch.all(a[128:] == 7)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_small_and_large_launches_agree(dtype):
    """The same sequences in a launch of their own (64 rows a work-group) and among many (128): the same bits."""
    lengths = [197, 65, 130, 33]
    rows, q, k, v, do, cu = _inputs(lengths, 3, dtype, 19, extra=0)
    few = _run(q, k, v, do, cu, 197, 0.125)
    many = 70
    more = torch.from_numpy(np.concatenate([[0], np.cumsum(lengths * many)]).astype(np.int32)).to(DEV)
    lot = [t.repeat(many, 1, 1) for t in (q, k, v, do)]
    o, lse = few[0].repeat(many, 1, 1), few[1].repeat(many, 1)
    grads = [torch.zeros_like(lot[0]) for _ in range(3)]
    binding.ragged_attn_backward(*lot[:3], o, lot[3], lse, *grads, more, 197, 0.125)
    for a, b in zip(few[2:], grads):
        assert torch.equal(a.repeat(many, 1, 1), b)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_lse_leaves_the_output_as_it_is(dtype):
    """Launches in phases and with key-split wavefronts: o is ragged_attn_strided's, bit for bit, and lse that of the row sums."""
    for lengths, H in (([577, 301] * 16, 12), ([300, 1, 64, 65, 128], 3)):
        rows, q, k, v, do, cu = _inputs(lengths, H, dtype, 20, extra=0)
        o, want = torch.full_like(q, 7.0), torch.full_like(q, 9.0)
        lse = torch.full((rows, H), 7.0, device=DEV)
        binding.prepare_attn_lse(q, k, v, o, lse, cu, max(lengths), -0.125)()
        binding.ragged_attn_strided(q, k, v, want, cu, max(lengths), -0.125)
        assert torch.equal(o, want)
        for i in (0, len(lengths) - 1):
            lo, hi = int(cu[i]), int(cu[i + 1])
            a, b = (t[lo:hi].cpu().double().transpose(0, 1) for t in (q, k))
            s = -0.125 * (a @ b.transpose(1, 2))
            e = 2.0 ** -18 * 0.125 * (a.abs() @ b.abs().transpose(1, 2)).amax(-1)
            L = torch.logsumexp(s, -1)
            assert torch.all((lse[lo:hi].cpu().double().transpose(0, 1) - L).abs() <= e + 2.0 ** -22 * (4 + L.abs()))


def test_rows_far_apart():
    """Token rows 4 MB apart: the last ones lie beyond 2^32 bytes of their tensors."""
    lengths, H, far = [600, 1, 499], 2, 1 << 21
    rows, q, k, v, do, cu = _inputs(lengths, H, "bf16", 21, extra=0)
    want = _run(q, k, v, do, cu, 600, 0.125)

    def apart(n):
        buffer = torch.empty((rows - 1) * far + n * H * D, dtype=q.dtype, device=DEV)
        return [buffer.as_strided((rows, H, D), (far, D, 1), i * H * D) for i in range(n)]
    ins, outs, grads = apart(3), apart(2), apart(3)
    for a, b in zip((*ins, outs[1]), (q, k, v, do)):
        a.copy_(b)
    lse = torch.zeros(rows, H, device=DEV)
    binding.ragged_attn_lse(*ins, outs[0], lse, cu, 600, 0.125)
    binding.ragged_attn_backward(*ins, *outs, lse, *grads, cu, 600, 0.125)
    for a, b in zip((outs[0], lse, *grads), want):
        assert torch.equal(a, b)
    freqs, coords = binding.rope_frequencies(32).to(DEV), torch.arange(rows, dtype=torch.float32, device=DEV).reshape(-1, 1)
    turned = torch.empty_like(q), torch.empty_like(k)
    binding.ragged_rope(q, k, *turned, coords, freqs)
    binding.ragged_rope(ins[0], ins[1], ins[0], ins[1], coords, freqs)
    assert torch.equal(ins[0], turned[0]) and torch.equal(ins[1], turned[1])
