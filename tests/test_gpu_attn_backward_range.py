"""Attention's gradients in fp16 where P and dS leave fp16's own range: tiny and huge gradients of the output, many keys, in every form
(up to 32 rows, up to 64, longer).

What bounds a gradient, u = 2^-11.  dS is rounded once, independently from element to element: u |dS|, and it is carried with a power of two F, so
that what lies below the normal range is off by 2^-25 / F: F is at least 2^-16 * 2^16 / max|dP - delta| (the last attempt that overflowed had 16
binades more), with |dP - delta| <= 2 |dO| |v|: 2^-24 max|dO| max|v| at most.  P is carried with 2^15: 2^-40.  The rest goes the same way in a whole row or
column: e = 2^-18 |c| max sum|q k| + 2^-22 (6 + |L|) of P, 2^-17 sum|dO v| of dP and u sum|dO o| of delta.
Element by element these add up (as for the other tests of the gradients).  Over all elements the independent part adds up by squares: an error of at
most b has a standard deviation of b / sqrt 3 at most, so that 3 times the root of the sum of b^2 is five standard deviations."""
import numpy as np
import pytest
import torch

from paper_2604_15408_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
D = 64
U, OUT = 2.0 ** -11, 2.0 ** -25                                # half a step of fp16: relative, and below its normal range


def _run(q, k, v, do, lengths, scale):
    cu = torch.from_numpy(np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)).to(DEV)
    q, k, v, do = (t.to(DEV) for t in (q, k, v, do))
    o, lse = torch.empty_like(q), torch.empty(q.shape[:2], device=DEV)
    dq, dk, dv = (torch.full_like(q, 7.0) for _ in range(3))
    binding.ragged_attn_lse(q, k, v, o, lse, cu, max(lengths), scale)
    binding.ragged_attn_backward(q, k, v, o, do, lse, dq, dk, dv, cu, max(lengths), scale)
    return [t.cpu() for t in (o, dq, dk, dv)]


def _check(q, k, v, do, lengths, scale, out):
    T = lambda t: t.transpose(1, 2)
    c = abs(scale)
    lo = 0
    for n in lengths:
        s = slice(lo, lo + n)
        lo += n
        Q, K, V, dO, O = (t[s].double().transpose(0, 1) for t in (q, k, v, do, out[0]))
        S = scale * (Q @ T(K))
        L = torch.logsumexp(S, dim=-1)
        P, dP = torch.exp(S - L[..., None]), dO @ T(V)
        dS = P * (dP - (P * dP).sum(-1, keepdim=True))
        e = 2.0 ** -18 * c * (Q.abs() @ T(K.abs())).amax(dim=-1, keepdim=True) + 2.0 ** -22 * (6 + L.abs()[..., None])
        off = 2.0 ** -17 * (dO.abs() @ T(V.abs()))
        row = dS.abs() * e + P * (off + (P * off).sum(-1, keepdim=True) + U * (dO * O).abs().sum(-1, keepdim=True)) + (P * dP).abs() * e \
            + P * (P * dP.abs()).sum(-1, keepdim=True) * (e + 2.0 ** -21)
        one = U * dS.abs() + 2.0 ** -24 * float(dO.norm(dim=-1).max() * V.norm(dim=-1).max())
        for got, want, independent, common, x, times in (
                (out[1], scale * (dS @ K), one, row, K, c), (out[2], scale * (T(dS) @ Q), T(one), T(row), Q, c),
                (out[3], T(P) @ dO, T(U * P + 2.0 ** -40), T(P * e), dO, 1.0)):
            got = got[s].transpose(0, 1).double()
            fits, beyond = want.abs() < 60000, want.abs() > 80000                  # an output beyond fp16 is infinite, and right so
            assert torch.isfinite(got[fits]).all(), (n, int((~torch.isfinite(got[fits])).sum()))
            assert torch.equal(got[beyond], want[beyond].sign() * float("inf"))
            err = torch.where(fits, got - want, 0.0)
            rounding = U * want.abs() + OUT
            bound = times * ((independent + common) @ x.abs()) + rounding
            assert torch.all(err.abs() <= bound), (n, float((err.abs() / bound).max()))
            spread = (times ** 2 * (independent.square() @ x.square()) + rounding.square())[fits].sum().sqrt()
            limit = 3 * spread + (times * (common @ x.abs()))[fits].norm()
            assert err.norm() <= limit, (n, float(err.norm() / limit))


def _inputs(lengths, H, seed, q_times, k_times, do_times):
    gen = torch.Generator().manual_seed(seed)
    make = lambda times: (torch.randn(sum(lengths), H, D, generator=gen) * times).half()
    return make(q_times), make(k_times), make(1.0), make(do_times)


LENGTHS = [[2, 3, 9, 17, 32], [33, 50, 64], [65, 100, 197], [577]]


# one of dq and dk far smaller than the other, so that either can be seen above fp16's own lower end
@pytest.mark.parametrize("q_times,k_times", [(16.0, 2.0 ** -7), (2.0 ** -7, 16.0)])
@pytest.mark.parametrize("do_times", [2.0 ** -18, 1e-4, 1.0, 2.0 ** 12])
@pytest.mark.parametrize("lengths", LENGTHS, ids=str)
def test_sizes_of_the_output_gradient(lengths, do_times, q_times, k_times):
    q, k, v, do = _inputs(lengths, 2, len(lengths) + lengths[0], q_times, k_times, do_times)
    _check(q, k, v, do, lengths, 1.0, _run(q, k, v, do, lengths, 1.0))


def test_dS_beyond_the_largest_number():
    """q = 0, two keys, v = 1 and -1, dO = 4096: dS = 131072, dq = 327.68."""
    q, do = torch.zeros(2, 1, D).half(), torch.full((2, 1, D), 4096.0).half()
    k, v = torch.full((2, 1, D), 0.01).half(), torch.ones(2, 1, D).half()
    k[1], v[1] = -k[0], -1
    out = _run(q, k, v, do, [2], 0.125)
    want = 2 * 0.125 * 131072 * float(k[0, 0, 0])
    assert torch.all((out[1].double() - want).abs() <= 2 * U * want) and not out[2].any() and not out[3][:, 0, 0].isnan().any()


# every sixteenth row of 241 holds next to nothing, or every other one does: the size of what is coming cannot be told from them
@pytest.mark.parametrize("rare", [2.0 ** -20, 2.0 ** 20])
@pytest.mark.parametrize("what", ["do", "v", "both"])
def test_rows_of_very_different_sizes(what, rare):
    lengths = [241, 241]
    q, k, v, do = _inputs(lengths, 2, 31, 2.0, 2.0 ** -2, 1.0)
    odd = (torch.arange(482) % 241 % 16 == 0)[:, None, None]
    times = torch.where(odd, rare, 1.0) * (2.0 ** 9 if rare < 1 else 2.0 ** -11)
    if what != "v":
        do = (do.float() * times).half()
    if what != "do":
        v = (v.float() * times * 2.0 ** (-6 if rare < 1 else 3)).half()
    _check(q, k, v, do, lengths, 0.125, _run(q, k, v, do, lengths, 0.125))


def test_values_that_are_no_numbers_stay_in_their_sequence():
    lengths = [20, 60, 200, 20, 60, 200]
    q, k, v, do = _inputs(lengths, 2, 32, 1.0, 1.0, 1.0)
    want = _run(q, k, v, do, lengths, 0.125)
    do[100, 0, 3], v[0, 1, 5], do[30, 1, 7] = float("nan"), float("inf"), float("inf")
    got = _run(q, k, v, do, lengths, 0.125)
    assert all(torch.equal(a[280:], b[280:]) for a, b in zip(got, want))
    assert all(torch.equal(a[80:280, 1], b[80:280, 1]) for a, b in zip(got, want))
    assert torch.isnan(got[2][80:280, 0]).all()


@pytest.mark.parametrize("zero", ["q", "k"])
def test_equal_scores_of_many_keys(zero):
    """70 000 keys of the same probability, 1.4e-5: 240 steps of fp16's lowest range.  All scores are 0, so the gradients have closed forms.
    70 000 terms of one sum in fp32, 16 at a time: another n / 16 * 2^-24 of the sum of sizes."""
    n, c = 70000, 0.125
    gen = torch.Generator().manual_seed(33)
    q, k, v, do = (torch.randn(n, 1, D, generator=gen) for _ in range(4))
    (q if zero == "q" else k).zero_()
    q, k, v, do = (t.half() for t in (q, k, v, do * 0.1 + 1))
    o, dq, dk, dv = (t[:, 0].double() for t in _run(q, k, v, do, [n], c))
    Q, K, V, dO = (t[:, 0].double() for t in (q, k, v, do))
    e, long = 2.0 ** -22 * (6 + float(np.log(n))), n / 16 * 2.0 ** -24
    want = dO.mean(0)
    assert torch.all((dv - want).abs() <= (U + e + long) * dO.abs().mean(0) + U * want.abs())
    delta = dO @ V.mean(0)
    if zero == "q":
        want, size = c / n * (dO @ (V.t() @ K) - delta[:, None] * K.sum(0)), c / n * (dO.abs() @ (V.abs().t() @ K.abs()))
        got = dq
        assert not dk.any()
    else:
        want, size = c / n * (V @ (dO.t() @ Q) - delta @ Q), c / n * (V.abs() @ (dO.abs().t() @ Q.abs()))
        got = dk
        assert not dq.any()
    # sum over the keys of |dS x| is twice `size` at most (delta is the mean of what dP is); the rounding of o reaches delta
    bound = (U + e + long + 2.0 ** -17) * 2 * size + c / n * U * (dO * o).abs().sum(1).max() * (K if zero == "q" else Q).abs().sum(0)
    assert torch.all((got - want).abs() <= bound + U * want.abs() + OUT)


@pytest.mark.parametrize("n", [20, 60, 200, 600, 3000])
def test_a_huge_value_that_nobody_looks_at(n):
    """The first key has v = 30 000 and probabilities of about e^-34: it decides nothing, and must not cost the others' dS their bits.  dS and result are
    rounded once each, independently and to u: for terms of random signs an error of sqrt(2 / 3) u of the gradients' norm, with 2 u more than twice that."""
    q, k, v, do = _inputs([n], 1, 34, 0.5, 0.5, 1.0)
    q[:, :, 0], k[:, :, 0] = 8.0, 0.0
    k[0, :, 0], v[0] = -34.0, 30000.0
    _, dq, dk, dv = (t[:, 0].double() for t in _run(q, k, v, do, [n], 0.125))
    Q, K, V, dO = (t[:, 0].double() for t in (q, k, v, do))
    P = torch.softmax(0.125 * (Q @ K.t()), -1)
    dP = dO @ V.t()
    dS = P * (dP - (P * dP).sum(-1, keepdim=True))
    for got, want in ((dq, 0.125 * (dS @ K)), (dk[1:], 0.125 * (dS.t() @ Q)[1:]), (dv[1:], (P.t() @ dO)[1:])):
        assert (got - want).norm() <= 2 * U * want.norm() + OUT * want.numel() ** 0.5, float((got - want).norm() / want.norm())


@pytest.mark.parametrize("what", ["do", "v", "both"])
def test_second_attempts_have_the_same_bits_in_every_launch(what):
    """Rows far larger than those that the size is taken from: in a launch of work-groups of 64 rows and among many of 128."""
    n, many = 241, 70
    q, k, v, do = _inputs([n], 3, 35, 2.0, 2.0 ** -2, 1.0)
    rare = (torch.arange(n) % 80 == 0)[:, None, None]
    if what != "v":
        do = (do.float() * torch.where(rare, 2.0 ** -11, 2.0 ** 9)).half()
    if what != "do":
        v = (v.float() * torch.where(rare, 2.0 ** -14, 2.0 ** 3)).half()
    o, *few = _run(q, k, v, do, [n], 0.125)
    _check(q, k, v, do, [n], 0.125, [o, *few])
    lot = [t.repeat(many, 1, 1).to(DEV) for t in (q, k, v, do, o)]
    # the statistics of the first launch, whose own last place may differ from launch to launch
    one_o, one_lse = torch.empty_like(q, device=DEV), torch.empty(n, 3, device=DEV)
    cu = torch.tensor([0, n], dtype=torch.int32, device=DEV)
    binding.ragged_attn_lse(*(t.to(DEV) for t in (q, k, v)), one_o, one_lse, cu, n, 0.125)
    assert torch.equal(one_o.cpu(), o)
    grads = [torch.zeros_like(lot[0]) for _ in range(3)]
    ends = torch.arange(0, n * many + 1, n, dtype=torch.int32, device=DEV)
    binding.ragged_attn_backward(*lot[:3], lot[4], lot[3], one_lse.repeat(many, 1), *grads, ends, n, 0.125)
    for a, b in zip(few, grads):
        assert torch.equal(a.repeat(many, 1, 1), b.cpu())
