"""Gradients of rows whose sums are whole numbers: every exponential is exactly 1, so
that S is the number of unmasked places, and only the last few operations round.

Tolerance: 1/S, the row's factor, 1/tau, their products and the last one are rounded
once each: 6 * 2^-24 of the value, and 2^-126 where values are that small."""
import pytest
import torch

from paper_2504_11651_amd import ops

from conftest import gpu_available
from test_gpu_logits import INF, place

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs an MI355X")]

SIZES = [1, 2, 3, 7, 100, 1000, 8193, 20011, 32001, 50001, 99991, 128256]


def rows_of_ones(vocab):
    """All values alike; every third one alone; one part's alone."""
    z = torch.full((3, vocab), 1.75)
    z[1, 1::3] = -INF
    z[1, 2::3] = -INF
    z[2, min(vocab, 5000):] = -INF
    return z, (z > -INF).sum(1).double()


def near(got, want, what):
    off = (got.double().cpu() - want).abs()
    assert (off <= 6 * 2.0 ** -24 * want.abs() + 2.0 ** -126).all(), (what, (off / want.abs()).nan_to_num().max())


@pytest.mark.parametrize("tau", [1.0, 0.7])
@pytest.mark.parametrize("vocab", SIZES)
def test_log_probabilities(vocab, tau):
    z, count = rows_of_ones(vocab)
    t, zero = place(z, torch.float32), torch.zeros(3, dtype=torch.int64, device="cuda")
    got = ops.logprobs(t, zero, temperature=tau)
    gl = torch.tensor([1.0, -0.375, 3.0])
    over = 1 / float(torch.tensor(tau))
    grad = ops.logprobs_backward(t, zero, got.stats, gl.cuda(), temperature=tau).double().cpu()
    p = torch.where(z > -INF, 1 / count[:, None], 0.0)
    near(grad[:, 1:], -over * gl.double()[:, None] * p[:, 1:], "others")
    # the token's own: a difference of the two
    want = over * gl.double() * (1 - p[:, 0])
    assert ((grad[:, 0] - want).abs() <= 6 * 2.0 ** -24 * over * gl.abs()).all()


@pytest.mark.parametrize("tau", [1.0, 2.0, 0.7])
@pytest.mark.parametrize("vocab", SIZES[3:])
def test_distillation(vocab, tau):
    z, count = rows_of_ones(vocab)
    t = place(z, torch.float32)
    index = torch.tensor([[0, 3, -1]]).repeat(3, 1).cuda()
    logp = torch.log(torch.tensor([[0.25, 0.25, 0.0]])).repeat(3, 1).cuda()
    w = torch.tensor([1.0, -0.375, 3.0])
    factor = (w.double() / float(torch.tensor(tau)))[:, None]
    p = torch.where(z > -INF, 1 / count[:, None], 0.0)
    others = torch.ones(vocab, dtype=torch.bool)
    others[[0, 3]] = False
    # the teacher's probabilities as the given 32-bit logarithms have them
    mass = float(logp[0, :2].double().exp().sum())
    for tail in (False, True):
        got = ops.distill(t, index, logp, tail=tail, temperature=tau, weight=w.cuda())
        left = 1.0 if not tail else 1 - (1 - mass) / ((count[:, None] - 2) / count[:, None])
        want = factor * p * left
        if tail:  # 1 - r/Q loses what the two have in common
            rate = 6 * 2.0 ** -24 * (factor * p).abs()
            assert ((got.grad.double().cpu() - want).abs() <= rate + 2.0 ** -126)[:, others].all()
        else:
            near(got.grad[:, others.cuda()], want[:, others], "others")
