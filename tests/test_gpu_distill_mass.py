"""Teachers and students on the GPU whose probability is nearly all, or nearly none
of it, at the named places: loss and gradient against the formulas in 64 bits, with
the sums over named and other places taken by their logarithms.

Tolerances: as in test_gpu_logits, from the formats.  x = (z - m) / tau is off by
|x| U, its exponential by (|x| + 4) U relatively, a sum of them by 8 U more; the
logarithm of a sum over places with the largest value a is off by the sum's relative
error and by U of (a - m) / tau; a teacher's probability by (|lt| + 4) U relatively."""
import math

import pytest
import torch

from paper_2504_11651_amd import ops

from conftest import gpu_available
from test_gpu_logits import INF, U, check_grad, close, place

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs an MI355X")]

DTYPES = [torch.float32, torch.bfloat16, torch.float16]


def mean_abs(x, top):
    """sum |x| exp x / sum exp x with x relative to `top`, and 0 for no places."""
    d = torch.where(x > -INF, x - top, -INF)
    e = d.exp()
    return (torch.where(e > 0, e * d.abs(), 0.0).sum(1) / e.sum(1).clamp(min=1e-300))[:, None]


def expected(t, index, logp, tail, tau, weight):
    """Loss and gradient with tolerances, for distinct places and unmasked maxima."""
    z = t.double().cpu()
    there = index >= 0
    lt = torch.where(there, logp.double(), -INF)
    at = torch.where(there, index, 0)
    x = (z - z.amax(1, keepdim=True)) / tau
    ln_s = torch.logsumexp(x, 1, keepdim=True)
    tol_s = (mean_abs(x, torch.zeros_like(ln_s)) + 16 + ln_s.abs()) * U
    lq = x - ln_s
    ln_mass = torch.logsumexp(lt, 1, keepdim=True)
    aim = lt if tail else lt - ln_mass           # ln of what the named places should have
    p = aim.exp()
    tol_p = (torch.where(there, lt.abs(), 0.0) + 16) * U
    if not tail:
        tol_p = tol_p + (p * tol_p).sum(1, keepdim=True)
    lqn = lq.gather(1, at)
    loss = torch.where(p > 0, p * (aim - lqn), 0.0).sum(1, keepdim=True)
    size = torch.where(p > 0, p * ((aim.abs() + lqn.abs()) * U + tol_s + x.gather(1, at).abs() * U +
                                   tol_p * ((aim - lqn).abs() + 1)), 0.0).sum(1, keepdim=True)
    named = torch.zeros((z.shape[0], z.shape[1] + 1), dtype=torch.bool)
    named = named.scatter_(1, torch.where(there, index, z.shape[1]), True)[:, :-1]
    q = lq.exp()
    grad, tol = q.clone(), q * (x.abs() * U + tol_s + 16 * U)
    if tail:
        others = torch.where(named, -INF, x)
        most = others.amax(1, keepdim=True)
        rest = (1 - p.sum(1, keepdim=True)).clamp(min=0)
        rest = torch.where((most == -INF) & (rest <= 2.0 ** -18), 0.0, rest)
        off_rest = (p * tol_p).sum(1, keepdim=True)
        ln_q = torch.logsumexp(others, 1, keepdim=True) - ln_s
        some = (rest > 0) & (most > -INF)
        some_lnq = torch.where(some, ln_q, 0.0)
        top = torch.where(most > -INF, most, 0.0)
        tol_q = (mean_abs(others, top) + 16 + top.abs()) * U + tol_s
        ln_r = torch.where(rest > 0, rest, 1.0).log()
        loss = loss + torch.where(rest > 0, rest * (ln_r - ln_q), 0.0)
        size = size + torch.where(some, rest * (tol_q + (ln_r.abs() + some_lnq.abs()) * U) +
                                  off_rest * (ln_r.abs() + some_lnq.abs() + 2), 0.0)
        share = torch.where(named | (others == -INF) | ~some, 0.0, (others - ln_s - some_lnq).exp())
        grad = grad - rest * share
        tol = tol + share * (rest * ((others - top).abs().clamp(max=1e9) * U + tol_q + 16 * U) + off_rest)
    target = torch.zeros_like(z).scatter_add_(1, at, torch.where(there, p, 0.0))
    grad = torch.where(named, q - target, grad)
    tol = tol + torch.zeros_like(z).scatter_add_(1, at, torch.where(there, p * tol_p, 0.0))
    w = (weight.double() / tau)[:, None]
    return loss[:, 0], size[:, 0] + 1e-30, grad * w, tol * w.abs() + (grad * w).abs() * 4 * U


def check(t, index, logp, tail, tau=1.0, weight=None):
    weight = torch.ones(t.shape[0]) if weight is None else weight
    loss, tol, grad, tol_grad = expected(t, index, logp, tail, tau, weight)
    i, lp, w = index.cuda(), logp.cuda(), weight.cuda()
    got = ops.distill(t, i, lp, tail=tail, temperature=tau, weight=w)
    close(got.loss, loss, tol, ("loss", tail))
    check_grad(got.grad, grad, tol_grad, t.dtype, ("grad", tail))
    later = ops.distill_backward(t, i, lp, got.stats, w, tail=tail, temperature=tau)
    check_grad(later, grad, tol_grad, t.dtype, ("grad later", tail))
    return got


def student(rows, vocab, seed):
    return torch.randn((rows, vocab), generator=torch.Generator().manual_seed(seed)) * 1.6


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("level", [-1.0, -50.0, -88.0, -90.0, -95.0, -104.0, -200.0, -1000.0, -1e5])
def test_teachers_of_little_mass_without_the_tail(level, dtype):
    """What is scaled to sum to one may be as little as it likes."""
    for top in (1, 7, 128):
        z = student(3, 9001, 5)
        g = torch.Generator().manual_seed(top)
        index = torch.stack([torch.randperm(9001, generator=g)[:top] for _ in range(3)])
        logp = level - 4 * torch.rand((3, top), generator=g)
        logp[1] = level
        index[2, 1::2] = -1
        got = check(place(z, dtype), index, logp, False, 1.0, torch.tensor([1.0, -2.0, 0.5]))
        assert torch.isfinite(got.loss).all() and torch.isfinite(got.grad).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("ahead", [30.0, 60.0, 90.0, 110.0, 300.0, 2000.0])
def test_students_that_leave_the_others_next_to_nothing(ahead, dtype):
    """The places that are not named have less probability than 32 bits can say:
    all in one wave's values, in some, or everywhere behind one named place."""
    vocab = 20011
    for tau in (1.0, 0.5, 3.0):
        z = student(5, vocab, 8)
        index = torch.tensor([[3, 7000, 19000], [0, 1, 2], [8191, 8192, 16384], [5, 2050, 20010], [12, 13, 14]])
        top = z.amax(1, keepdim=True) + ahead
        z.scatter_(1, index.clamp(min=0), top + torch.tensor([[0.0, -1.0, -0.5]]))
        z[3, 6:2050] = -INF                      # waves in which all the others are masked
        z[3, 2051:20010] = -INF
        z[4, :] -= 1e3                           # and rows far from zero
        logp = torch.log(torch.tensor([[0.6, 0.2, 0.1]])).repeat(5, 1)
        check(place(z, dtype, 1), index, logp, True, tau, torch.linspace(0.5, 1.5, 5))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("live", [1, 2, 10, 19])
def test_a_grammar_leaves_fewer_places_than_the_teacher_may_name(live, dtype):
    """The teacher's alternatives of a masked row are all there is: what its 32-bit
    values leave of 1 is no probability, for the row itself or for a student's."""
    rows, vocab = 64, 9001
    g = torch.Generator().manual_seed(live)
    mask = torch.full((rows, vocab), -INF)
    for r in range(rows):
        mask[r, torch.randperm(vocab, generator=g)[:live]] = 0.0
    z = student(rows, vocab, 6) * 2
    for tau in (1.0, 0.7):
        t = place(z + mask, dtype)
        teacher = ops.logprobs(t, top=20, temperature=tau)
        same = ops.distill(t, teacher.top_index, teacher.top_logprob, temperature=tau,
                           weight=torch.ones(rows, device="cuda"))
        # p = q up to what 32 bits hold: ln p and ln q agree to about |x| U
        x = (z.amax(1) - z.amin(1)).max() / tau
        assert same.loss.abs().max() <= (x + 16) * 2 * U and same.grad.abs().max() <= (x + 16) * 2 * U / tau
        t = place(student(rows, vocab, 7) + mask, dtype)
        got = check(t, teacher.top_index.cpu(), teacher.top_logprob.cpu(), True, tau)
        assert torch.isfinite(got.loss).all()


@pytest.mark.parametrize("short", [2.0 ** -10, 2.0 ** -16])
def test_probability_that_meets_no_place_is_infinite(short):
    """More than rounding is missing from the named places: the formula's loss."""
    z = torch.full((2, 5000), -INF)
    z[:, 100:110] = 1.0
    index = torch.arange(100, 110).repeat(2, 1)
    logp = torch.full((2, 10), math.log((1 - short) / 10))
    got = ops.distill(place(z, torch.float32), index.cuda(), logp.cuda(), weight=torch.ones(2, device="cuda"))
    assert (got.loss == INF).all() and torch.isfinite(got.grad).all()
    assert (got.grad[:, :100] == 0).all() and (got.grad[:, 110:] == 0).all()
