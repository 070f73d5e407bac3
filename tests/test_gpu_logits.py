"""Log probabilities and distillation on the GPU against their definitions in
64 bits, at the sizes, masks and strides where rows of logits can go wrong.

Tolerances, from the formats alone.  With x = (z - m) / tau: x is off by up to
|x| 2^-22 (difference, factor, its rounding), its exponential by a relative
(|x| + 4) 2^-22, a sum of n of them by another 64 * 2^-24 (at most 64 additions
on a path), so ln S by E (|x| + 8) 2^-21, E the mean under p.  Results follow by
their derivatives; an output adds the rounding of its type."""
import math

import pytest
import torch

from paper_2504_11651_amd import codec, ops

from conftest import gpu_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs an MI355X")]

DTYPES = [torch.float32, torch.bfloat16, torch.float16]
U = 2.0 ** -21
ROUND = {torch.float32: 2.0 ** -23, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -10}
INF, NAN = math.inf, math.nan


def place(z, dtype, pad=0, offset=0):
    """The rows on the GPU with `pad` NaNs between them and `offset` in front."""
    rows, vocab = z.shape
    whole = torch.full((offset + rows * (vocab + pad),), NAN, dtype=dtype, device="cuda")
    t = whole[offset:].view(rows, vocab + pad)[:, :vocab]
    t.copy_(z)
    return t


def close(got, want, tol, what):
    # the value that the output's type has for it: beyond its range that is an infinity
    got, want, tol = got.double().cpu(), want.float().double(), tol.expand_as(want)
    same = (got == want) | (got.isnan() & want.isnan())
    off = torch.where(same, 0.0, (got - want).abs())
    bad = ~(off <= tol)
    assert not bad.any(), (what, int(bad.sum()), got[bad][:4], want[bad][:4], tol[bad][:4])


class Rows:
    """p, log p and the tolerances of one set of rows in 64 bits (CPU)."""

    def __init__(self, t, tau):
        z = t.double().cpu()
        self.z, self.tau = z, tau
        self.m = z.amax(1, keepdim=True)
        self.empty = (self.m == -INF)[:, 0]
        self.broken = (z.isnan() | (z == INF)).any(1)
        x = (z - torch.where(self.empty[:, None], 0.0, self.m)) / tau
        self.s = x.exp().sum(1, keepdim=True)
        self.ln_s = self.s.log()
        self.lp = x - self.ln_s
        self.lp[self.empty] = -INF
        self.p = torch.where(x > -INF, x.exp() / self.s, 0.0)
        ax = torch.where(x > -INF, x.abs(), 0.0)
        self.mean_x = (self.p * ax).sum(1)
        self.mean_xx = (self.p * ax * ax).sum(1)
        self.tol_ln = (self.mean_x + 8) * U + self.ln_s[:, 0].abs() * U
        self.tol_ln[self.empty | self.broken] = 0.0
        self.ax = ax
        self.entropy = -(self.p * torch.where(self.p > 0, self.lp, 0.0)).sum(1)
        self.tol_entropy = (self.mean_xx + 8 * self.mean_x + 8) * U + self.tol_ln
        self.tol_entropy[self.empty | self.broken] = 0.0
        self.entropy[self.empty] = 0.0
        self.entropy[self.broken] = NAN

    def tol_lp(self):
        lp = torch.where(self.lp > -INF, self.lp.abs(), 0.0)
        t = self.tol_ln[:, None] + (self.ax + lp) * U
        return torch.where(t.isnan(), 0.0, t)


def check_logprobs(t, tokens, top, tau, **more):
    r = Rows(t, tau)
    got = ops.logprobs(t, tokens.cuda(), top=top, temperature=tau, **more)
    torch.cuda.synchronize()
    rows, vocab = t.shape
    at = tokens.clamp(0, vocab - 1)[:, None]
    zt = r.z.gather(1, at)
    there = (tokens >= 0) & (tokens < vocab) & ~r.broken
    want = r.lp.gather(1, at)[:, 0]
    want = torch.where(tokens < 0, 0.0, torch.where(tokens < vocab, want, NAN))
    want = torch.where(r.broken, NAN, want)
    close(got.logprob, want, r.tol_lp().gather(1, at)[:, 0], "logprob")
    j = torch.arange(vocab)
    rank = ((r.z > zt) | ((r.z == zt) & (j < at))).sum(1)
    assert torch.equal(got.rank.cpu(), torch.where(there, rank, -1))
    close(got.entropy, r.entropy, r.tol_entropy, "entropy")
    if top:
        z = torch.where(r.broken[:, None], 0.0, r.z)
        order = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :top]
        lp = r.lp.gather(1, order)
        index = torch.where(lp > -INF, order, -1)
        index[r.broken] = -1
        lp[r.broken] = NAN
        assert torch.equal(got.top_index.cpu(), index), (got.top_index.cpu() != index).nonzero()[:4]
        close(got.top_logprob, lp, r.tol_lp().gather(1, order), "top_logprob")
    return got, r


def draw(rows, vocab, seed, peaks=True):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn((rows, vocab), generator=g) * 1.6
    if peaks:
        z[:, ::max(1, vocab // 7)] += 6.0 * torch.rand((rows, z[:, ::max(1, vocab // 7)].shape[1]), generator=g)
    return z, torch.randint(vocab, (rows,), generator=g)


SIZES = [(1, 1), (3, 2), (2, 7), (1, 64), (5, 65), (2, 257), (3, 4099), (1, 8192), (2, 8193), (2, 8199),
         (4, 16384), (3, 20001), (2, 65536), (1, 128256)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows, vocab", SIZES)
def test_logprobs_sizes(rows, vocab, dtype):
    z, tokens = draw(rows, vocab, vocab)
    for pad, offset in ((0, 0), (1, 0), (3, 5), (8, 8)):
        check_logprobs(place(z, dtype, pad, offset), tokens, min(vocab, 20), 1.0)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("top", [0, 1, 2, 31, 63, 64, 65, 100, 127, 128])
def test_logprobs_alternatives(top, dtype):
    z, tokens = draw(3, 30011, top)
    check_logprobs(place(z, dtype), tokens, top, 0.7)
    z, tokens = draw(2, 129, top)
    check_logprobs(place(z, dtype), tokens, top, 2.0)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kind", ["constant", "rising", "falling", "steps", "two values", "zeros of both signs",
                                  "one lane's"])
def test_alternatives_among_equal_and_ordered_values(kind, dtype):
    vocab = 20011
    j = torch.arange(vocab, dtype=torch.float32)
    z = {"constant": torch.full_like(j, 1.5), "rising": j / vocab * 8, "falling": -j / vocab * 8,
         "steps": (j // 3000) % 5, "two values": (j % 2 == 0).float(),
         "zeros of both signs": torch.where(j % 3 == 0, -0.0, torch.where(j % 3 == 1, 0.0, -1.0)),
         "one lane's": torch.where(j % 2048 < 8, 5.0 + j / vocab, -1.0)}[kind]
    for top in (1, 20, 128):
        check_logprobs(place(z[None].repeat(2, 1), dtype), torch.tensor([vocab // 2, 0]), top, 1.0)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("top", [1, 20, 64, 128])
def test_alternatives_that_crowd_in_few_lanes(top, dtype):
    """Sorted rows, and rows in which a run of places holds all that is not masked,
    by -inf or by the lowest finite value."""
    z = torch.randn((6, 24600), generator=torch.Generator().manual_seed(top)) * 2
    z[0] = z[0].sort(descending=True).values
    z[1] = z[1].sort().values
    z[2, :9000] = torch.finfo(dtype).min
    z[2, 9300:] = torch.finfo(dtype).min
    z[3, :9000] = -INF
    z[3, 9300:] = -INF
    z[4, 300:] = torch.finfo(dtype).min
    z[5] = torch.where(torch.arange(24600) % 8200 < 300, 4.0, z[5].clamp(max=3.0))
    tokens = torch.tensor([0, 24599, 9100, 9100, 20000, 8300])
    check_logprobs(place(z, dtype), tokens, top, 1.0)
    check_logprobs(place(z, dtype, 3), tokens, top, 0.8)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("best", [-0.0, 0.0, -1.0, -2.0 ** -14])
def test_few_alternatives_above_negative_values(best, dtype):
    """The bound of the alternatives is 0 or negative, in either half of a word."""
    vocab = 9001
    for odd in (0, 1):
        z = torch.full((2, vocab), -3.5)
        z[:, 1::2] = -4.25
        places = torch.arange(7) * 1200 + 2 * torch.arange(7) + odd
        z[0, places] = best
        z[1, places[:3]] = best
        z[1, places[3:]] = 0.0 if best == 0 else best
        check_logprobs(place(z, dtype), torch.tensor([int(places[3]), 5]), 7, 1.0)
        check_logprobs(place(z, dtype, 1), torch.tensor([int(places[3]), 5]), 3, 0.5)


@pytest.mark.parametrize("dtype", DTYPES)
def test_masked_rows(dtype):
    vocab, top = 18001, 40
    z, _ = draw(9, vocab, 5)
    lowest = torch.finfo(dtype).min
    z[0] = -INF                                  # nothing is left
    z[1] = -INF
    z[1, 17000] = 2.0                            # one is left
    z[2, :17990] = -INF                          # fewer than `top`, all in one place
    z[3] = lowest                                # the lowest finite value is a value
    z[4, 100:] = lowest
    z[5, 9000] = NAN
    z[6, 3] = INF
    z[7, ::2] = -INF
    z[8, :] = -INF
    z[8, ::450] = lowest                         # masked values below the lowest one
    tokens = torch.tensor([5, 17000, 17995, 7, 50, 1, 3, 8, 450])
    for tau in (1.0, 0.25, 3.0):
        got, _ = check_logprobs(place(z, dtype, 1), tokens, top, tau)
        assert got.entropy[0] == 0 and got.logprob[0] == -INF and (got.top_index[0] == -1).all()
        assert got.logprob[1] == 0 and got.top_index[1, 0] == 17000 and (got.top_index[1, 1:] == -1).all()
        assert (got.top_index[2] >= 0).sum() == 11
    # a masked token that is asked for
    check_logprobs(place(z, dtype), torch.tensor([-1, 16999, 3, vocab, 2 ** 40, -5, 0, 1, 1]), top, 1.0)


def test_values_far_apart_and_large():
    z = torch.tensor([[3e38, -3e38, 0.0, 1.0], [80.0, -80.0, 79.0, 0.0], [-3e38, -3e38, -3.1e38, -3e38]])
    for tau in (1.0, 0.5, 2.0):
        check_logprobs(place(z, torch.float32), torch.tensor([0, 2, 3]), 4, tau)


def test_without_tokens_and_with_given_outputs():
    z, tokens = draw(6, 9001, 8)
    t = place(z, torch.float32)
    full = ops.logprobs(t, tokens.cuda(), top=5)
    none = ops.logprobs(t, top=5)
    assert none.logprob is None and none.rank is None
    assert torch.equal(none.entropy, full.entropy) and torch.equal(none.top_index, full.top_index)
    out = tuple(torch.full_like(f, 7) for f in full)
    ws = torch.empty(max(16, ops.logprobs_workspace_bytes(torch.float32, 6, 9001, 5)), dtype=torch.uint8, device="cuda")
    got = ops.logprobs(t, tokens.cuda(), top=5, out=out, workspace=ws)
    for a, b, c in zip(full, got, out):
        assert torch.equal(a, b) and b.data_ptr() == c.data_ptr()
    part = ops.logprobs(t, tokens.cuda(), out=(out[0], None, None, None, None, None))
    assert torch.equal(part.logprob, full.logprob)
    assert ops.logprobs(t[:0], tokens[:0].cuda(), top=5).top_index.shape == (0, 5)


# ----------------------------------------------------------------- gradients
def grad_logprobs(r, tokens, gl, ge):
    """The formula's gradient and its tolerance."""
    vocab = r.z.shape[1]
    gl, ge = gl.double()[:, None], ge.double()[:, None]
    asked = (tokens >= 0)[:, None]
    hit = (torch.arange(vocab) == tokens[:, None]).double()
    lp = torch.where(r.p > 0, r.lp, 0.0)
    h = r.entropy[:, None]
    gl = torch.where(asked, gl, 0.0)
    want = (gl * (hit - r.p) - ge * r.p * (lp + h)) / r.tau
    rel = (r.ax + r.ln_s.abs() + 8) * U + r.tol_ln[:, None]
    by_entropy = r.p * ((lp + h).abs() * rel + rel + r.tol_entropy[:, None])
    tol = (gl.abs() * (r.p * rel + hit * U) + ge.abs() * by_entropy) / r.tau
    want[r.empty] = 0.0
    tol[r.empty] = 0.0
    want[r.broken | (tokens >= vocab)] = NAN
    return want, tol


def tiny(dtype):
    """The spacing next to zero."""
    return torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps


def check_grad(got, want, tol, dtype, what):
    close(got, want, torch.nan_to_num(tol) + torch.nan_to_num(want.abs()) * ROUND[dtype] + tiny(dtype) + 1e-37, what)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows, vocab", SIZES)
def test_logprobs_gradient(rows, vocab, dtype):
    z, tokens = draw(rows, vocab, vocab + 1)
    g = torch.Generator().manual_seed(vocab)
    gl, ge = torch.randn(rows, generator=g), torch.randn(rows, generator=g)
    for tau, pad, offset in ((1.0, 0, 0), (0.7, 3, 5)):
        t = place(z, dtype, pad, offset)
        r = Rows(t, tau)
        stats = ops.logprobs(t, tokens.cuda(), temperature=tau).stats
        zero = torch.zeros(rows)
        for a, b in ((gl, ge), (gl, None), (None, ge)):
            want, tol = grad_logprobs(r, tokens, zero if a is None else a, zero if b is None else b)
            got = ops.logprobs_backward(t, tokens.cuda(), stats, None if a is None else a.cuda(),
                                        None if b is None else b.cuda(), temperature=tau)
            check_grad(got, want, tol, dtype, (tau, a is None, b is None))
        # in place, with the padding left alone
        want = ops.logprobs_backward(t, tokens.cuda(), stats, gl.cuda(), ge.cuda(), temperature=tau).clone()
        into = place(z, dtype, pad, offset)
        ops.logprobs_backward(into, tokens.cuda(), stats, gl.cuda(), ge.cuda(), temperature=tau, out=into)
        assert torch.equal(into, want)
        if pad and rows > 1:
            assert into.as_strided((rows - 1, pad), (vocab + pad, 1), into.storage_offset() + vocab).isnan().all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_logprobs_gradient_of_masked_and_broken_rows(dtype):
    vocab = 9001
    z, _ = draw(8, vocab, 6)
    z[0] = -INF
    z[1] = -INF
    z[1, 4] = 1.0
    z[2, :8000] = -INF
    z[3] = torch.finfo(dtype).min
    z[4, 7] = NAN
    z[5, 8] = INF
    tokens = torch.tensor([3, 4, 8500, 0, 1, 2, -3, vocab + 4])
    t = place(z, dtype)
    r = Rows(t, 1.0)
    gl, ge = torch.linspace(-1, 1, 8), torch.linspace(0.5, -0.5, 8)
    stats = ops.logprobs(t, tokens.cuda()).stats
    want, tol = grad_logprobs(r, tokens, gl, ge)
    got = ops.logprobs_backward(t, tokens.cuda(), stats, gl.cuda(), ge.cuda())
    check_grad(got, want, tol, dtype, "masked")
    assert (got[0] == 0).all() and got[4].isnan().all() and got[7].isnan().all()


def test_logprobs_gradient_against_differences():
    z, tokens = draw(3, 5001, 9)
    t = place(z, torch.float32)
    gl, ge = torch.tensor([1.0, -0.5, 2.0]), torch.tensor([0.3, 1.0, -0.7])
    tau = 1.3
    stats = ops.logprobs(t, tokens.cuda(), temperature=tau).stats
    grad = ops.logprobs_backward(t, tokens.cuda(), stats, gl.cuda(), ge.cuda(), temperature=tau).double().cpu()
    step = torch.randn(z.shape, generator=torch.Generator().manual_seed(1)).double()

    def value(h):
        r = Rows(t.double().cpu() + h * step, tau)
        return (r.lp.gather(1, tokens[:, None])[:, 0] * gl + r.entropy * ge).sum()

    h = 1e-4
    slope = (value(h) - value(-h)) / (2 * h)
    # the difference's own error is of order h^2; each gradient entry is good to 32 bits
    tol = 1e-6 * (1 + slope.abs()) + (grad_logprobs(Rows(t, tau), tokens, gl, ge)[1] * step.abs()).sum() + \
        (grad * step).abs().sum() * 2.0 ** -23
    assert abs(float((grad * step).sum() - slope)) <= float(tol)


# --------------------------------------------------------------- distillation
def teacher(rows, vocab, top, seed, mass=0.9, holes=True):
    g = torch.Generator().manual_seed(seed)
    index = torch.stack([torch.randperm(vocab, generator=g)[:top] for _ in range(rows)])
    raw = torch.randn((rows, top), generator=g).double() * 2
    logp = (raw - raw.exp().sum(1, keepdim=True).log() + math.log(mass)).float()
    if holes and top > 1:
        index[:, 1::3] = -1
    return index, logp


def distill_want(r, index, logp, tail, weight):
    """Loss, gradient and their tolerances in 64 bits."""
    rows, vocab = r.z.shape
    there = index >= 0
    bad = (there & ((index >= vocab) | ~(logp < INF))).any(1)
    lt = torch.where(there, logp.double(), -INF)
    p = torch.nan_to_num(lt.exp(), nan=0.0)
    at = torch.where(there, index, 0).clamp(max=vocab - 1)
    mass = p.sum(1)
    dp = (p * (torch.where(p > 0, lt.abs(), 0.0) + 8) * U).sum(1)
    aim = p if tail else p / torch.where(mass > 0, mass, 1.0)[:, None]
    named = torch.zeros((rows, vocab + 1), dtype=torch.bool).scatter_(1, torch.where(there, at, vocab), True)[:, :-1]
    lq = r.lp.gather(1, at)
    la = torch.where(aim > 0, aim, 1.0).log()
    terms = torch.where(aim > 0, aim * (la - lq), 0.0)
    loss = terms.sum(1)
    size = torch.where(aim > 0, aim * (la.abs() + lt.abs() + torch.where(lq > -INF, lq.abs(), 0.0) + 16), 0.0).sum(1)
    tol = size * U + aim.sum(1) * r.tol_ln
    tol = tol + torch.where(aim > 0, aim * r.ax.gather(1, at), 0.0).sum(1) * U
    other = torch.ones(rows, dtype=torch.double)
    tol_other = torch.zeros(rows, dtype=torch.double)
    if tail:
        rest = (1 - mass).clamp(min=0)
        q = torch.where(named, 0.0, r.p).sum(1)
        some = rest > 0
        safe = torch.where(some, rest, 1.0)
        loss = loss + torch.where(some, rest * (safe.log() - q.log()), 0.0)
        lnq = torch.where(q > 0, q, 1.0).log()
        tol = tol + rest * ((lnq.abs() + safe.log().abs() + 16) * U + 2 * r.tol_ln + r.mean_x * U) + \
            dp * (safe.log().abs() + lnq.abs() + 2)
        other = torch.where(some, torch.where(q > 0, 1 - rest / q, 0.0), 1.0)
        tol_other = torch.where(some & (q > 0), (rest * (2 * r.tol_ln + 32 * U) + dp) / torch.where(q > 0, q, 1.0), 0.0)
    target = torch.zeros((rows, vocab), dtype=torch.double).scatter_add_(1, at, torch.where(there, aim, 0.0))
    grad = torch.where(named, r.p, r.p * other[:, None]) - target
    rel = (r.ax + r.ln_s.abs() + 8) * U + r.tol_ln[:, None]
    lmax = torch.where(there & (lt > -INF), lt.abs(), 0.0).amax(1)
    dm = dp / torch.where(mass > 0, mass, 1.0)
    tol_grad = r.p * rel * torch.where(named, 1.0, other.abs()[:, None]) + r.p * tol_other[:, None] + \
        target * ((lmax + 16) * U + dm)[:, None]
    grad, tol_grad = grad * (weight.double() / r.tau)[:, None], tol_grad * (weight.abs().double() / r.tau)[:, None]
    tol_grad = tol_grad + grad.abs() * 4 * U
    grad[r.empty] = 0.0
    for x in (loss, grad):
        x[r.broken] = NAN
        x[~there.any(1) | ((mass == 0) & (not tail))] = 0.0
        x[bad] = NAN
    ok = ~(r.broken | bad)
    return loss, torch.where(ok, torch.nan_to_num(tol), 0.0) + 1e-30, grad, tol_grad


def check_distill(t, index, logp, tail, tau, weight):
    r = Rows(t, tau)
    loss, tol, grad, tol_grad = distill_want(r, index, logp, tail, weight)
    i, lp, w = index.cuda(), logp.cuda(), weight.cuda()
    got = ops.distill(t, i, lp, tail=tail, temperature=tau, weight=w)
    close(got.loss, loss, tol, ("loss", tail))
    check_grad(got.grad, grad, tol_grad, t.dtype, ("grad", tail))
    alone = ops.distill(t, i, lp, tail=tail, temperature=tau)
    assert alone.grad is None
    close(alone.loss, loss, tol, ("loss alone", tail))
    later = ops.distill_backward(t, i, lp, alone.stats, w, tail=tail, temperature=tau)
    check_grad(later, grad, tol_grad, t.dtype, ("grad later", tail))
    return got


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows, vocab", SIZES)
def test_distill_sizes(rows, vocab, dtype):
    z, _ = draw(rows, vocab, vocab + 2)
    index, logp = teacher(rows, vocab, min(vocab, 20), vocab)
    weight = torch.linspace(0.5, 2.0, rows)
    for pad, offset, tail, tau in ((0, 0, True, 1.0), (1, 0, False, 2.0), (3, 5, True, 0.7), (8, 8, False, 1.0)):
        check_distill(place(z, dtype, pad, offset), index, logp, tail, tau, weight)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("top", [1, 2, 63, 64, 65, 128])
def test_distill_alternatives(top, dtype):
    for vocab in (128, 16500):
        z, _ = draw(3, vocab, top)
        for holes in (False, True):
            index, logp = teacher(3, vocab, top, top, holes=holes)
            for tail in (True, False):
                check_distill(place(z, dtype), index, logp, tail, 1.0, torch.tensor([1.0, -2.0, 0.0]))


@pytest.mark.parametrize("tail", [True, False])
@pytest.mark.parametrize("dtype", DTYPES)
def test_distill_rows_that_hold_little(dtype, tail):
    vocab, top = 12001, 6
    z, _ = draw(12, vocab, 3)
    index, logp = teacher(12, vocab, top, 4, holes=False)
    index[0] = -1                          # no teacher
    logp[1] = -INF                         # a teacher without probability
    index[2, 1:] = -1
    index[3, 2] = vocab                    # out of range
    logp[4, 3] = NAN
    logp[5, 3] = INF
    z[6] = -INF                            # the student's row is masked
    z[7, index[7, 0]] = -INF               # a named place is masked
    z[8, 5] = NAN
    z[9] = -INF
    z[9, index[9]] = torch.randn(top)      # nothing but the named places is left
    index[10, 1] = index[10, 0]            # a place named twice
    index[10, 5] = index[10, 0]
    logp[11] = math.log(1 / top)           # all the probability
    logp[11, 2] = -INF
    index[11, 3] = -7
    logp[11, 3] = NAN                      # ignored with its place
    got = check_distill(place(z, dtype, 1), index, logp, tail, 1.0, torch.full((12,), 1.5))
    assert got.loss[0] == 0 and (got.grad[0] == 0).all() and got.loss[6] == INF and (got.grad[6] == 0).all()
    for row in (3, 4, 5, 8):
        assert got.loss[row].isnan() and got.grad[row].isnan().all()
    z[0] = NAN                             # a row that does not count may hold anything
    got = check_distill(place(z[:1], dtype), index[:1], logp[:1], tail, 1.0, torch.ones(1))
    assert got.loss[0] == 0 and (got.grad == 0).all()


@pytest.mark.parametrize("tail", [True, False])
def test_distill_gradient_against_differences(tail):
    vocab, top, tau = 4003, 12, 1.4
    z, _ = draw(3, vocab, 12)
    index, logp = teacher(3, vocab, top, 13, mass=0.8)
    t = place(z, torch.float32)
    w = torch.tensor([1.0, 0.25, 3.0])
    got = ops.distill(t, index.cuda(), logp.cuda(), tail=tail, temperature=tau, weight=w.cuda())
    step = torch.randn(z.shape, generator=torch.Generator().manual_seed(2)).double()

    def value(h):
        return (distill_want(Rows(t.double().cpu() + h * step, tau), index, logp, tail, w)[0] * w).sum()

    h = 1e-4
    slope = (value(h) - value(-h)) / (2 * h)
    grad = got.grad.double().cpu()
    tol = 1e-6 * (1 + slope.abs()) + (distill_want(Rows(t, tau), index, logp, tail, w)[3] * step.abs()).sum() + \
        (grad * step).abs().sum() * 2.0 ** -23
    assert abs(float((grad * step).sum() - slope)) <= float(tol)


@pytest.mark.parametrize("dtype", DTYPES)
def test_distill_in_place(dtype):
    z, _ = draw(4, 33333, 20)
    index, logp = teacher(4, 33333, 30, 21)
    index[2, 2:8] = index[2, 0]
    for pad, offset in ((0, 0), (3, 1)):
        t = place(z, dtype, pad, offset)
        want = ops.distill(t, index.cuda(), logp.cuda(), weight=torch.ones(4, device="cuda"))
        got = ops.distill(t, index.cuda(), logp.cuda(), grad=t)
        assert got.grad.data_ptr() == t.data_ptr()
        assert torch.equal(t, want.grad) and torch.equal(got.loss, want.loss)
        again = place(z, dtype, pad, offset)
        ops.distill_backward(again, index.cuda(), logp.cuda(), want.stats, out=again)
        r = Rows(place(z, dtype), 1.0)
        _, _, grad, tol = distill_want(r, index, logp, True, torch.ones(4))
        check_grad(again, grad, tol, dtype, "in place")
        if pad:
            assert again.as_strided((3, pad), (33333 + pad, 1), offset + 33333).isnan().all()


# ---------------------------------------------------------- use in a program
def test_rows_past_32_bit_offsets():
    """Three rows 2^31 + 40 elements apart: the last starts past 2^32."""
    vocab, stride = 10007, (1 << 31) + 40
    z, tokens = draw(3, vocab, 30)
    index, logp = teacher(3, vocab, 9, 31)
    whole = torch.empty(2 * stride + vocab, dtype=torch.bfloat16, device="cuda")
    t = whole.as_strided((3, vocab), (stride, 1))
    t.copy_(z)
    got, r = check_logprobs(t, tokens, 12, 1.0)
    gl = torch.tensor([1.0, 2.0, -1.0])
    w = torch.ones(3)
    loss, tol, grad, tol_grad = distill_want(r, index, logp, True, w)
    d = ops.distill(t, index.cuda(), logp.cuda(), weight=w.cuda())
    close(d.loss, loss, tol, "loss")
    check_grad(d.grad, grad, tol_grad, torch.bfloat16, "grad")
    want, tol = grad_logprobs(r, tokens, gl, torch.zeros(3))
    ops.logprobs_backward(t, tokens.cuda(), got.stats, gl.cuda(), out=t)
    check_grad(t, want, tol, torch.bfloat16, "in place")


def test_more_rows_than_a_grid_dimension():
    rows, vocab = 70001, 33
    z, tokens = draw(rows, vocab, 32, peaks=False)
    got, r = check_logprobs(place(z, torch.float32), tokens, 3, 1.0)
    gl, ge = torch.ones(rows), torch.full((rows,), 0.5)
    want, tol = grad_logprobs(r, tokens, gl, ge)
    check_grad(ops.logprobs_backward(place(z, torch.float32), tokens.cuda(), got.stats, gl.cuda(), ge.cuda()),
               want, tol, torch.float32, "grad")
    index = torch.stack([tokens, (tokens + 1) % vocab], 1)
    check_distill(place(z, torch.float32), index, torch.full((rows, 2), -1.2), True, 1.0, gl)


def everything(t, tokens, index, logp, gl, ge, **more):
    a = ops.logprobs(t, tokens, top=17, **more)
    b = ops.logprobs_backward(t, tokens, a.stats, gl, ge, **more)
    c = ops.distill(t, index, logp, weight=gl, **more)
    d = ops.distill_backward(t, index, logp, c.stats, gl, tail=True, **more)
    return [*a, b, c.loss, c.stats, c.grad, d]


@pytest.mark.parametrize("rows, vocab", [(1, 50001), (37, 9999)])
def test_streams_graphs_and_repeats(rows, vocab):
    z, tokens = draw(rows, vocab, 40)
    index, logp = teacher(rows, vocab, 11, 41)
    z2, _ = draw(rows, vocab, 42)
    args = [tokens.cuda(), index.cuda(), logp.cuda(), torch.linspace(-1, 1, rows).cuda(), torch.ones(rows).cuda()]
    t, t2 = place(z, torch.bfloat16), place(z2, torch.bfloat16)
    want, want2 = everything(t, *args), everything(t2, *args)
    for a, b in zip(want, everything(t, *args)):
        assert torch.equal(a, b)  # the same inputs give the same bits
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        late = t2.clone()  # made on the stream that uses it
        got = everything(late, *args)
    side.synchronize()
    for a, b in zip(want2, got):
        assert torch.equal(a, b)
    got = everything(t, *args, stream=side)  # named, not current
    side.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    held = t.clone()
    with torch.cuda.stream(side):
        everything(held, *args)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        replayed = everything(held, *args)
    for k in range(4):
        held.copy_(t2 if k % 2 else t)
        for x in replayed:
            x.fill_(-7)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want2 if k % 2 else want, replayed):
            assert torch.equal(a, b), k
        everything(t, *args)


def test_what_is_refused():
    z, tokens = draw(3, 100, 50)
    t, tok = place(z, torch.float32), tokens.cuda()
    f = torch.ones(3, device="cuda")
    stats = ops.logprobs(t, tok).stats
    index, logp = (x.cuda() for x in teacher(3, 100, 4, 51))
    for call in (lambda: ops.logprobs(t.double(), tok), lambda: ops.logprobs(t[0], tok),
                 lambda: ops.logprobs(t.t(), tok), lambda: ops.logprobs(t, tok.int()),
                 lambda: ops.logprobs(t, tok[:2]), lambda: ops.logprobs(t, tokens),
                 lambda: ops.logprobs(t, tok, out=(f[:2], None, None, None, None, None)),
                 lambda: ops.logprobs_backward(t, tok, stats[:2], f),
                 lambda: ops.logprobs_backward(t, tok, stats, f, out=t.bfloat16()),
                 lambda: ops.distill(t, index, logp[:, :3]), lambda: ops.distill(t, index.int(), logp),
                 lambda: ops.distill(t, index, logp, weight=f[:2]),
                 lambda: ops.distill(t, index, logp, grad=t[:2]),
                 lambda: ops.distill_backward(t, index, logp, stats, f.double())):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: ops.logprobs(t, tok, top=101), lambda: ops.logprobs(t, tok, temperature=0.0),
                 lambda: ops.logprobs_backward(t, tok, stats),
                 lambda: ops.distill(t, index[:, :0].contiguous(), logp[:, :0].contiguous()),
                 lambda: ops.distill(t, index, logp, temperature=-1.0)):
        with pytest.raises(codec.DF11Error):
            call()
    if ops.logprobs_workspace_bytes(torch.float32, 3, 100, 4):
        with pytest.raises(codec.DF11Error):
            ops.logprobs(t, tok, top=4, workspace=torch.empty(1, dtype=torch.uint8, device="cuda"))
