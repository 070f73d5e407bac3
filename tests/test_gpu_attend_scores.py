"""Attention where scores lie far from each other or from zero: many tokens that one
outweighs, against the definition in 64 bits."""
import math

import pytest
import torch

from paper_2504_11651_amd import ops

from conftest import gpu_available
from kv_reference import BF16, F16, Case, half_step, near

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs an MI355X")]


def fill(c):
    """A case's sets, changed, to their pages."""
    for pages, kv in zip([c.prefix_table.long(), *c.pages], c.sets):
        i = torch.arange(kv[0].shape[0], device="cuda")
        if i.numel():
            c.k[pages[i // c.page], :, i % c.page] = kv[0]
            c.v[pages[i // c.page], :, i % c.page] = kv[1]


def one_outweighs(c, gap, place):
    """Scores of 0 and values of 1, but for the token at `place` of the prefix or of every
    sequence's own: a score of `gap` and a value of 0."""
    c.q[:] = 0
    c.q[:, ::c.dim] = 1  # a head's first value: a score is a key's first value
    for x, kv in enumerate(c.sets):
        kv[0][:], kv[1][:] = 0, 1
        if (x == 0) == bool(c.prefix) and kv[0].shape[0]:
            kv[0][place, :, 0] = gap
            kv[1][place] = 0
    fill(c)


def check_outweighed(c, gap, place, got):
    """n others give n e^-gap / (1 + n e^-gap).

    The score's multiple by log2 e and its exponential are off by 2^-22 of it and 2^-22
    more, a p by half a step of its type, the sums by n 2^-24 each, the result by half a
    step.  In fp16 the steps end at 2^-24, of a sum that is at least 2^7 there: each of n
    is off by 2^-25 at most, together by n 2^-32 of the sum; the result by 2^-25."""
    at = 0
    for n, own in zip(c.new, c.own):
        seen = c.prefix + torch.arange(own - n, own, device="cuda", dtype=torch.float64) + 1
        outweighed = (seen > place).double() if not c.prefix else torch.ones_like(seen)
        others = seen - outweighed
        rest = others * torch.where(outweighed == 1, math.exp(-gap), 1.0)
        want = rest / (outweighed + rest)
        u = half_step(c.dtype)
        tol = want * (2 * u + 2 * (gap + 1) * 2 ** -22 + 2 * seen * 2 ** -24)
        if c.dtype == F16:
            tol = tol + seen * 2 ** -32 + 2 ** -25
        shape = (n, c.heads * c.dim)
        near(got.out[at:at + n], want[:, None].expand(shape), tol[:, None].expand(shape), f"gap {gap}")
        lse = torch.where(outweighed == 1, gap, 0.0) + (outweighed + rest).log()
        near(got.lse[at:at + n], lse[:, None].expand(n, c.heads),
             ((gap + 1) * 2 ** -21 + seen * 2 ** -24)[:, None].expand(n, c.heads), f"lse, gap {gap}")
        at += n


GAPS = [10.0, 14.0, 15.0, 16.0, 17.0, 17.5, 18.0, 20.0]


@pytest.mark.parametrize("dtype, dim", [(F16, 64), (F16, 128), (BF16, 128)])
@pytest.mark.parametrize("place", [0, 1, 4097])
@pytest.mark.parametrize("gap", GAPS)
def test_many_tokens_that_one_outweighs(gap, place, dtype, dim):
    """In shares: the prefix' tokens, and own tokens without one."""
    for new, own, prefix in (([1, 2], [1, 40], 8192), ([1], [8193], 0)):
        c = Case(new, own, prefix=prefix, dim=dim, dtype=dtype, seed=1)
        assert ops.prefix_attention_workspace_bytes(c.tokens, c.heads, c.cache, c.batch) > 0
        one_outweighs(c, gap, place)
        check_outweighed(c, gap, place, c.attend(scale=1.0))


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("place", [0, 200])
@pytest.mark.parametrize("gap", GAPS)
def test_many_tokens_of_a_prompt_that_one_outweighs(gap, place, dtype):
    """In one kernel, with one bound over all that a row sees."""
    for own, prefix in ((8742, 0), (550, 8192)):
        c = Case([550], [own], prefix=prefix, heads=64, kv_heads=8, dim=64, dtype=dtype, seed=2)
        assert ops.prefix_attention_workspace_bytes(c.tokens, c.heads, c.cache, c.batch) == 0
        one_outweighs(c, gap, place)
        check_outweighed(c, gap, place, c.attend(scale=1.0))


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_the_longest_prefix_that_one_token_outweighs(dtype):
    """131,072 tokens 25 powers of two below the first: 0.4% of the sum."""
    c = Case([1], [1], prefix=131072, heads=4, kv_heads=1, dim=64, dtype=dtype, seed=3)
    gap = 17.328125 if dtype == F16 else 17.375
    one_outweighs(c, gap, 0)
    check_outweighed(c, gap, 0, c.attend(scale=1.0))
