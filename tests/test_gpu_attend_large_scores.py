"""Attention with scores so large that 32 bits hold them in steps of many: the largest
take the row, as in the definition."""
import pytest
import torch

from paper_2504_11651_amd import ops

from conftest import gpu_available
from kv_reference import BF16, F16, Case, half_step, near

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs an MI355X")]


def check(c, q, scale):
    """Scores are products of one value each, exact in 32 bits, with steps between keys that
    leave the exponential of all but the largest 0: a result is the mean of the largest's
    values (whole numbers) within half a step of p, which is the same for all of them, half a
    step of its own and those of the sums; lse is off by the roundings of scale log2 e, its
    product and that with ln 2."""
    c.q[:] = 0
    c.q[:, ::c.dim] = q
    for pages, kv in zip([c.prefix_table.long(), *c.pages], c.sets):
        i = torch.arange(kv[0].shape[0], device="cuda")
        kv[1][:] = torch.randint(-8, 9, kv[1].shape, generator=c.g, device="cuda").to(c.dtype)
        if i.numel():
            c.k[pages[i // c.page], :, i % c.page] = kv[0]
            c.v[pages[i // c.page], :, i % c.page] = kv[1]
    got = c.attend(scale=scale)
    at = 0
    for b, (n, own) in enumerate(zip(c.new, c.own)):
        k, v = (torch.cat((c.sets[0][i], c.sets[b + 1][i])).double() for i in (0, 1))
        score = k[..., 0] * float(c.q[0, 0])  # tokens, kv heads
        for r in range(n):
            end = c.prefix + own - n + r + 1
            top = score[:end].amax(0)
            best = score[:end] == top
            want = (v[:end] * best[..., None]).sum(0) / best.sum(0)[:, None]
            want = want.repeat_interleave(c.group, 0).flatten()
            near(got.out[at + r], want, want.abs() * (2 * half_step(c.dtype) + 2 ** -19) + 2 ** -19, f"row {at + r}")
            lse = (top * scale + best.sum(0).log()).repeat_interleave(c.group, 0)
            near(got.lse[at + r], lse, lse.abs() * 2 ** -21 + 2 ** -21, f"lse of row {at + r}")
        at += n


CASES = [([1, 3], [300, 700], 1000), ([2, 1], [90, 40], 0), ([40], [40], 0), ([20, 1], [500, 1], 2000)]


# the largest products: from 10^5 to 10^9.5 in fp16, to 10^35 in bf16; scale as it was found,
# and one whose log2 e multiple has other last bits
@pytest.mark.parametrize("dtype, q, size", [
    (F16, 100.0, 1001.0), (F16, 999.0, 4001.0), (F16, 60000.0, 2001.0), (F16, 60000.0, 60000.0), (F16, 47008.0, 60000.0),
    (F16, -60000.0, 60000.0), (BF16, 1e3, 1e4), (BF16, 3e4, 1e5), (BF16, -7e8, 1e10), (BF16, 3e15, 1e20)])
@pytest.mark.parametrize("new, own, prefix", CASES)
@pytest.mark.parametrize("scale", [1.0, 0.7])
def test_the_largest_score_takes_the_row(new, own, prefix, scale, dtype, q, size):
    """Keys on both sides of zero in steps of a percent of the largest; ties among them in
    several parts of a row."""
    for seed in range(4):
        c = Case(new, own, prefix=prefix, dtype=dtype, dim=128 if seed % 2 else 64, seed=seed)
        for kv in c.sets:
            steps = torch.randint(-100, 101, kv[0].shape[:2], generator=c.g, device="cuda")
            kv[0][:] = 0
            kv[0][..., 0] = (steps * (size / 128)).to(dtype)
        check(c, q, scale)


@pytest.mark.parametrize("dtype, q, size", [(F16, 60000.0, 60000.0), (F16, 47008.0, 60000.0), (BF16, -7e8, 1e10)])
@pytest.mark.parametrize("scale", [1.0, 0.7])
def test_scores_that_are_all_far_below_zero(scale, dtype, q, size):
    c = Case([1, 2, 40], [100, 500, 40], prefix=700, dtype=dtype, seed=5)
    for kv in c.sets:
        steps = torch.randint(1, 128, kv[0].shape[:2], generator=c.g, device="cuda")
        kv[0][:] = 0
        kv[0][..., 0] = (steps * (-size / 128 * (1 if q > 0 else -1))).to(dtype)
    check(c, q, scale)


@pytest.mark.parametrize("dtype, q, size", [(F16, 60000.0, 60000.0), (BF16, 3e15, 1e20)])
def test_large_scores_of_a_prompt(dtype, q, size):
    """One kernel, rows that see up to themselves: the bound rises along the way."""
    c = Case([300], [300], prefix=0, heads=64, kv_heads=8, dim=64, dtype=dtype, seed=6)
    for kv in c.sets:
        steps = torch.arange(kv[0].shape[0], device="cuda") % 97
        kv[0][:] = 0
        kv[0][..., 0] = (steps * (size / 128))[:, None].to(dtype)
    check(c, q, 1.0)
