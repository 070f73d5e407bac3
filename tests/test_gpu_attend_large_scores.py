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


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("prefix", [100, 1000, 5000])
@pytest.mark.parametrize("q, k", [(0.0, 0.0), (16.0, 44.0), (30.0, 180.0), (200.0, 240.0), (1000.0, 300.0),
                                  (1000.0, 720.0), (-1000.0, 720.0), (1000.0, 1600.0)])
def test_weights_of_near_scores_in_parts_of_a_row(q, k, prefix, dtype):
    """One token of the prefix and one of its own outweigh a row's others, by scores q k + d
    that lie within 3 of each other: their weights go by the difference, however large they
    are.  Scores and d are exact; each p is off by half a step and by 2^-15 at most where c s
    is below 2^10 (half a step of it), the result by half a step."""
    n = 17
    c = Case([1] * n, [1 + 5 * i for i in range(n)], prefix=prefix, dtype=dtype, seed=7)
    c.q[:] = 0
    q, k = (float(torch.tensor(x).to(dtype)) for x in (q, k))
    c.q[:, ::c.dim], c.q[:, 1::c.dim] = q, 1
    d = (torch.arange(n, device="cuda") - 8) * 0.375
    for i, kv in enumerate(c.sets):
        kv[0][:], kv[1][:] = 0, 0
        kv[0][..., 1] = -200  # the others
        kv[0][..., 0] = k
        at = kv[0].shape[0] // 2
        kv[0][at, :, 1] = 0 if not i else d[i - 1].to(dtype)
        if not i:
            kv[1][at] = 1
    for pages, kv in zip([c.prefix_table.long(), *c.pages], c.sets):
        i = torch.arange(kv[0].shape[0], device="cuda")
        c.k[pages[i // c.page], :, i % c.page] = kv[0]
        c.v[pages[i // c.page], :, i % c.page] = kv[1]
    score = q * k
    assert score == float(torch.tensor(score).float()) and float((torch.tensor(score) + 0.375).float()) == score + 0.375
    got = c.attend(scale=1.0)
    want = 1 / (1 + d.double().exp())
    tol = want * (3 * half_step(dtype) + 2 ** -14 + 2 ** -20)
    near(got.out, want[:, None].expand(got.out.shape), tol[:, None].expand(got.out.shape), "out")
    lse = score + (1 + d.double().exp()).log()
    near(got.lse, lse[:, None].expand(got.lse.shape), (lse.abs() * 2 ** -21 + 2 ** -21)[:, None].expand(got.lse.shape), "lse")
