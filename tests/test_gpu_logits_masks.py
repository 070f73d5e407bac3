"""Finite masks and far-off values on the GPU: rows whose masked places fill whole
waves and parts with a large negative number instead of -inf, rows of such a number
alone, rows with a large common offset, and very large temperatures.  Oracle and
tolerances are those of test_gpu_logits."""
import math

import pytest
import torch

from paper_2504_11651_amd import ops

from conftest import gpu_available
from test_gpu_logits import (INF, check_distill, check_grad, check_logprobs, grad_logprobs, place)

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs an MI355X")]

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
LOWEST = {d: torch.finfo(d).min for d in (F32, BF16, F16)}
# masks of a training or serving program; the last ones are the types' lowest values
MASKS = [(d, m) for d in (F32, BF16) for m in (-1e4, -1e9, -5e9, -1e10, -1e12, -1e20, -1e30, -1e37)]
MASKS += [(F16, -6e4)] + [(d, LOWEST[d]) for d in (F32, BF16, F16)]
TAUS = [0.5, 0.7, 1.0, 2.0, 5.0, 8.0, 10.0]


def masked_rows(mask, seed):
    """Live values in one place, in some, in every other one, behind the masks, none,
    and all with the mask's own neighbours; the token of each row."""
    vocab = 18001
    z = torch.randn((6, vocab), generator=torch.Generator().manual_seed(seed)) * 2
    live = torch.zeros(z.shape, dtype=torch.bool)
    live[0, [3, 9000, 9001]] = True
    live[1, 17500:17600] = True
    live[2, ::2] = True
    live[3, :8200] = True
    live[5, ::3000] = True
    return torch.where(live, z, torch.full_like(z, mask)), torch.tensor([9000, 17555, 5, 17000, 11, 6000])


@pytest.mark.parametrize("tau", TAUS)
@pytest.mark.parametrize("dtype, mask", MASKS)
def test_log_probabilities(dtype, mask, tau):
    z, tokens = masked_rows(mask, 3)
    for top in (0, 20):
        got, r = check_logprobs(place(z, dtype, 1), tokens, top, tau)
    assert torch.isfinite(got.entropy).all()
    gl, ge = torch.linspace(-1, 2, 6), torch.linspace(0.5, -0.5, 6)
    want, tol = grad_logprobs(r, tokens, gl, ge)
    t = place(z, dtype, 1)
    grad = ops.logprobs_backward(t, tokens.cuda(), got.stats, gl.cuda(), ge.cuda(), temperature=tau)
    check_grad(grad, want, tol, dtype, "grad")


@pytest.mark.parametrize("tail", [True, False])
@pytest.mark.parametrize("tau", TAUS)
@pytest.mark.parametrize("dtype, mask", MASKS)
def test_distillation(dtype, mask, tau, tail):
    z, _ = masked_rows(mask, 4)
    # live places and masked ones; in every row something live is left to the others
    index = torch.tensor([[3, 9000, 8], [17500, 17599, 17999], [0, 2, 1], [5, 8199, 18000], [0, 1, 2], [0, 3000, 1]])
    logp = torch.log(torch.tensor([[0.5, 0.3, 0.01]])).repeat(6, 1)
    check_distill(place(z, dtype, 3), index, logp, tail, tau, torch.linspace(0.5, 2, 6))


@pytest.mark.parametrize("tau", [0.7, 1.0, 5.0])
@pytest.mark.parametrize("offset", [1e3, -1e5, 1e6, -3e6, 1e7, 1e9, 1e10, 1e20, -1e30, 1e37])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_common_offset(dtype, offset, tau):
    """Values a few representable steps around a large number, and far below it."""
    vocab = 10007
    g = torch.Generator().manual_seed(7)
    step = abs(offset) * torch.finfo(dtype).eps
    z = offset + step * torch.randint(-3, 3, (3, vocab), generator=g).double()
    z[1] = offset
    z[2, ::2] = -abs(offset) * 8
    z = z.to(dtype).float()
    tokens = torch.tensor([1, 10000, 5001])
    got, r = check_logprobs(place(z, dtype), tokens, 7, tau)
    gl, ge = torch.ones(3), torch.full((3,), 0.25)
    want, tol = grad_logprobs(r, tokens, gl, ge)
    check_grad(ops.logprobs_backward(place(z, dtype), tokens.cuda(), got.stats, gl.cuda(), ge.cuda(), temperature=tau),
               want, tol, dtype, "grad")
    # the first places hold the row's largest value too, so that something of its size is left
    z[:, :2] = z.amax(1, keepdim=True)
    index = torch.stack([torch.zeros(3, dtype=torch.int64), tokens], 1)
    for tail in (True, False):
        check_distill(place(z, dtype), index, torch.tensor([[-0.5, -2.0]]).repeat(3, 1), tail, tau, gl)


@pytest.mark.parametrize("tau", [1e20, 1e30, 1e37, 1e38, 3e38])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_very_large_temperatures(dtype, tau):
    """All that is not masked is alike; what is masked stays so."""
    z, tokens = masked_rows(-INF, 9)
    z[4] = -INF
    check_logprobs(place(z, dtype), tokens, 5, tau)
    index = torch.tensor([[3, 9000, 8]]).repeat(6, 1)
    logp = torch.log(torch.tensor([[0.5, 0.3, 0.0]])).repeat(6, 1)
    index[1:4] = torch.tensor([[17500, 17599, 0], [0, 2, 4], [5, 8199, 1]])
    index[5] = torch.tensor([0, 3000, 6000])
    for tail in (True, False):
        check_distill(place(z, dtype), index, logp, tail, tau, torch.full((6,), math.sqrt(tau)))
