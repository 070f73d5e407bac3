"""The position rotation at far positions: angles next to whole turns, whose sines show
what of the angle's fraction of a turn was lost, against exact whole numbers."""
import math

import pytest
import torch

from paper_2504_11651_amd import ops

from conftest import gpu_available
from kv_reference import BF16, F16, Case, half_step, near

BITS = 200  # behind the binary point


def _pi():
    """pi in BITS + 20 binary places, by Machin's formula 16 atan(1/5) - 4 atan(1/239)."""
    one = 1 << BITS + 20

    def atan_of_inverse(n):
        term, total, k = one // n, 0, 0
        while term:
            total += (-1) ** k * (term // (2 * k + 1))
            term //= n * n
            k += 1
        return total

    return 16 * atan_of_inverse(5) - 4 * atan_of_inverse(239)


TURNS = (1 << 2 * BITS + 20) // (2 * _pi())  # 1 / (2 pi) in BITS binary places


def fraction(position, frequency):
    """position * frequency / (2 pi) without its nearest whole number, in 64 bits; frequency:
    a multiple of 2^-24."""
    turns = position * int(frequency * 2 ** 24) * TURNS >> 24
    rest = turns & (1 << BITS) - 1
    return (rest - (1 << BITS) * (rest >> BITS - 1)) / (1 << BITS)


def near_whole_turns(position, n, most):
    """n frequencies of 24 bits between a half and one whose angles at this position are
    less than `most` of a turn from a whole one, but not less than a thousandth of that."""
    found, step = [], position * TURNS >> 24
    mask, limit = (1 << BITS) - 1, int(most * (1 << BITS))
    f = 1 << 23
    while len(found) < n:
        # the next one that is near: of an arithmetic sequence on a circle
        turns = position * f * TURNS >> 24 & mask
        while not (turns < limit or mask - turns < limit):
            turns = turns + step & mask
            f += 1
        if abs(fraction(position, f / 2 ** 24)) > most / 1000:
            found.append(f / 2 ** 24)
        f += 1
        assert f < 1 << 24
    return found


def test_the_whole_numbers():
    assert fraction(1, 0.5) == pytest.approx(0.5 / (2 * math.pi), rel=1e-15)
    assert fraction(10, 0.5) == pytest.approx(5 / (2 * math.pi) - 1, rel=1e-14)
    assert TURNS / (1 << BITS) == 1 / (2 * math.pi)


@pytest.mark.gpu
@pytest.mark.skipif(not gpu_available(), reason="needs an MI355X")
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("position", [1000, 131071, 10 ** 7 + 3, 2 ** 28 + 1, 2 ** 29 - 5, 2 ** 30 + 7, 2 ** 31 - 77,
                                      2 ** 31 + 99, 2 ** 32 - 3])
def test_angles_next_to_whole_turns(position, dtype, interleaved):
    """Pairs (0, b) give (-b sin, b cos) of a small angle.  Its fraction of a turn is held in
    64 bits and rounded once to 32, by 2^-24 of itself; sine and cosine are off by 2^-22, the
    products and the sum by 2^-22 more, the result by half a step."""
    most = 2.0 ** (-19 if position > 2 ** 24 else -14 if position > 10 ** 5 else -10)
    n = 16 if most < 2 ** -15 else 32
    freq = near_whole_turns(position, n, most)
    angle = torch.tensor([2 * math.pi * fraction(position, f) for f in freq], dtype=torch.float64, device="cuda")
    inv_freq = torch.tensor(freq, device="cuda")
    assert inv_freq.tolist() == freq
    # the row's place is a page's last token at most; the rest of its position is the prefix
    own = 50 if position < 2 ** 31 else 2 ** 31 - 1
    c = Case([1], [50], heads=4, kv_heads=2, dim=64, dtype=dtype, filled=False)
    c.length.fill_(own)
    batch = ops.KVBatch(c.start, c.length, c.table, None, position - (own - 1))
    b = 4096.0
    first, second = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    q, k = (torch.zeros((1, h, 64), device="cuda") for h in (4, 2))
    q[..., second], k[..., second] = b, b
    got = ops.kv_append(q.flatten(1), k.flatten(1), k.flatten(1), inv_freq, c.cache, batch, interleaved=interleaved)
    results = [got.view(4, 64)]
    if own == 50:  # appended
        results.append(c.k[c.pages[0][49 // 64], :, 49])
    for x in results:
        for place, want in ((first, -b * angle.sin()), (second, b * angle.cos())):
            tol = want.abs() * (half_step(dtype) + 2 ** -20) + (2 ** -25 if dtype == F16 else 0)
            near(x[:, place], want.expand(x.shape[0], n), tol.expand(x.shape[0], n), f"position {position}")
