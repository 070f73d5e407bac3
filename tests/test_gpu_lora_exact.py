"""All bits of the adapters' low-rank values and of an fp32 gradient: whole numbers
chosen so that every product and every sum on the way is a whole number below 2^24,
and the result has no rounding at all.  Whatever is cut off shows."""
import pytest
import torch

from paper_2504_11651_amd import ops

from conftest import gpu_available

DTYPES = [torch.float32, torch.bfloat16]
on_gpu = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs an MI355X")]


def gpu(f):
    for m in on_gpu:
        f = m(f)
    return f


def digits(v):
    """Whole numbers below 2^24 as three of 8 bits, the lowest first."""
    return [(v.abs() >> (8 * i) & 255) * v.sign() for i in range(3)]


def low_values(tokens, rank, pairs, seed):
    """What v (or u) is to be: of either sign, with bits in all three digits; with
    `pairs` the second half of the ranks takes all but the lowest digit away again."""
    g = torch.Generator().manual_seed(seed)
    v = torch.randint(1, 1 << 23, (tokens, rank), generator=g) | 0x410081
    v *= 2 * torch.randint(2, (tokens, rank), generator=g) - 1
    if pairs:
        half = rank // 2
        v[:, half:] = -(v[:, :half] - digits(v[:, :half])[0])
    return v


def forward(tokens, rank, n, dtype, seed, cols=64, rows=256):
    """x, a, b, adapter and what the adapters add, in whole numbers: A_i picks rank r's
    digits out of x (times 1, 2^8, 2^16), B_i sends rank r to the rows of r."""
    pairs = dtype == torch.bfloat16
    g = torch.Generator().manual_seed(seed)
    adapter = torch.randint(-1, n, (tokens,), generator=g).sort().values.int()
    x = torch.zeros((tokens, cols), dtype=torch.int64)
    a, b = torch.zeros((n, rank, cols), dtype=torch.int64), torch.zeros((n, rows, rank), dtype=torch.int64)
    # x holds the powers, A the digits: every token of an adapter has the same v
    x[:, :3] = torch.tensor([1, 256, 65536])
    v = low_values(n, rank, pairs, seed + 1)
    a[:, :, :3] = torch.stack(digits(v), 2)
    for r in range(rank):
        b[:, r % (rank // 2 if pairs else rank)::rank // 2 if pairs else rank, r] = 1
    add = torch.zeros((tokens, rows), dtype=torch.int64)
    for t in range(tokens):
        if adapter[t] >= 0:
            add[t] = b[adapter[t]] @ v[adapter[t]]
    return x, a, b, adapter, add


CASES = [(tokens, rank) for tokens in (1, 5, 64, 65, 300) for rank in (8, 16, 24, 32, 40, 64, 128)] + [(9000, 16), (4200, 64)]


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tokens, rank", CASES)
def test_forward(tokens, rank, dtype):
    x, a, b, adapter, add = forward(tokens, rank, 3, dtype, rank)
    base = torch.randint(-60, 60, add.shape, generator=torch.Generator().manual_seed(1))
    got = ops.lora(x.bfloat16().cuda(), a.bfloat16().cuda(), b.bfloat16().cuda(), None, adapter.cuda(),
                   base=base.to(dtype).cuda())
    assert torch.equal(got.cpu(), (base + add).to(dtype))


@gpu
@pytest.mark.parametrize("tokens, rank", CASES)
def test_dx(tokens, rank):
    """The same with the sides exchanged: u from a dy of powers, dx in BF16."""
    x, a, b, adapter, add = forward(tokens, rank, 3, torch.bfloat16, rank + 1)
    at, bt = b.transpose(1, 2).contiguous(), a.transpose(1, 2).contiguous()  # (n, rank, 256), (n, 64, rank)
    zeros = torch.zeros((tokens, 256), dtype=torch.bfloat16, device="cuda")
    for dtype in DTYPES:
        got = ops.lora_backward(zeros, at.bfloat16().cuda(), bt.bfloat16().cuda(), None, adapter.cuda(),
                                x.to(dtype).cuda(), need_ab=False)
        assert torch.equal(got.dx.cpu(), add.bfloat16())


@gpu
@pytest.mark.parametrize("tokens, rank", CASES)
def test_da_and_db(tokens, rank):
    """dA from a u of 24 bits and an x that is 1 at one place of a token, dB from an
    fp32 dy of 24 bits where v is small, and from a v of 24 bits where dy is small."""
    n, cols, rows = 3, 64, 256
    g = torch.Generator().manual_seed(rank)
    adapter = torch.randint(-1, n, (tokens,), generator=g).int()
    one = torch.zeros((tokens, cols), dtype=torch.int64)
    # the first tokens only, so that no two of them meet in a sum
    live = torch.arange(min(tokens, cols))
    one[live, live] = 1
    dy = torch.zeros((tokens, rows), dtype=torch.int64)
    dy[:, :rank] = low_values(tokens, rank, False, 3)
    dy[len(live):] = 0
    a = torch.zeros((n, rank, cols), dtype=torch.int64)
    a[:] = torch.randint(1, 2, a.shape)  # v[t][r] = sum of x[t]
    b = torch.zeros((n, rows, rank), dtype=torch.int64)
    for r in range(rank):
        b[:, r, r] = 1
    got = ops.lora_backward(one.bfloat16().cuda(), a.bfloat16().cuda(), b.bfloat16().cuda(), None, adapter.cuda(),
                            dy.float().cuda(), need_dx=False)
    da = torch.zeros(a.shape, dtype=torch.int64)
    for t in live.tolist():
        if adapter[t] >= 0:
            da[adapter[t], :, t] += dy[t, :rank]
    assert torch.equal(got.da.cpu().long(), da)
    # one token of an adapter gives dB its dy; several a sum that may round, so one each
    first = [int((adapter == i).nonzero()[0]) if (adapter == i).any() else -1 for i in range(n)]
    lone = torch.full_like(adapter, -1)
    for i, t in enumerate(first):
        if 0 <= t < len(live):
            lone[t] = i
    for dtype in DTYPES:
        x = one if dtype == torch.float32 else one * 0
        y = dy if dtype == torch.float32 else torch.zeros_like(dy)
        ai = a.clone()
        if dtype == torch.bfloat16:  # v of 24 bits against a dy of one
            x[:, :3] = torch.tensor([1, 256, 65536])
            v = low_values(n, rank, False, 4)
            ai[:, :, :3] = torch.stack(digits(v), 2)
            y[torch.arange(tokens), torch.arange(tokens) % rows] = 1
        got = ops.lora_backward(x.bfloat16().cuda(), ai.bfloat16().cuda(), b.bfloat16().cuda(), None, lone.cuda(),
                                y.to(dtype).cuda(), need_dx=False)
        db = torch.zeros(b.shape, dtype=torch.int64)
        for i, t in enumerate(first):
            if 0 <= t < len(live):
                db[i] = y[t][:, None] * (v[i] if dtype == torch.bfloat16 else torch.ones(rank, dtype=torch.int64))
        assert torch.equal(got.db.cpu().long(), db), dtype


def test_a_lost_term_would_show():
    """The oracle with two digits of three, as if the last term of a low-rank value
    were dropped, differs wherever a token has an adapter."""
    for dtype in DTYPES:
        x, a, b, adapter, add = forward(40, 16, 3, dtype, 16)
        cut = a.clone()
        cut[:, :, 0] = 0
        for t in range(40):
            less = b[adapter[t]] @ (cut[adapter[t]] @ x[t])
            assert adapter[t] < 0 or (less != add[t]).all()


@gpu
@pytest.mark.parametrize("tokens, rank", [(5, 8), (50, 40), (300, 16), (5000, 64)])
def test_infinite_weights_stay_with_their_adapter(tokens, rank):
    """An infinity or a NaN in one adapter's A or B, in a row of B that others' rows of
    the same tile pass by, reaches its own tokens, and of these its own row, alone."""
    n, cols, rows = 3, 128, 256
    g = torch.Generator().manual_seed(tokens)
    x = torch.randn((tokens, cols), generator=g).bfloat16().cuda()
    a = torch.randn((n, rank, cols), generator=g).bfloat16().cuda()
    b = torch.randn((n, rows, rank), generator=g).bfloat16().cuda()
    dy = torch.randn((tokens, rows), generator=g).cuda()
    adapter = (torch.arange(tokens) % (n + 1) - 1).int().cuda()
    own, others = adapter == 1, adapter != 1
    for dtype in DTYPES:
        base = dy.to(dtype)
        out = ops.lora(x, a, b, None, adapter, base=base)
        back = ops.lora_backward(x, a, b, None, adapter, base)
        for value in (float("inf"), float("nan")):
            bad = b.clone()
            bad[1, 77, 3] = value
            got = ops.lora(x, a, bad, None, adapter, base=base)
            row = torch.arange(rows, device="cuda") == 77
            assert torch.equal(got[others], out[others]) and torch.equal(got[own][:, ~row], out[own][:, ~row])
            assert not torch.isfinite(got[own][:, row]).any()
            bad = a.clone()
            bad[1, 2, 5] = value
            assert torch.equal(ops.lora(x, bad, b, None, adapter, base=base)[others], out[others])
            got = ops.lora_backward(x, bad, b, None, adapter, base)
            col = torch.arange(cols, device="cuda") == 5
            assert torch.equal(got.dx[others], back.dx[others])
            assert torch.equal(got.dx[own][:, ~col], back.dx[own][:, ~col])
            for i in (0, 2):
                assert torch.equal(got.da[i], back.da[i]) and torch.equal(got.db[i], back.db[i])
