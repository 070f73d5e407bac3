"""Low-rank adapters on the GPU against their definition in 64 bits.

Tolerances: a sum of n products in 32 bits is within n 2^-24 of the sum of the
products' sizes, whatever its order; the low-rank intermediate keeps 16 bits of
mantissa (2^-16 of its size, in each of the two factors of a product where both
are split); an output adds the rounding of its type."""
import pytest
import torch

from paper_2504_11651_amd import codec, ops

from conftest import gpu_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs an MI355X")]

ROUND = {torch.float32: 2.0 ** -23, torch.bfloat16: 2.0 ** -8}
E, SPLIT = 2.0 ** -24, 2.0 ** -16


def rows_of(t, pad=0, offset=0, dtype=None):
    """A copy on the GPU with `pad` NaNs after each row and `offset` in front."""
    n, c = t.shape
    dtype = dtype or t.dtype
    whole = torch.full((offset + n * (c + pad),), float("nan"), dtype=dtype, device="cuda")
    v = whole[offset:].view(n, c + pad)[:, :c]
    v.copy_(t)
    return v


def draw(tokens, cols, rows, rank, n, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((tokens, cols), generator=g).bfloat16()
    a = (torch.randn((n, rank, cols), generator=g) * cols ** -0.5).bfloat16()
    b = (torch.randn((n, rows, rank), generator=g) * 0.1).bfloat16()
    scale = torch.rand(n, generator=g) + 0.5
    y = torch.randn((tokens, rows), generator=g)
    z = torch.randn((tokens, cols), generator=g).bfloat16()
    return x, a, b, scale, y, z


def near(got, want, tol, what):
    got = got.double().cpu()
    off = (got - want).abs()
    bad = ~(off <= tol)
    assert not bad.any(), (what, int(bad.sum()), bad.nonzero()[:3], got[bad][:4], want[bad][:4], tol[bad][:4])


def forward_want(x, a, b, scale, adapter, base):
    """The output and its tolerance without its own rounding."""
    x, a, b, scale = x.double(), a.double(), b.double(), scale.double()
    cols, rank = a.shape[2], a.shape[1]
    out, tol = base.double().clone(), torch.zeros_like(base, dtype=torch.double)
    for i in range(a.shape[0]):
        t = (adapter == i).nonzero()[:, 0]
        v, dv = x[t] @ a[i].T, cols * E * (x[t].abs() @ a[i].abs().T)
        out[t] += scale[i] * (v @ b[i].T)
        tol[t] += scale[i] * ((dv + (SPLIT + (3 * rank + 8) * E) * (v.abs() + dv)) @ b[i].abs().T)
    return out, tol


def backward_want(x, a, b, scale, adapter, dy, dx_base, split_dy):
    x, a, b, scale, dy = x.double(), a.double(), b.double(), scale.double(), dy.double()
    cols, rank, rows = a.shape[2], a.shape[1], b.shape[1]
    dx, tol_dx = dx_base.double().clone(), torch.zeros_like(dx_base, dtype=torch.double)
    da, db = torch.zeros_like(a), torch.zeros_like(b)
    tol_da, tol_db = torch.zeros_like(a), torch.zeros_like(b)
    sy = SPLIT if split_dy else 0.0
    for i in range(a.shape[0]):
        t = (adapter == i).nonzero()[:, 0]
        n = len(t)
        v, dv = x[t] @ a[i].T, cols * E * (x[t].abs() @ a[i].abs().T)
        u = scale[i] * (dy[t] @ b[i])
        du = scale[i] * ((3 * rows * E + sy) * (dy[t].abs() @ b[i].abs()))
        dx[t] += u @ a[i]
        tol_dx[t] += (du + (SPLIT + (3 * rank + 8) * E) * (u.abs() + du)) @ a[i].abs()
        da[i] = u.T @ x[t]
        tol_da[i] = (du + (SPLIT + (2 * n + 64) * E) * (u.abs() + du)).T @ x[t].abs()
        db[i] = scale[i] * (dy[t].T @ v)
        tol_db[i] = scale[i] * (dy[t].abs().T @ (dv + (SPLIT + sy + (3 * n + 64) * E) * (v.abs() + dv)))
    return (dx, tol_dx), (da, tol_da), (db, tol_db)


def check(tokens, cols, rows, rank, n, adapter, dtype, seed, pad=0, offset=0, ab=True):
    x, a, b, scale, y, z = draw(tokens, cols, rows, rank, n, seed)
    y = y.to(dtype)
    args = [rows_of(x, pad, offset), a.cuda(), b.cuda(), scale.cuda(), adapter.cuda()]
    base = rows_of(y, pad, offset)
    want, tol = forward_want(x, a, b, scale, adapter, y)
    got = ops.lora(*args, base=base)
    assert got.dtype == dtype
    near(got, want, tol + want.abs() * ROUND[dtype] + 1e-37, "out")
    alone = (adapter < 0) | (adapter >= n)
    assert torch.equal(got.cpu()[alone], y[alone])
    wants = backward_want(x, a, b, scale, adapter, y, z, dtype == torch.float32)
    back = ops.lora_backward(*args, rows_of(y, pad, offset), dx_base=rows_of(z, pad, offset))
    for name, g, (w, t) in zip(("dx", "da", "db"), back, wants):
        near(g, w, t + w.abs() * ROUND[g.dtype] + 1e-37, name)
    assert torch.equal(back.dx.cpu()[alone], z[alone])
    for i in range(n):
        if not (adapter == i).any():
            assert not back.da[i].any() and not back.db[i].any()
    return args, y, z, got, back


def runs(tokens, n, seed, none=True):
    """Adapters of ragged requests, some without."""
    g = torch.Generator().manual_seed(seed)
    which = torch.randint(-1 if none else 0, n, (max(1, tokens // 5),), generator=g)
    return which[torch.randint(len(which), (tokens,), generator=g).sort().values].int()


DTYPES = [torch.float32, torch.bfloat16]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rank", [8, 16, 24, 32, 40, 56, 64, 72, 104, 128])
def test_ranks(rank, dtype):
    for tokens in (1, 7, 50):
        check(tokens, 256, 176, rank, 3, runs(tokens, 3, rank), dtype, rank)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tokens", [1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 100, 127, 129, 255, 257, 300, 513, 1000])
def test_tokens(tokens, dtype):
    check(tokens, 192, 208, 16, 4, runs(tokens, 4, tokens), dtype, tokens, pad=8, offset=8)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols, rows", [(64, 16), (64, 1040), (128, 48), (320, 4112), (4096, 1024), (1024, 4096),
                                        (8192, 80), (14336, 336), (576, 14352)])
def test_shapes(cols, rows, dtype):
    for tokens in (3, 70):
        check(tokens, cols, rows, 16, 2, runs(tokens, 2, cols), dtype, rows)
    check(40, cols, rows, 64, 2, runs(40, 2, rows), dtype, cols, pad=16)


@pytest.mark.parametrize("kind", ["one each", "scattered", "one for all", "none", "out of range", "last only"])
@pytest.mark.parametrize("tokens", [5, 64, 200])
def test_adapters(kind, tokens):
    n = 21
    g = torch.Generator().manual_seed(tokens)
    adapter = {"one each": torch.arange(tokens) % n, "scattered": torch.randint(-1, n, (tokens,), generator=g),
               "one for all": torch.full((tokens,), 3), "none": torch.full((tokens,), -1),
               "out of range": torch.where(torch.arange(tokens) % 3 > 0, torch.tensor(2 ** 31 - 1), n - 1),
               "last only": torch.where(torch.arange(tokens) == tokens - 1, n - 1, -2)}[kind].int()
    for dtype in DTYPES:
        check(tokens, 128, 160, 8, n, adapter, dtype, tokens)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rank", [8, 16, 24, 32, 40, 64, 72, 128])
@pytest.mark.parametrize("kind", ["runs", "scattered", "one for all", "mostly none"])
def test_many_tokens(kind, rank, dtype):
    """More tokens than are spread over workgroups by adapter."""
    n, tokens = 5, 333
    g = torch.Generator().manual_seed(rank)
    adapter = {"runs": runs(tokens, n, rank), "scattered": torch.randint(-1, n, (tokens,), generator=g).int(),
               "one for all": torch.full((tokens,), 2, dtype=torch.int32),
               "mostly none": torch.where(torch.rand(tokens, generator=g) < 0.05, 4, -1).int()}[kind]
    check(tokens, 448, 336, rank, n, adapter, dtype, rank)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tokens, rank", [(6001, 16), (8211, 24), (4099, 64), (2131, 128)])
@pytest.mark.parametrize("scattered", [False, True])
def test_long_prompts(tokens, rank, scattered, dtype):
    """So many values that a wave takes tiles of tokens of its own: whole tiles of one
    adapter, tiles that several share, tokens without."""
    n = 3
    g = torch.Generator().manual_seed(tokens)
    adapter = torch.randint(-1, n, (tokens,), generator=g).int() if scattered else runs(tokens, n, rank)
    check(tokens, 4096, 48, rank, n, adapter, dtype, rank)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n", [1, 3, 40])
def test_chunks_of_tokens(n, dtype):
    """Token counts that the gradients take in several chunks, and in more than one
    look at the adapters; some chunks hold nothing of an adapter."""
    tokens = 9100
    adapter = (torch.arange(tokens) // 700 % (n + 1) - 1).int()
    check(tokens, 64, 48, 16, n, adapter, dtype, n)


@pytest.mark.parametrize("dtype", DTYPES)
def test_optional_arguments(dtype):
    tokens, n = 37, 3
    x, a, b, scale, y, z = draw(tokens, 128, 96, 16, n, 5)
    adapter = runs(tokens, n, 6)
    args = [x.cuda(), a.cuda(), b.cuda()]
    ad = adapter.cuda()
    ones = torch.ones(n)
    none = torch.zeros_like(y)
    want, tol = forward_want(x, a, b, ones, adapter, none)
    out = torch.full((tokens, 96), float("nan"), dtype=dtype, device="cuda")
    got = ops.lora(*args, None, ad, out=out)
    assert got is out
    near(got, want, tol + want.abs() * ROUND[dtype] + 1e-37, "no base, no scale")
    assert not got[((adapter < 0) | (adapter >= n)).cuda()].any()
    assert ops.lora(*args, None, ad).dtype == torch.float32
    # in place
    base = y.to(dtype).cuda()
    want = ops.lora(*args, scale.cuda(), ad, base=base)
    got = ops.lora(*args, scale.cuda(), ad, base=base, out=base)
    assert got.data_ptr() == base.data_ptr() and torch.equal(got, want)
    dy = y.to(dtype).cuda()
    full = ops.lora_backward(*args, scale.cuda(), ad, dy, dx_base=z.cuda())
    only = ops.lora_backward(*args, scale.cuda(), ad, dy, need_dx=False)
    assert only.dx is None and torch.equal(only.da, full.da) and torch.equal(only.db, full.db)
    zc = z.cuda()
    only = ops.lora_backward(*args, scale.cuda(), ad, dy, dx_base=zc, dx=zc, need_ab=False)
    assert only.da is None and only.db is None and torch.equal(zc, full.dx)
    (w, t), _, _ = backward_want(x, a, b, ones, adapter, dy.cpu(), torch.zeros_like(z), dtype == torch.float32)
    got = ops.lora_backward(*args, None, ad, dy)
    near(got.dx, w, t + w.abs() * ROUND[torch.bfloat16] + 1e-37, "dx alone")


def test_no_tokens():
    x, a, b, scale, y, z = draw(4, 64, 16, 8, 2, 1)
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    args = [x[:0].cuda(), a.cuda(), b.cuda(), scale.cuda(), none]
    assert ops.lora(*args).shape == (0, 16)
    back = ops.lora_backward(*args, y[:0].cuda())
    assert back.dx.shape == (0, 64) and not back.da.any() and not back.db.any()
    assert back.da.shape == a.shape and back.db.shape == b.shape


def test_gradients_against_differences():
    """The slope of sum(w * out) along a direction in x, A and B."""
    tokens, cols, rows, rank, n = 23, 128, 64, 8, 2
    x, a, b, scale, y, z = draw(tokens, cols, rows, rank, n, 9)
    adapter = runs(tokens, n, 10)
    w = torch.randn(y.shape, generator=torch.Generator().manual_seed(3))
    back = ops.lora_backward(x.cuda(), a.cuda(), b.cuda(), scale.cuda(), adapter.cuda(), w.cuda())
    steps = [torch.randn(t.shape, generator=torch.Generator().manual_seed(k)).double() for k, t in enumerate((x, a, b))]
    wants = backward_want(x, a, b, scale, adapter, w, torch.zeros_like(z), True)
    for k, (got, (_, tol)) in enumerate(zip(back, wants)):
        def value(h):
            at = [t.double() + (h * steps[k] if k == j else 0) for j, t in enumerate((x, a, b))]
            return (forward_want(*at, scale, adapter, torch.zeros_like(y))[0] * w.double()).sum()

        slope = (value(1.0) - value(-1.0)) / 2  # linear in each of the three
        g = got.double().cpu()
        room = (tol * steps[k].abs()).sum() + (g * steps[k]).abs().sum() * ROUND[got.dtype] + 1e-9 * abs(float(slope))
        assert abs(float((g * steps[k]).sum() - slope)) <= float(room), k


def test_values_that_spread():
    """Masked-out gradients (zeros), large and tiny values, an infinity of one
    token that must not reach another's row."""
    tokens, n = 48, 2
    x, a, b, scale, y, z = draw(tokens, 128, 64, 16, n, 11)
    adapter = (torch.arange(tokens) % 3 - 1).int()
    x[5] *= 1e4
    x[6] *= 1e-4
    y[7] = 0
    want, tol = forward_want(x, a, b, scale, adapter, y)
    args = [x.cuda(), a.cuda(), b.cuda(), scale.cuda(), adapter.cuda()]
    near(ops.lora(*args, base=y.cuda()), want, tol + want.abs() * ROUND[torch.float32], "spread")
    clean = ops.lora(*args, base=y.cuda())
    clean_back = ops.lora_backward(*args, y.cuda())
    x[9, 3] = float("inf")
    x[11, 4] = float("nan")
    y[9, 2] = float("nan")
    args[0] = x.cuda()
    got = ops.lora(*args, base=y.cuda())
    back = ops.lora_backward(*args, y.cuda())
    others = [t for t in range(tokens) if t not in (9, 11)]
    assert adapter[9] == -1 and adapter[11] == 1
    assert torch.equal(got[others], clean[others]) and torch.equal(back.dx[others], clean_back.dx[others])
    assert torch.equal(got[9].cpu().isnan(), y[9].isnan()) and got[11].isnan().all()
    # a token without an adapter counts nowhere, whatever it holds
    assert torch.equal(back.da[0], clean_back.da[0]) and torch.equal(back.db[0], clean_back.db[0])


def test_rows_past_32_bit_offsets():
    """x and out with rows 2^30 + 8 elements apart: the last starts past 2^32."""
    tokens, stride = 6, (1 << 30) + 8
    x, a, b, scale, y, z = draw(tokens, 64, 32, 8, 2, 12)
    adapter = torch.tensor([0, 1, -1, 0, 1, 1], dtype=torch.int32)
    whole = torch.empty((tokens - 1) * stride + 128, dtype=torch.bfloat16, device="cuda")
    xs, ys = whole.as_strided((tokens, 64), (stride, 1)), whole.as_strided((tokens, 32), (stride, 1), 64)
    xs.copy_(x)
    ys.copy_(y)
    want, tol = forward_want(x, a, b, scale, adapter, ys.cpu())
    wants = backward_want(x, a, b, scale, adapter, ys.cpu(), x, False)
    args = [xs, a.cuda(), b.cuda(), scale.cuda(), adapter.cuda()]
    back = ops.lora_backward(*args, ys, dx_base=xs)
    for name, g, (w, t) in zip(("dx", "da", "db"), back, wants):
        near(g, w, t + w.abs() * ROUND[g.dtype] + 1e-37, name)
    got = ops.lora(*args, base=ys, out=ys)
    near(got, want, tol + want.abs() * ROUND[torch.bfloat16] + 1e-37, "out")


def everything(x, a, b, scale, adapter, y, z, **more):
    return [ops.lora(x, a, b, scale, adapter, base=y, **more),
            *ops.lora_backward(x, a, b, scale, adapter, y, dx_base=z, **more)]


@pytest.mark.parametrize("tokens, rank", [(1, 16), (40, 32), (700, 8)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_streams_graphs_and_repeats(tokens, rank, dtype):
    n = 3
    x, a, b, scale, y, z = (t.cuda() for t in draw(tokens, 1024, 528, rank, n, 13))
    x2, y2 = (t.cuda() for t in (draw(tokens, 1024, 528, rank, n, 14)[k] for k in (0, 4)))
    y, y2 = y.to(dtype), y2.to(dtype)
    rest = [a, b, scale, runs(tokens, n, 15, none=False).cuda()]
    want, want2 = everything(x, *rest, y, z), everything(x2, *rest, y2, z)
    for p, q in zip(want, everything(x, *rest, y, z)):
        assert torch.equal(p, q)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        got = everything(x2.clone(), *rest, y2.clone(), z)
    side.synchronize()
    for p, q in zip(want2, got):
        assert torch.equal(p, q)
    got = everything(x, *rest, y, z, stream=side)
    side.synchronize()
    for p, q in zip(want, got):
        assert torch.equal(p, q)
    xh, yh = x.clone(), y.clone()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        replayed = everything(xh, *rest, yh, z)
    for k in range(4):
        xh.copy_(x2 if k % 2 else x)
        yh.copy_(y2 if k % 2 else y)
        for t in replayed:
            t.fill_(-7)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for p, q in zip(want2 if k % 2 else want, replayed):
            assert torch.equal(p, q), k
        everything(x, *rest, y, z)


def test_what_is_refused():
    x, a, b, scale, y, z = (t.cuda() for t in draw(4, 64, 32, 8, 2, 16))
    ad = torch.zeros(4, dtype=torch.int32, device="cuda")
    for call in (lambda: ops.lora(x.float(), a, b, scale, ad), lambda: ops.lora(x, a.float(), b, scale, ad),
                 lambda: ops.lora(x, a, b[:1], scale, ad), lambda: ops.lora(x, a, b, scale, ad.long()),
                 lambda: ops.lora(x, a, b, scale[:1], ad), lambda: ops.lora(x[:, :32], a, b, scale, ad),
                 lambda: ops.lora(x, a, b, scale, ad, base=y.half()), lambda: ops.lora(x, a, b, scale, ad, base=y[:3]),
                 lambda: ops.lora(x, a, b, scale, ad, base=y, out=y.bfloat16()),
                 lambda: ops.lora(x.cpu(), a, b, scale, ad), lambda: ops.lora(x, a.cpu(), b, scale, ad),
                 lambda: ops.lora_backward(x, a, b, scale, ad, y[:, :16]),
                 lambda: ops.lora_backward(x, a, b, scale, ad, y, dx=z.float()),
                 lambda: ops.lora_backward(x, a, b, scale, ad, y, da=a)):
        with pytest.raises(ValueError):
            call()
    wide = torch.zeros((4, 68), dtype=torch.bfloat16, device="cuda")
    for call in (lambda: ops.lora(wide[:, :64], a, b, scale, ad),
                 lambda: ops.lora(x, a[:, :4].contiguous(), b[:, :, :4].contiguous(), scale, ad),
                 lambda: ops.lora(x, a, b, scale, ad, workspace=torch.empty(4, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(codec.DF11Error):
            call()
