"""Appending to a paged cache with the position rotation, against its definition in 64
bits, and the cache's operators together with the products around them."""
import math

import pytest
import torch

from paper_2504_11651_amd import codec, ops

from conftest import gpu_available
from kv_reference import BF16, F16, F32, Case, half_step, near

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs an MI355X")]


def frequencies(rotary, base=500000.0):
    return (base ** -(torch.arange(rotary // 2, dtype=torch.float64, device="cuda") / max(rotary // 2, 1))).float()


def rotated(x, position, inv_freq, interleaved, dim, dtype):
    """x (rows, heads * dim) turned, in 64 bits, and how far a result may be off: an
    angle by 2^-22 (half a step of a fraction of a turn in 32 bits, times 2 pi), its
    cosine and sine by 2^-23 more, the two products and their sum by 2^-23, the result by
    half a step of its type (of the least normal value for a half float)."""
    x = x.double().view(x.shape[0], -1, dim)
    want, size = x.clone(), x.abs().clone()
    n = inv_freq.numel()
    if n:
        j = torch.arange(n, device=x.device)
        a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + n)
        angle = (position.double()[:, None] * inv_freq.double())[:, None]
        c, s = angle.cos(), angle.sin()
        want[..., a] = x[..., a] * c - x[..., b] * s
        want[..., b] = x[..., b] * c + x[..., a] * s
        size[..., a] = size[..., b] = x[..., a].abs() + x[..., b].abs()
    tol = size * (2 ** -21 if n else 0) + want.abs() * half_step(dtype) + (2 ** -25 if dtype == F16 else 1e-40)
    return want.flatten(1), tol.flatten(1)


def append(c, source, rotary, interleaved=False, inv_freq=None, sentinel=7.0, **more):
    """Appends random rows of a case and checks everything that the call may write."""
    q = c.normal(c.tokens, c.heads * c.dim).to(source)
    k, v = (c.normal(c.tokens, c.kv_heads * c.dim).to(source) for _ in range(2))
    inv_freq = frequencies(rotary) if inv_freq is None else inv_freq
    c.k.fill_(sentinel), c.v.fill_(sentinel)
    q_out = torch.full((c.tokens, c.heads * c.dim), 77.0, dtype=c.dtype, device="cuda")
    batch = c.batch._replace(prefix_table=None)
    got = ops.kv_append(q, k, v, inv_freq if rotary else None, c.cache, batch, interleaved=interleaved, q_out=q_out,
                        **more)
    assert got is q_out
    check_append(c, q, k, v, inv_freq if rotary else inv_freq[:0], interleaved, q_out, sentinel)
    return q, k, v, q_out


def check_append(c, q, k, v, inv_freq, interleaved, q_out, sentinel):
    rows = sum(c.new)
    place = torch.cat([torch.arange(m - n, m, device="cuda") for n, m in zip(c.new, c.own)] + [
        torch.zeros(0, dtype=torch.int64, device="cuda")])
    seq = torch.repeat_interleave(torch.arange(len(c.new)), torch.tensor(c.new)).tolist()
    position = place + c.prefix
    near(q_out[:rows], *rotated(q[:rows], position, inv_freq, interleaved, c.dim, c.dtype), "q")
    assert (q_out[rows:] == 77.0).all()
    want_k, tol_k = rotated(k[:rows], position, inv_freq, interleaved, c.dim, c.dtype)
    want_v, tol_v = rotated(v[:rows], position, inv_freq[:0], False, c.dim, c.dtype)
    written = torch.zeros(c.k.shape[::2], dtype=torch.bool, device="cuda")  # pages x tokens of a page
    kept = [r for r in range(rows) if 0 <= int(place[r]) < c.table.shape[1] * c.page]
    pages = torch.tensor([int(c.table[seq[r], int(place[r]) // c.page]) for r in kept], dtype=torch.int64,
                         device="cuda")
    there = (pages >= 0) & (pages < c.k.shape[0])
    kept, pages = torch.tensor(kept, dtype=torch.int64, device="cuda")[there], pages[there]
    at = place[kept] % c.page
    near(c.k[pages, :, at].flatten(1), want_k[kept], tol_k[kept], "k")
    near(c.v[pages, :, at].flatten(1), want_v[kept], tol_v[kept], "v")
    written[pages, at] = True
    for cache in (c.k, c.v):
        assert (cache.transpose(1, 2)[~written] == sentinel).all(), "written beside the rows' places"


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("source", [F32, BF16, F16])
@pytest.mark.parametrize("dim, rotary", [(128, 128), (128, 64), (128, 16), (128, 0), (64, 64), (64, 48), (64, 32)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_types_and_rotations(dtype, source, dim, rotary, interleaved):
    append(Case([1, 4, 0, 3], [1, 60, 7, 300], prefix=1234, dim=dim, dtype=dtype, spare=2, filled=False,
                seed=rotary), source, rotary, interleaved)


@pytest.mark.parametrize("heads, kv_heads", [(1, 1), (3, 1), (7, 7), (12, 4), (32, 8), (64, 8), (142, 2)])
@pytest.mark.parametrize("page", [16, 64, 1024])
def test_head_layouts_and_pages(heads, kv_heads, page):
    append(Case([5, 1, 40], [5, page + 1, 2 * page], heads=heads, kv_heads=kv_heads, page=page, filled=False), F32, 64)


@pytest.mark.parametrize("prefix", [0, 4095, 131072, 10 ** 7, 2 ** 30])
def test_far_positions(prefix):
    """The angle's fraction of a turn is as exact at a far position as at a near one."""
    c = Case([3, 1], [3, 1000], filled=False)
    c.prefix = prefix  # its pages are not looked at
    append(c, F32, 128)


def test_rotation_by_whole_turns_changes_nothing():
    """Frequencies of 0: cosines of 1 and sines of 0, so that values stay as they are."""
    c = Case([3, 1], [3, 1000], prefix=999, filled=False)
    q, k, _, q_out = append(c, BF16, 128, inv_freq=torch.zeros(64, device="cuda"))
    assert torch.equal(q_out, q)


def test_ragged_prompts():
    append(Case([700, 1, 0, 333], [700, 65, 4, 1000], heads=32, kv_heads=8, spare=5, filled=False), F32, 128)
    append(Case([2500], [2500], prefix=17, heads=4, kv_heads=4, dim=64, page=16, dtype=F16, filled=False), F16, 32, True)


@pytest.mark.parametrize("sequences", [64, 65, 300, 4097])
def test_many_sequences(sequences):
    own = [1 + (37 * i) % 90 for i in range(sequences)]
    append(Case([min(x, i % 3) for i, x in enumerate(own)], own, heads=2, kv_heads=1, dim=64, page=16, spare=3,
                filled=False), F32, 64)


def test_rows_without_a_place():
    """Places below 0, past the table's width, and on pages outside the cache."""
    append(Case([5, 3, 1], [2, -1, 1], prefix=40, filled=False), F32, 128)
    append(Case([6, 1], [131, 20], page=16, width=8, filled=False), F32, 128)
    for wrong in (-1, 10 ** 6, 2 ** 31 - 1, -2 ** 31):
        c = Case([40, 2], [40, 70], page=16, filled=False)
        c.table[0, 1] = wrong
        append(c, F32, 128)


def test_in_place_and_strides():
    """q, k and v as columns of one tensor, q turned where it lies; pages of a layer."""
    c = Case([3, 1, 40], [100, 200, 40], prefix=77, heads=8, kv_heads=2, filled=False, spare=1)
    wide = c.normal(45, 12 * 128).bfloat16()
    q, k, v = wide.clone().split([1024, 256, 256], dim=1)
    layers = torch.full((c.k.shape[0], 3, 2, *c.k.shape[1:]), 7.0, dtype=BF16, device="cuda")
    c.k, c.v = layers[:, 1, 0], layers[:, 1, 1]
    got = ops.kv_append(wide[:, :1024], wide[:, 1024:1280], wide[:, 1280:], frequencies(128), c.cache, c.batch,
                        q_out=wide[:, :1024])
    assert torch.equal(got[44], q[44])
    got[44] = 77.0
    check_append(c, q, k, v, frequencies(128), False, got, 7.0)
    assert torch.equal(wide[:, 1024:1280], k) and torch.equal(wide[:, 1280:], v)
    assert (layers[:, ::2] == 7.0).all()


def test_far_pages():
    stride = 1 << 31
    c = Case([2, 1], [100, 30], filled=False)
    room = torch.empty((c.k.shape[0] - 1) * stride + 2 * 2 * 64 * 128, dtype=BF16, device="cuda")
    shape = c.k.shape
    c.k, c.v = (room.as_strided(shape, (stride, 64 * 128, 128, 1), i * 2 * 64 * 128) for i in (0, 1))
    append(c, F32, 128)


def test_on_a_stream_and_captured():
    c = Case([1, 2, 1], [100, 200, 30], prefix=9, filled=False, width=8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    q, k, v = (c.normal(4, n * 128) for n in (8, 2, 2))
    torch.cuda.synchronize()
    inv_freq = frequencies(128)
    want = ops.kv_append(q, k, v, inv_freq, c.cache, c.batch)
    torch.cuda.synchronize()
    got = ops.kv_append(q, k, v, inv_freq, c.cache, c.batch, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    out = torch.empty_like(want)
    with torch.cuda.graph(graph):
        ops.kv_append(q, k, v, inv_freq, c.cache, c.batch, q_out=out)
    for i in range(4):
        c.own = [100 + 9 * i, 200 - i, 30 + 40 * i]
        c.length.copy_(torch.tensor(c.own))
        c.table.copy_(torch.randperm(24, generator=torch.Generator().manual_seed(i)).view(3, 8) % c.k.shape[0])
        c.table[:] = torch.arange(3, device="cuda")[:, None]  # a page for each sequence
        q.normal_(), k.normal_(), v.normal_()
        c.k.fill_(7.0), c.v.fill_(7.0), out.fill_(77.0)
        graph.replay()
        torch.cuda.synchronize()
        check_append(c, q, k, v, inv_freq, False, out, 7.0)


def test_products_append_and_attention_of_a_block():
    """A block's attention as a program runs it: products of the compressed block, the
    cache, attention, the output product; two requests' prompts behind a prefix, then
    steps of single tokens, against the same in 64 bits on the operators' inputs."""
    from paper_2504_11651_amd import synth
    hidden, heads, kv_heads, dim, page = 1024, 8, 2, 128, 32
    mats, at = [], 0
    for rows in (heads * dim, kv_heads * dim, kv_heads * dim, hidden):
        mats.append((at, rows, hidden))
        at += rows * hidden
    stream = codec.to_device(codec.encode(synth.gaussian(at, 0.02, 5)), "cuda")
    weights = torch.empty(at, dtype=BF16, device="cuda")
    codec.decode_block(stream, weights)
    ws = torch.empty(max(codec.gemm_workspace_bytes(mats, 64), 16), dtype=torch.uint8, device="cuda")
    inv_freq = frequencies(dim)
    pages = 40
    cache = ops.KVCache(*(torch.zeros((pages, kv_heads, page, dim), dtype=BF16, device="cuda") for _ in range(2)))
    free = torch.randperm(pages, generator=torch.Generator().manual_seed(2)).int().cuda()
    g = torch.Generator(device="cuda").manual_seed(3)
    history = []  # per sequence (0: the prefix), keys and values turned, as 64-bit rows

    def attention(x, batch):
        y = [torch.empty((x.shape[0], r), device="cuda") for _, r, _ in mats[:3]]
        codec.block_gemm(weights, mats[:3], [x] * 3, y, ws)
        q = ops.kv_append(*y, inv_freq, cache, batch)
        out = ops.prefix_attention(q, cache, batch, need_lse=True)
        o = torch.empty((x.shape[0], hidden), device="cuda")
        codec.block_gemm(weights, mats[3:], [out.out], [o], ws)
        return y, q, out, o

    def i32(*values):
        return torch.tensor(values, dtype=torch.int32, device="cuda")

    prefix = 50
    x = torch.randn((prefix, hidden), generator=g, device="cuda").bfloat16()
    table = free[:2].view(1, 2).contiguous()
    y, *_ = attention(x, ops.KVBatch(i32(0, prefix), i32(prefix), table))
    shared = (y[1], y[2])
    own = [[torch.zeros((0, 2 * kv_heads * dim), device="cuda")] for _ in range(2)]
    tables = free[2:12].view(2, 5).contiguous()
    lengths = [0, 0]
    for new in ([20, 43], [1, 1], [0, 1], [1, 1], [3, 2]):
        lengths = [a + b for a, b in zip(lengths, new)]
        x = torch.randn((sum(new), hidden), generator=g, device="cuda").bfloat16()
        batch = ops.KVBatch(i32(0, new[0], sum(new)), i32(*lengths), tables, table[0], prefix)
        y, q, got, o = attention(x, batch)
        for s, part in enumerate(torch.cat(y[1:], 1).split(new)):
            own[s].append(part)
        lo = 0
        for s, n in enumerate(new):
            if not n:
                continue
            rows = torch.cat(own[s])
            k = torch.cat((shared[0], rows[:, :kv_heads * dim]))
            v = torch.cat((shared[1], rows[:, kv_heads * dim:]))
            position = torch.arange(k.shape[0], device="cuda")
            k = rotated(k, position, inv_freq, False, dim, BF16)[0].bfloat16().double().view(-1, kv_heads, dim)
            v = v.bfloat16().double().view(-1, kv_heads, dim)
            wq = rotated(y[0][lo:lo + n], position[k.shape[0] - n:], inv_freq, False, dim, BF16)[0].bfloat16()
            wq = wq.double().view(n, kv_heads, heads // kv_heads, dim)
            for r in range(n):
                end = k.shape[0] - n + r + 1
                scores = (wq[r][:, :, None] * k[:end].transpose(0, 1)[:, None]).sum(-1) / math.sqrt(dim)
                lse = scores.logsumexp(-1)
                p = (scores - lse[..., None]).exp()
                vv = v[:end].transpose(0, 1)[:, None]
                want, weight = (p[..., None] * vv).sum(-2), (p[..., None] * vv.abs()).sum(-2)
                # a rounding of q or k that falls to the other side is a step of one
                # value: 2^-7 |q k| / sqrt(dim) of it in a score; a few of them in a row
                tol = want.abs() * 2 ** -8 + weight * (2 ** -8 + 2 ** -6)
                near(got.out[lo + r], want.flatten(), tol.flatten())
                near(got.lse[lo + r], lse.flatten(), 2 ** -6)
            lo += n
        w = weights[mats[3][0]:].view(hidden, hidden)
        want = got.out.double() @ w.double().T
        near(o, want, hidden * 2 ** -23 * (got.out.double().abs() @ w.double().abs().T) + 1e-30)


def test_tokens_one_by_one_as_a_prompt_at_once():
    """The same cache, bit for bit, and the same results within the roundings."""
    n, prefix = 70, 33
    one, all_ = (Case([n], [n], prefix=prefix, page=16, seed=1) for _ in range(2))
    q, k, v = (one.normal(n, h * 128) for h in (8, 2, 2))
    inv_freq = frequencies(128)
    qa = ops.kv_append(q, k, v, inv_freq, all_.cache, all_.batch)
    want = ops.prefix_attention(qa, all_.cache, all_.batch, need_lse=True)
    start = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    for i in range(n):
        batch = one.batch._replace(start=start, length=torch.tensor([i + 1], dtype=torch.int32, device="cuda"))
        qi = ops.kv_append(q[i:i + 1], k[i:i + 1], v[i:i + 1], inv_freq, one.cache, batch)
        assert torch.equal(qi[0], qa[i])
        got = ops.prefix_attention(qi, one.cache, batch, need_lse=True)
        # p's and the result's roundings on either side
        assert ((got.out[0].double() - want.out[i].double()).abs() <=
                2 ** -8 * 4 * v.abs().max()).all()
        assert (got.lse[0] - want.lse[i]).abs().max() <= 1e-4
    assert torch.equal(one.k[one.pages[0]].nan_to_num(), all_.k[all_.pages[0]].nan_to_num())
    assert torch.equal(one.v[one.pages[0]].nan_to_num(), all_.v[all_.pages[0]].nan_to_num())
