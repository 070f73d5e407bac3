"""Attention to a shared prefix and to each sequence's own tokens over a paged cache,
against its definition in 64 bits."""
import math
import random

import pytest
import torch

from paper_2504_11651_amd import ops

from conftest import gpu_available
from kv_reference import BF16, F16, Case, near

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs an MI355X")]


@pytest.fixture(autouse=True, params=[0, 100], ids=["short tables", "long tables"])
def both_plans(request, monkeypatch):
    """Few pages are read by one workgroup; where the tables have room for many, the work
    is cut into shares and joined."""
    monkeypatch.setattr(Case, "spare_pages", request.param)


@pytest.mark.parametrize("dtype, dim", [(BF16, 128), (BF16, 64), (F16, 128), (F16, 64)])
@pytest.mark.parametrize("own", [1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 191, 193, 257])
def test_one_token_of_one_sequence(own, dtype, dim):
    Case([1], [own], dim=dim, dtype=dtype, seed=own).check()


@pytest.mark.parametrize("dtype, dim", [(BF16, 128), (F16, 64)])
@pytest.mark.parametrize("prefix", [1, 16, 63, 64, 65, 128, 255, 256, 257, 320, 1000, 5001])
def test_prefix_of_any_length(prefix, dtype, dim):
    Case([1, 1, 1], [1, 40, 300], prefix=prefix, dim=dim, dtype=dtype, seed=prefix).check()


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256, 512, 1024])
def test_page_sizes(page):
    Case([2, 1, 5], [2, 333, 77], prefix=page + 5, page=page, seed=page).check()


@pytest.mark.parametrize("heads, kv_heads", [(1, 1), (3, 3), (3, 1), (7, 1), (12, 4), (28, 4), (40, 8), (33, 11),
                                             (64, 8), (64, 1), (66, 1), (142, 2), (200, 1), (16, 16)])
def test_head_layouts(heads, kv_heads):
    Case([1, 3, 2, 1], [70, 3, 200, 1], prefix=150, heads=heads, kv_heads=kv_heads, seed=heads).check()
    Case([1] * 40, [1 + 7 * i for i in range(40)], prefix=70, heads=heads, kv_heads=kv_heads, dim=64, dtype=F16,
         seed=heads).check()


@pytest.mark.parametrize("new, own", [
    ([64], [64]), ([65], [65]), ([33], [200]), ([31, 32, 33], [31, 64, 99]), ([128, 1, 129], [128, 1, 129]),
    ([100, 3, 1, 57], [400, 3, 1000, 57]), ([17], [4000]),
])
@pytest.mark.parametrize("prefix", [0, 99])
@pytest.mark.parametrize("dtype, dim", [(BF16, 128), (F16, 64)])
def test_several_rows_see_up_to_themselves(new, own, prefix, dtype, dim):
    Case(new, own, prefix=prefix, dim=dim, dtype=dtype, page=16, seed=len(own)).check()


@pytest.mark.parametrize("new, own, prefix, heads, kv_heads, dim, dtype", [
    ([1100], [1100], 0, 32, 8, 128, BF16), ([700, 1, 0, 500], [700, 900, 0, 777], 333, 32, 8, 128, BF16),
    ([2500, 40], [2600, 40], 65, 16, 8, 64, F16), ([513, 600, 1027], [513, 600, 1027], 64, 16, 16, 64, BF16),
    ([3001], [3001], 1, 12, 4, 128, F16), ([1500, 2600], [1500, 2600], 0, 10, 1, 128, BF16),
])
def test_prompts_that_fill_the_gpu(new, own, prefix, heads, kv_heads, dim, dtype):
    """Rows read the prefix and their own tokens in one go, without a workspace."""
    c = Case(new, own, prefix=prefix, heads=heads, kv_heads=kv_heads, dim=dim, dtype=dtype, seed=len(new), spare=3)
    c.check()


def test_prompts_take_no_workspace_where_they_fill_the_gpu():
    c = Case([1100], [1100], prefix=10, heads=32, kv_heads=8)
    assert ops.prefix_attention_workspace_bytes(1100, 32, c.cache, c.batch) == 0
    assert ops.prefix_attention_workspace_bytes(10, 32, c.cache, c.batch) > 0


@pytest.mark.parametrize("spare", [0, 1, 200])
def test_sequences_without_rows_and_rows_without_sequence(spare):
    Case([0, 2, 0, 0, 1, 0], [5, 2, 0, 70, 300, 9], prefix=65, spare=spare, seed=spare).check()
    Case([0, 0], [5, 2], prefix=65, spare=2 + spare).attend()  # no row at all


@pytest.mark.parametrize("sequences", [63, 64, 65, 129, 300, 4097])
def test_many_sequences(sequences):
    own = [1 + (37 * i) % 90 for i in range(sequences)]
    # in a long batch few have rows: the reference takes them one by one
    new = [min(x, (i * 7) % 3) if sequences < 200 or i % 41 == 0 or i > sequences - 9 else 0 for i, x in enumerate(own)]
    Case(new, own, prefix=130, heads=2, kv_heads=1, dim=64, page=16, seed=sequences, spare=2).check()


@pytest.mark.parametrize("prefix", [0, 40])
def test_rows_that_see_nothing(prefix):
    """Places below 0: the prefix alone, and where there is none a result of 0."""
    c = Case([5, 1, 3, 1], [2, 0, -4, 1], prefix=prefix, seed=prefix)
    got = c.check()
    if not prefix:
        for r in (0, 1, 2, 5, 6, 7, 8):
            assert (got.out[r] == 0).all() and (got.lse[r] == -math.inf).all()


def test_no_sequences_and_no_rows():
    c = Case([1], [1])
    none = ops.KVBatch(c.start[:1], c.length[:0], c.table[:0])
    out = torch.full_like(c.q, 77.0)
    ops.prefix_attention(c.q, c.cache, none, out=out)
    assert (out == 77.0).all()
    assert ops.prefix_attention(c.q[:0], c.cache, c.batch, need_lse=True).lse.shape == (0, 8)


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("new, own, prefix, heads, kv_heads", [
    ([70, 3], [70, 40], 20, 8, 2), ([1200, 1], [1200, 3], 0, 32, 8)])
@pytest.mark.parametrize("dtype, dim", [(BF16, 128), (F16, 64)])
def test_later_tokens_have_no_effect(value, new, own, prefix, heads, kv_heads, dtype, dim):
    """Keys and values of tokens behind a row's place, in its own tile too."""
    at = [(0, own[0] - 13), (0, own[0] - 2), (1, own[1] - 1)]
    c = Case(new, own, prefix=prefix, heads=heads, kv_heads=kv_heads, dim=dim, dtype=dtype, seed=3)
    clean = c.attend()
    for s, i in at:
        for cache in (c.k, c.v):
            cache[c.pages[s][i // c.page], :, i % c.page, ::3] = value
    got = c.attend()
    lo = 0
    for s, n in enumerate(new):
        first = min(i for q, i in at if q == s)
        before = lo + max(0, first - (own[s] - n))
        assert torch.equal(got.out[lo:before], clean.out[lo:before])
        assert torch.equal(got.lse[lo:before], clean.lse[lo:before])
        if value != value:
            assert got.out[before:lo + n].isnan().all() and got.lse[before:lo + n].isnan().all()
        lo += n


@pytest.mark.parametrize("dtype, dim", [(BF16, 128), (BF16, 64), (F16, 128), (F16, 64)])
@pytest.mark.parametrize("new, own", [([20, 90], [20, 90]), ([33], [200]), ([1024], [1024])])
def test_values_that_are_not_finite(new, own, dtype, dim):
    """Rows that see an infinity or a NaN among the values have it in that place of
    the result alone; the others have what they had."""
    c = Case(new, own, heads=32, kv_heads=8, dim=dim, dtype=dtype, seed=4)
    clean = c.check()
    s, lo = len(new) - 1, sum(new[:-1])
    n, length = new[s], own[s]
    marks = {length - 5: (3, math.inf), length - 3: (40, -math.inf), length - 2: (5, math.nan),
             length - 1: (3, -math.inf), length - 17: (8, -math.inf)}
    for i, (d, value) in marks.items():
        c.v[c.pages[s][i // c.page], 1, i % c.page, d] = value
    got = c.attend()
    want = clean.out.view(-1, 32, dim).clone()
    row = torch.arange(length - n, length, device="cuda")
    for d in {d for d, _ in marks.values()}:
        total = torch.zeros(n, device="cuda")
        for i, (e, value) in marks.items():
            if d == e:
                total += torch.where(row >= i, value, 0.0)
        hit = ~(total == 0)
        want[lo:, 4:8, d] = torch.where(hit[:, None], total[:, None].to(dtype), want[lo:, 4:8, d])
    got_out = got.out.view(-1, 32, dim)
    assert torch.equal(got_out.isnan(), want.isnan())
    assert torch.equal(got_out[~want.isnan()], want[~want.isnan()])
    assert torch.equal(got.lse, clean.lse)


def test_scores_that_are_not_finite():
    """An infinity among the scores: as the formula has it (inf - inf)."""
    c = Case([1, 1], [70, 90], prefix=30, seed=5)
    c.q[:] = c.q.abs()
    c.k[c.pages[0][0], 0, 5] = math.inf   # rows of sequence 0, heads 0..3
    c.k[c.pages[1][0], 1, 6] = -math.inf  # sequence 1, heads 4..7: as if it were not there
    got = c.attend()
    assert got.out[0, :4 * 128].isnan().all() and got.lse[0, :4].isnan().all()
    assert got.out[0, 4 * 128:].isfinite().all() and got.out[1].isfinite().all()
    # all scores of a row -inf: nothing seen
    one = Case([1], [3], seed=6)
    one.q[:] = one.q.abs()
    one.k[one.pages[0][0], :, :3] = -math.inf
    got = one.attend()
    assert (got.out == 0).all() and (got.lse == -math.inf).all()


@pytest.mark.parametrize("new, own, prefix, heads, kv_heads, page", [
    ([3, 2, 1], [200, 300, 1], 130, 8, 2, 64), ([3, 2, 1], [200, 300, 1], 130, 8, 2, 16),
    ([700, 500], [700, 500], 100, 32, 8, 32)])
@pytest.mark.parametrize("wrong", [-1, 10 ** 6, 2 ** 31 - 1, -2 ** 31])
def test_pages_outside_the_cache(new, own, prefix, heads, kv_heads, page, wrong):
    """Rows that see one have no result, the others all of theirs."""
    c = Case(new, own, prefix=prefix, heads=heads, kv_heads=kv_heads, page=page, seed=7)
    clean = c.attend()
    hurt = 2 if page < 64 else 1
    c.table[0, hurt] = wrong
    got = c.attend()
    place = torch.arange(own[0] - new[0], own[0], device="cuda")
    seen = place >= hurt * page
    assert got.out[:new[0]][seen].isnan().all() and got.lse[:new[0]][seen].isnan().all()
    assert torch.equal(got.out[:new[0]][~seen], clean.out[:new[0]][~seen])
    assert torch.equal(got.out[new[0]:], clean.out[new[0]:]) and torch.equal(got.lse[new[0]:], clean.lse[new[0]:])
    c.prefix_table[0] = wrong
    got = c.attend()
    assert got.out.isnan().all() and got.lse.isnan().all()


@pytest.mark.parametrize("hurt", [0, 1, 2, 3, 4, 5, 6])
def test_pages_outside_the_cache_among_rows_of_a_tile(hurt):
    """One head, so that a hundred rows share their tiles: those in front of the page have
    all of their result."""
    c = Case([100, 7], [100, 107], heads=2, kv_heads=2, page=16, seed=hurt)
    clean = c.attend()
    c.table[0, hurt] = -1
    got = c.attend()
    for name in ("out", "lse"):
        a, b = getattr(got, name), getattr(clean, name)
        assert torch.equal(a[:16 * hurt], b[:16 * hurt]) and a[16 * hurt:100].isnan().all(), name
        assert torch.equal(a[100:], b[100:]), name


def test_places_past_the_tables_width():
    c = Case([4, 1], [130, 20], prefix=10, page=16, width=8, seed=8)
    got = c.attend()
    want = c.expected()
    near(got.out[:2], want["out"][0][:2], want["out"][1][:2])  # 126 and 127 are on the eighth page
    assert got.out[2:4].isnan().all() and got.lse[2:4].isnan().all()
    near(got.out[4:], want["out"][0][4:], want["out"][1][4:])
    c.length[1] = 2 ** 31 - 1
    c.table[1, 1:] = c.table[1, 0]
    assert c.attend().out[4].isnan().all()


@pytest.mark.parametrize("scale", [1e-6, 0.01, 1.0, 30.0])
def test_scales(scale):
    """From the mean of all values to the value of the largest score."""
    Case([2, 1, 40], [200, 300, 40], prefix=130, seed=9).check(scale=scale)


def test_scores_that_rise_and_fall():
    """Bounds that rise all the way, by much and by little, and a first token that
    outweighs all others."""
    for slope in (0.02, 0.5, -0.5, 8.0, -8.0):
        c = Case([1, 30], [700, 700], prefix=500, seed=10)
        c.q[:] = 0
        c.q[:, ::128] = 1  # a head's first value
        for b, kv in enumerate(c.sets):
            steps = torch.arange(kv[0].shape[0], device="cuda") * slope
            kv[0][:, :, 0] = steps[:, None].to(c.dtype)
        rewrite(c)
        c.check(scale=1.0)


def rewrite(c):
    """The sets, changed, to their pages."""
    for pages, kv in zip([c.prefix_table.long(), *c.pages], c.sets):
        i = torch.arange(kv[0].shape[0], device="cuda")
        if i.numel():
            c.k[pages[i // c.page], :, i % c.page] = kv[0]
            c.v[pages[i // c.page], :, i % c.page] = kv[1]


def test_equal_scores_give_the_mean_of_whole_numbers():
    """Scores of 0 and values that are whole: the sums have no rounding but the last."""
    c = Case([1, 64], [128, 256], seed=11)
    c.q[:] = 0
    for kv in c.sets:
        kv[1][:] = torch.randint(-8, 9, kv[1].shape, generator=c.g, device="cuda").to(c.dtype)
    rewrite(c)
    got = c.attend()
    mean = c.sets[1][1].double().mean(0).to(c.dtype).repeat_interleave(4, 0).flatten()
    assert torch.equal(got.out[0], mean)
    assert (got.lse[0] - math.log(128)).abs().max() <= 2 ** -21


def test_strides():
    """q and out in wider tensors, k and v side by side in one, a table's first columns."""
    c = Case([3, 1, 40], [100, 200, 40], prefix=77, seed=12)
    want = c.attend()
    wide = torch.zeros((44, 4 * 1024), dtype=BF16, device="cuda")
    wide[:, 1024:2048] = c.q
    both = torch.stack((c.k, c.v), 1)
    table = torch.full((3, c.table.shape[1] + 5), 10 ** 8, dtype=torch.int32, device="cuda")
    table[:, :c.table.shape[1]] = c.table
    batch = c.batch._replace(table=table[:, :c.table.shape[1]])
    got = ops.prefix_attention(wide[:, 1024:2048], ops.KVCache(both[:, 0], both[:, 1]), batch, out=wide[:, 2048:-1024])
    assert torch.equal(wide[:, 2048:-1024], want.out) and torch.equal(wide[:, 1024:2048], c.q) and got.lse is None
    assert (wide[:, :1024] == 0).all()


@pytest.mark.parametrize("new, own", [([3, 1], [100, 200]), ([1100], [1100])])
def test_in_place(new, own):
    c = Case(new, own, prefix=70, heads=32, kv_heads=8, seed=13, spare=1)
    want, q = c.attend(), c.q.clone()
    ops.prefix_attention(c.q, c.cache, c.batch, out=c.q)
    rows = sum(new)
    assert torch.equal(c.q[:rows], want.out[:rows]) and torch.equal(c.q[rows:], q[rows:])


def test_pages_that_sequences_share():
    """A sequence forked from another: the same pages in two tables, and the prefix' pages
    in a table of their own, each as if it had a copy."""
    c = Case([2, 2, 1], [300, 300, 90], prefix=130, seed=17)
    c.table[1] = c.table[0]
    c.pages[1], c.sets[2] = c.pages[0], c.sets[1]
    c.table[2, :2] = c.prefix_table[:2]
    c.sets[3] = [x[:90] for x in c.sets[0]]
    c.check()


def test_far_pages():
    """Pages whose offsets pass 2^32 elements."""
    page, stride = 64, 1 << 31
    c = Case([2, 1], [100, 30], prefix=70, seed=14, heads=4, kv_heads=2)
    pages = c.k.shape[0]
    each = 2 * page * 128
    want = c.attend()
    room = torch.empty((pages - 1) * stride + 2 * each, dtype=BF16, device="cuda")
    k = room.as_strided(c.k.shape, (stride, page * 128, 128, 1))
    v = room.as_strided(c.v.shape, (stride, page * 128, 128, 1), each)
    k.copy_(c.k), v.copy_(c.v)
    got = ops.prefix_attention(c.q, ops.KVCache(k, v), c.batch, need_lse=True)
    assert torch.equal(got.out, want.out) and torch.equal(got.lse, want.lse)


@pytest.mark.parametrize("seed", range(60))
def test_random_batches(seed):
    """Sizes, layouts and lengths of all kinds together."""
    rng = random.Random(seed)
    group = rng.choice([1, 2, 3, 4, 5, 8, 13, 40])
    kv_heads = rng.choice([1, 2, 3, 4, 8])
    page = rng.choice([16, 32, 64, 128, 512])
    new, own = [], []
    for _ in range(rng.choice([1, 2, 3, 10, 40, 70])):
        new.append(rng.choice([0, 1, 1, 1, 2, 5, rng.randint(1, 90)]))
        own.append(new[-1] + rng.choice([0, 0, 1, rng.randint(0, 70), rng.randint(0, 900)]) - (rng.random() < 0.1) * 3)
    c = Case(new, own, prefix=rng.choice([0, 0, 1, rng.randint(1, 200), rng.randint(1, 3000)]), heads=group * kv_heads,
             kv_heads=kv_heads, dim=rng.choice([64, 128]), page=page, dtype=rng.choice([BF16, F16]), seed=seed,
             spare=rng.choice([0, 1, 20]))
    if sum(new):
        c.check(scale=rng.choice([None, 0.02, 0.5]))


def test_the_same_bits_every_time():
    for new, own, heads, kv in (([1] * 20, range(1, 2001, 100), 8, 2), ([1100], [1100], 32, 8)):
        c = Case(new, own, prefix=3001, heads=heads, kv_heads=kv, seed=15)
        first = c.attend()
        for _ in range(5):
            again = c.attend()
            assert torch.equal(again.out, first.out) and torch.equal(again.lse, first.lse)


def test_two_streams_at_once():
    """Two batches under way together, with a workspace each."""
    cases = [Case([1, 2, 1], [900, 200, 3000], prefix=900 + i, seed=18 + i) for i in range(2)]
    want = [c.attend() for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for i, c in enumerate(cases):
            got[i].append(ops.prefix_attention(c.q, c.cache, c.batch, need_lse=True, stream=streams[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for x in got[i]:
            assert torch.equal(x.out, want[i].out) and torch.equal(x.lse, want[i].lse)


def test_a_workspace_given_and_on_a_stream():
    c = Case([1, 2, 1], [100, 200, 3000], prefix=900, seed=16)
    want = c.attend()
    need = ops.prefix_attention_workspace_bytes(4, 8, c.cache, c.batch)
    ws = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    got = c.attend(workspace=ws[:need])
    assert torch.equal(got.out, want.out) and (ws[need:] == 0xFF).all()
    with pytest.raises(ops.codec.DF11Error):
        c.attend(workspace=ws[:need - 16])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = ops.prefix_attention(c.q, c.cache, c.batch, need_lse=True, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got.out, want.out) and torch.equal(got.lse, want.lse)


def test_a_captured_call_follows_the_batch():
    """Lengths, tables, rows and sequences change between replays, up to the capture's
    sizes."""
    cases = [Case(new, own, prefix=200, width=12, seed=20 + i, spare=8 - sum(new))
             for i, (new, own) in enumerate((([1] * 4, [5, 700, 64, 1]), ([2, 0, 1, 5], [130, 9, 65, 500]),
                                             ([0, 0, 0, 0], [3, 3, 3, 3]), ([1, 1, 6, 0], [768, 1, 6, 0])))]
    most = max(c.k.shape[0] for c in cases)
    fixed = Case([1] * 4, [1] * 4, prefix=200, width=12, spare=4)
    k, v = (torch.zeros((most, *fixed.k.shape[1:]), dtype=BF16, device="cuda") for _ in range(2))
    batch = ops.KVBatch(fixed.start, fixed.length, fixed.table, fixed.prefix_table, 200)
    q, out = torch.zeros_like(fixed.q), torch.zeros_like(fixed.q)
    lse = torch.zeros((8, 8), device="cuda")
    cache = ops.KVCache(k, v)
    ws = torch.empty(ops.prefix_attention_workspace_bytes(8, 8, cache, batch), dtype=torch.uint8, device="cuda")
    fixed.start.zero_()
    ops.prefix_attention(q, cache, batch, out=out, lse=lse, workspace=ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ops.prefix_attention(q, cache, batch, out=out, lse=lse, workspace=ws)
    for c in cases + cases[::-1]:
        k[:c.k.shape[0]], v[:c.k.shape[0]] = c.k, c.v
        for name in ("start", "length", "table", "prefix_table"):
            getattr(batch, name).copy_(getattr(c, name))
        q.copy_(c.q), out.fill_(77.0), lse.fill_(77.0), ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        want = c.attend()
        assert torch.equal(out, want.out) and torch.equal(lse, want.lse)
        if sum(c.new):
            c.check(ops.Attention(out, lse))
