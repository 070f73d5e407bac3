"""What the paged cache's entry points refuse before anything is enqueued, and their
declarations (CPU only: addresses are numbers that nothing reads)."""
import ctypes
import os
import re

import pytest
import torch

from paper_2504_11651_amd import ops

from test_ops_host import A, INVALID, SMALL, UNSUPPORTED

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "df11_ops.h")
CACHE = dict(k=A, v=A, dtype=1, pages=10, heads=2, page_size=64, dim=128, k_stride=2 * 64 * 128,
             v_stride=2 * 64 * 128)
BATCH = dict(start=A, length=A, table=A, sequences=3, width=100, table_stride=100, prefix_table=A, prefix_pages=2,
             prefix_len=128)


class Cache(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("k", "v")] + [
        (n, ctypes.c_uint32) for n in ("dtype", "pages", "heads", "page_size", "dim")] + [
        (n, ctypes.c_uint64) for n in ("k_stride", "v_stride")]


class Batch(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("start", "length", "table")] + [
        ("sequences", ctypes.c_uint32), ("width", ctypes.c_uint32), ("table_stride", ctypes.c_uint64),
        ("prefix_table", ctypes.c_void_p), ("prefix_pages", ctypes.c_uint32), ("prefix_len", ctypes.c_uint32)]


def structs(change):
    """The two structs, and what of `change` is neither's."""
    rest = dict(change)
    cache = Cache(**{k: rest.pop(k, v) for k, v in CACHE.items()})
    batch = Batch(**{k: rest.pop(k, v) for k, v in BATCH.items()})
    return bytes(cache), bytes(batch), rest


def append(**change):
    cache, batch, change = structs(change)
    a = dict(q=2 * A, q_stride=1024, ak=2 * A, ak_stride=256, av=2 * A, av_stride=256, source=0, tokens=5, q_heads=8,
             inv_freq=A, rotary=128, interleaved=0, cache=cache, batch=batch, q_out=3 * A, out_stride=1024,
             stream=None)
    assert set(change) <= set(a)
    return ops.lib().df11_kv_append(*(a | change).values())


def attention(**change):
    cache, batch, change = structs(change)
    a = dict(q=2 * A, q_stride=1024, tokens=5, q_heads=8, scale=0.1, cache=cache, batch=batch, out=3 * A,
             out_stride=1024, lse=A, ws=A, ws_bytes=1 << 30, stream=None)
    assert set(change) <= set(a)
    return ops.lib().df11_prefix_attention(*(a | change).values())


NOTHING = dict(tokens=0)  # what is right with it launches nothing


@pytest.mark.parametrize("call", [append, attention])
@pytest.mark.parametrize("change, rc", [
    (dict(cache=None), INVALID), (dict(batch=None), INVALID),
    (dict(dtype=0), INVALID), (dict(dtype=3), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID),
    (dict(k=A + 8), INVALID), (dict(v=A + 2), INVALID), (dict(pages=0), INVALID), (dict(pages=2 ** 31), INVALID),
    (dict(heads=0), INVALID), (dict(page_size=8), INVALID), (dict(page_size=48), INVALID),
    (dict(page_size=2048), INVALID), (dict(page_size=0), INVALID), (dict(dim=32), INVALID),
    (dict(dim=96), INVALID), (dict(dim=256), INVALID), (dict(k_stride=2 * 64 * 128 - 8), INVALID),
    (dict(v_stride=2 * 64 * 128 + 4), INVALID), (dict(k_stride=1 << 41), INVALID),
    (dict(heads=1 << 20, page_size=1024, k_stride=1 << 38, v_stride=1 << 38), INVALID),
    (dict(start=None), INVALID), (dict(length=None), INVALID), (dict(table=None), INVALID),
    (dict(start=A + 2), INVALID), (dict(table_stride=99), INVALID), (dict(sequences=(1 << 24) + 1), INVALID),
    (dict(prefix_len=2 ** 31), INVALID), (dict(q=None), INVALID), (dict(q=A + 8), INVALID),
    (dict(q_stride=1023), INVALID), (dict(q_stride=1028 - 3), INVALID), (dict(q_stride=512), INVALID),
    (dict(out_stride=512), INVALID), (dict(out_stride=1028), INVALID), (dict(q_heads=0), INVALID),
    (dict(tokens=(1 << 24) + 1), INVALID), (dict(tokens=1 << 24, q_heads=1 << 10), INVALID),
    (dict(q_heads=1 << 21, tokens=1), INVALID), (NOTHING, 0), (dict(NOTHING, q=None), 0),
    (dict(sequences=0, start=None, length=None, table=None), 0), (dict(NOTHING, width=0, table=None), 0),
    (dict(NOTHING, sequences=1, table_stride=0), 0), (dict(NOTHING, pages=1, k_stride=0, v_stride=0), 0),
    (dict(NOTHING, page_size=16), 0), (dict(NOTHING, page_size=1024, k_stride=1 << 20, v_stride=1 << 20), 0),
])
def test_refusals_of_both(call, change, rc):
    assert call(**change) == rc


@pytest.mark.parametrize("change, rc", [
    (dict(source=3), INVALID), (dict(rotary=8), INVALID), (dict(rotary=144), INVALID), (dict(rotary=24), INVALID),
    (dict(inv_freq=None), INVALID), (dict(inv_freq=A + 2), INVALID), (dict(ak=None), INVALID),
    (dict(av=A + 4), INVALID), (dict(ak_stride=255), INVALID), (dict(av_stride=128), INVALID),
    (dict(q_out=None), INVALID), (dict(q_out=3 * A + 8), INVALID), (dict(q_out=2 * A), INVALID),
    (dict(q_out=2 * A, source=2), INVALID), (dict(tokens=1 << 24), UNSUPPORTED), (dict(q_out=2 * A, source=1, q_stride=2048), INVALID),
    (dict(NOTHING, inv_freq=None, rotary=0), 0), (dict(NOTHING, prefix_table=None), 0),
])
def test_append_refusals(change, rc):
    assert append(**change) == rc


@pytest.mark.parametrize("change, rc", [
    (dict(q_heads=7), INVALID), (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID),
    (dict(scale=1e-40), INVALID), (dict(NOTHING, scale=2.0 ** -126), 0),
    (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID), (dict(scale=3e38), INVALID),
    (dict(prefix_table=None), INVALID), (dict(prefix_table=A + 2), INVALID), (dict(prefix_len=129), INVALID),
    (dict(out=None), INVALID), (dict(out=2 * A, out_stride=2048), INVALID), (dict(lse=A + 2), INVALID),
    (dict(ws=None), INVALID), (dict(ws=A + 8), INVALID), (dict(ws_bytes=16), SMALL),
    (dict(tokens=1 << 23, sequences=1 << 22), UNSUPPORTED), (dict(sequences=1 << 23, width=1 << 16, table_stride=1 << 16), UNSUPPORTED),
    (dict(NOTHING, prefix_table=None, prefix_len=0), 0),
])
def test_attention_refusals(change, rc):
    assert attention(**change) == rc


def test_workspace_sizes():
    n = ctypes.c_uint64(77)

    def size(tokens, q_heads, into=ctypes.byref(n), **change):
        cache, batch, rest = structs(change)
        assert not rest
        return ops.lib().df11_prefix_attention_workspace_bytes(tokens, q_heads, cache, batch, into)

    assert size(0, 8) == 0 and n.value == 0
    assert size(5, 8) == 0 and n.value >= 2 * 5 * 8 * (128 * 4 + 8)  # the prefix' and the own tokens' results
    assert size(5, 8, k=None, start=None, table=None, prefix_table=None) == 0  # sizes alone count
    assert size(5, 8, into=None) == INVALID and size(5, 7) == INVALID and size(5, 8, dim=80) == INVALID
    assert size(4096, 32, heads=8, sequences=2) == 0 and n.value == 0  # enough rows to fill the GPU


def test_constants_and_structs_are_the_headers():
    header = open(HEADER).read()
    for name, value in (("DF11_MIN_PAGE", ops.MIN_PAGE), ("DF11_MAX_PAGE", ops.MAX_PAGE)):
        assert re.search(rf"#define {name} (\d+)", header).group(1) == str(value)
    for name, struct, packed in (("df11_kv_cache", Cache, ops._CACHE), ("df11_kv_batch", Batch, ops._BATCH)):
        body = re.findall(r"typedef struct \{([^}]*)\} " + name, header)[0]
        assert re.findall(r"\w+(?=\s*[,;])", body) == [f for f, _ in struct._fields_]
        values = range(1, len(struct._fields_) + 1)
        assert packed.pack(*values) == bytes(struct(*values))


def cpu_case():
    cache = ops.KVCache(torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16), torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16))
    i = torch.zeros(2, dtype=torch.int32)
    return cache, ops.KVBatch(i, i[:1], torch.zeros((1, 3), dtype=torch.int32))


def test_tensors_that_do_not_fit():
    cache, batch = cpu_case()
    q = torch.zeros((1, 256), dtype=torch.bfloat16)
    for call in (lambda: ops.prefix_attention(q, cache, batch),
                 lambda: ops.kv_append(q, q[:, :128], q[:, :128], None, cache, batch)):
        with pytest.raises(ValueError, match="must be on a GPU"):
            call()
    def sizes(cache):
        return ops._cache_sizes(ops._look(cache.k), ops._look(cache.v), -1)

    def batch_sizes(**change):
        return ops._batch_sizes(*map(ops._look, batch._replace(**change)[:4]), -1)

    assert sizes(cache) == (1, 4, 2, 16, 64, 2048, 2048) and batch_sizes() == ((1, 3, 3), 0)
    k = cache.k
    for bad in (k.float(), k[0], k.transpose(1, 2), k[..., :32]):
        with pytest.raises(ValueError):
            sizes(ops.KVCache(bad, bad))
    for bad in (k[:3], k.half(), k.transpose(2, 3)):
        with pytest.raises(ValueError, match="cache.v"):
            sizes(ops.KVCache(k, bad))
    for change in (dict(start=batch.start[:1]), dict(start=batch.start.long()), dict(length=batch.length[0]),
                   dict(start=torch.zeros(4, dtype=torch.int32)[::2]), dict(table=batch.table[0]),
                   dict(table=batch.table.long()), dict(table=torch.zeros((2, 3)).int()),
                   dict(table=batch.table.T), dict(prefix_table=batch.table.long()[0]),
                   dict(prefix_table=batch.table)):
        with pytest.raises(ValueError):
            batch_sizes(**change)
    for length in (-1, 2 ** 31):
        with pytest.raises(ValueError, match="prefix_len"):
            ops._pack(cache, batch._replace(prefix_len=length), (1, 4, 2, 16, 64, 2048, 2048), (1, 3, 3), 0)
    with pytest.raises(ValueError, match="heads of 64"):
        ops._heads(100, 64, "q")


def test_another_gpu_than_the_current_one_is_refused(monkeypatch):
    class Elsewhere:
        device = "cuda:1"

        def get_device(self):
            return 1

    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    with pytest.raises(ValueError, match="current GPU, not cuda:1"):
        ops._on_gpu(Elsewhere(), "q")
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1, raising=False)
    assert ops._on_gpu(Elsewhere(), "q") == 1


def sizes_of(**change):
    """What kv_append makes of CPU tensors that would fit but for `change`."""
    cache, batch = cpu_case()
    q = torch.zeros((1, 256))
    a = dict(index=-1, q=q, k=q[:, :128], v=q[:, :128], inv_freq=torch.zeros(32), q_out=None, cache_k=cache.k,
             cache_v=cache.v, start=batch.start, length=batch.length, table=batch.table, prefix_table=None)
    a = a | change
    return ops._append_sizes(a.pop("index"), *map(ops._look, a.values()))


def test_rows_that_do_not_fit():
    q = torch.zeros((4, 256))
    assert sizes_of()[3:] == (256, 128, 128, 0, 1, 4, 64, 256)
    assert sizes_of(q=q[:1], k=q[:1, :128], v=q[:1, 128:], q_out=q[:1].half().bfloat16())[3:] == (
        256, 128, 128, 0, 1, 4, 64, 256)
    for change in (dict(q=q[0]), dict(q=q[:1, :100]), dict(q=q.T), dict(q=q[:1].double()), dict(k=q[:2, :128]),
                   dict(k=q[:1, :64]), dict(v=q[:1, :128].half()), dict(v=q[:1, ::2]), dict(inv_freq=q[0].double()),
                   dict(inv_freq=q[:2]), dict(q_out=q[:1]), dict(q_out=q[:1, :128].bfloat16()), dict(index=0)):
        with pytest.raises(ValueError):
            sizes_of(**change)
