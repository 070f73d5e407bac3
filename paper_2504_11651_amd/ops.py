"""Thin ctypes binding of the operators around a frozen, compressed model (the
C ABI declared in include/df11_ops.h): low-rank adapters beside a shared
projection, log probabilities of given tokens with rank, entropy and top
alternatives, distillation from a teacher's top log probabilities, and the
gradients of all three; and, between a block's products, a paged cache of keys
and values, appended to with the position rotation and read by attention to a
prefix that the batch shares and to each sequence's own tokens.

Argument marshalling only, as in ``codec``: every value is computed by the
library's HIP kernels, on ``stream`` (default: torch's current stream), and a
call returns without waiting.  Outputs and workspaces that are not given are
allocated by torch, in ``stream``'s memory; tensors that are given are the
caller's to keep, and to have ready on ``stream``.  A workspace holds nothing
between calls, so calls that overlap in time need one each.  ValueError for
tensors that do not fit each other, ``codec.DF11Error`` for what the library
refuses.  As for ``codec``'s calls, the tensors' GPU is to be the current one.

The calls know nothing of autograd: results are detached also where an input
requires a gradient, and a tensor that is filled or replaced is written
without its version being counted.  A program that differentiates through them
calls the ``_backward`` functions from its own ``torch.autograd.Function``.
"""
from __future__ import annotations

import ctypes
import functools
import struct
from typing import NamedTuple, Optional

import torch

from . import codec

# every function include/df11_ops.h declares
EXPORTS = (
    "df11_logprobs_workspace_bytes", "df11_logprobs", "df11_logprobs_backward",
    "df11_distill_workspace_bytes", "df11_distill", "df11_distill_backward",
    "df11_lora_workspace_bytes", "df11_lora", "df11_lora_backward_workspace_bytes",
    "df11_lora_backward", "df11_kv_append", "df11_prefix_attention_workspace_bytes",
    "df11_prefix_attention",
)

MAX_TOP = 128   # DF11_MAX_TOP
MAX_RANK = 128  # DF11_MAX_RANK
MIN_PAGE, MAX_PAGE = 16, 1024  # DF11_MIN_PAGE, DF11_MAX_PAGE
DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}

_lib = None


# df11_kv_cache: k, v, dtype, pages, heads, page_size, dim, k_stride, v_stride;
# df11_kv_batch: start, length, table, sequences, width, table_stride, prefix_table,
# prefix_pages, prefix_len
_CACHE, _BATCH = struct.Struct("@QQIIIIIQQ"), struct.Struct("@QQQIIQQII")


def lib():
    """libdf11.so with the signatures of include/df11_ops.h."""
    global _lib
    if _lib is None:
        L = codec.lib()
        vp, u32, u64, f32 = ctypes.c_void_p, ctypes.c_uint32, ctypes.c_uint64, ctypes.c_float
        size = ctypes.POINTER(u64)
        logits = [vp, u32, u64, u32, u64]
        shapes = [u64, u32, u32, u32, u32]
        adapters = [vp, u64, *shapes, vp, vp, vp, vp]
        sig = {
            "df11_logprobs_workspace_bytes": [u32, u64, u32, u32, size],
            "df11_logprobs": [*logits, vp, u32, f32, vp, vp, vp, vp, vp, vp, vp, u64, vp],
            "df11_logprobs_backward": [*logits, vp, vp, vp, vp, f32, vp, u64, vp],
            "df11_distill_workspace_bytes": [u32, u64, u32, size],
            "df11_distill": [*logits, vp, vp, u32, u32, f32, vp, vp, vp, vp, u64, vp, u64, vp],
            "df11_distill_backward": [*logits, vp, vp, u32, u32, f32, vp, vp, vp, u64, vp],
            "df11_lora_workspace_bytes": [*shapes, size],
            "df11_lora": [*adapters, vp, u64, vp, u64, u32, vp, u64, vp],
            "df11_lora_backward_workspace_bytes": [*shapes, size],
            "df11_lora_backward": [*adapters, vp, u64, u32, vp, u64, vp, u64, vp, vp, vp, u64, vp],
        }
        sig |= {
            "df11_kv_append": [vp, u64, vp, u64, vp, u64, u32, u64, u32, vp, u32, u32, vp, vp, vp,
                               u64, vp],
            "df11_prefix_attention_workspace_bytes": [u64, u32, vp, vp, size],
            "df11_prefix_attention": [vp, u64, u64, u32, f32, vp, vp, vp, u64, vp, vp, u64, vp],
        }
        for name, args in sig.items():
            fn = getattr(L, name)
            fn.argtypes = args
            fn.restype = ctypes.c_int
        _lib = L
    return _lib


class Logprobs(NamedTuple):
    """What ``logprobs`` gives, one row per row of the logits."""
    logprob: Optional[torch.Tensor]  # float32 (rows,), None without tokens
    rank: Optional[torch.Tensor]     # int64 (rows,), None without tokens
    entropy: torch.Tensor            # float32 (rows,)
    top_logprob: torch.Tensor        # float32 (rows, top)
    top_index: torch.Tensor          # int64 (rows, top)
    stats: torch.Tensor              # float32 (rows, 4), for the backward pass


class Distill(NamedTuple):
    """What ``distill`` gives, one row per row of the logits."""
    loss: torch.Tensor            # float32 (rows,)
    stats: torch.Tensor           # float32 (rows, 4), for the backward pass
    grad: Optional[torch.Tensor]  # as the logits, None where none was asked for


class LoraGrads(NamedTuple):
    dx: Optional[torch.Tensor]  # bfloat16 (tokens, cols)
    da: Optional[torch.Tensor]  # float32 (adapters, rank, cols)
    db: Optional[torch.Tensor]  # float32 (adapters, rows, rank)


class KVCache(NamedTuple):
    """A paged cache: page p holds page_size tokens of every head.  Any stride
    between pages (layers or k and v side by side), each page contiguous."""
    k: torch.Tensor  # bfloat16 or float16 (pages, kv_heads, page_size, head_dim)
    v: torch.Tensor  # as k


class KVBatch(NamedTuple):
    """The sequences that a call works on, and where their tokens lie."""
    start: torch.Tensor   # int32 (sequences + 1,): first row of each, ascending from 0, and the end
    length: torch.Tensor  # int32 (sequences,): own tokens of each, with the call's rows, its last
    table: torch.Tensor   # int32 (sequences, width): pages of each sequence's own tokens
    prefix_table: Optional[torch.Tensor] = None  # int32 (n,): pages of the shared prefix
    prefix_len: int = 0                          # its tokens


class Attention(NamedTuple):
    """What ``prefix_attention`` gives."""
    out: torch.Tensor            # as q
    lse: Optional[torch.Tensor]  # float32 (tokens, heads), None where none was asked for


def _ptr(t):
    return None if t is None else t.data_ptr()


def _want(t, shape, dtype, device, what):
    """A contiguous tensor of this shape and type on this GPU; None passes."""
    if t is not None and (t.shape != shape or t.dtype != dtype or t.device != device or
                          not t.is_contiguous()):
        raise ValueError(f"{what} must be a contiguous {dtype} tensor of shape {tuple(shape)} on "
                         f"{device}, not {t.dtype} {tuple(t.shape)} on {t.device}")


def _rows(t, dtypes, device, what, shape=None):
    """The row stride of a 2-d tensor on this GPU whose rows are contiguous."""
    if t.dim() != 2 or t.dtype not in dtypes or t.device != device or (
            shape is not None and t.shape != shape):
        raise ValueError(f"{what} must be a 2-d tensor of {' or '.join(map(str, dtypes))}"
                         f"{'' if shape is None else ' and shape ' + str(tuple(shape))} on "
                         f"{device}, not {t.dtype} {tuple(t.shape)} on {t.device}")
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise ValueError(f"{what} must have contiguous rows")
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _gpu(t, what):
    if t.device.type != "cuda":
        raise ValueError(f"{what} must be on a GPU, not {t.device}")
    return t.device


def _new(shape, dtype, device, stream):
    """A tensor that the kernels on ``stream`` write: of that stream's memory, so
    that nothing the current stream still does with memory it gave back meets
    them, nor they what it allocates when the tensor is dropped early."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    if not hasattr(stream, "cuda_stream"):
        stream = torch.cuda.ExternalStream(int(stream), device=device)
    here = torch.cuda.current_stream(device)
    with torch.cuda.stream(stream):
        t = torch.empty(shape, dtype=dtype, device=device)
    if stream.cuda_stream != here.cuda_stream:
        t.record_stream(here)  # which reads it later, and may when it is dropped
    return t


@functools.lru_cache(maxsize=1024)
def _bytes(size, *sizes):
    """What the library's size function says for these sizes."""
    n = ctypes.c_uint64()
    codec._check(getattr(lib(), size)(*sizes, ctypes.byref(n)), size)
    return int(n.value)


def _workspace(given, size, sizes, device, stream):
    """(tensor, bytes): the given workspace or one of the size the library asks for."""
    if given is not None:
        codec._on_device(given, device, "workspace")
        if not given.is_contiguous():
            raise ValueError("workspace must be contiguous")
        return given, given.numel() * given.element_size()
    n = _bytes(size, *sizes)
    return (_new((n,), torch.uint8, device, stream), n) if n else (None, 0)


def _handle(stream, device):
    """codec._handle without making a Stream object for torch's current stream,
    which costs as much as a launch."""
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(device.index)
    return codec._handle(stream, device)


# ----------------------------------------------------------- log probabilities
def logprobs_workspace_bytes(dtype, rows: int, vocab: int, top: int = 0) -> int:
    return _bytes("df11_logprobs_workspace_bytes", DTYPES[dtype], rows, vocab, top)


def logprobs(logits, tokens=None, top: int = 0, temperature: float = 1.0, out=None, workspace=None,
             stream=None) -> Logprobs:
    """Log probability and rank of ``tokens`` (int64, one per row; negative:
    none asked), entropy and the ``top`` best alternatives of each row of
    ``logits`` (2-d float32, bfloat16 or float16 with contiguous rows) at
    ``temperature``.  ``out``: a Logprobs, or a tuple in its order, to fill."""
    device = _gpu(logits, "logits")
    stride = _rows(logits, DTYPES, device, "logits")
    rows, vocab = logits.shape
    _want(tokens, (rows,), torch.int64, device, "tokens")
    if out is None:
        def new(*shape, dtype=torch.float32):
            return _new(shape, dtype, device, stream)
        asked = tokens is not None
        out = Logprobs(new(rows) if asked else None,
                       new(rows, dtype=torch.int64) if asked else None, new(rows), new(rows, top),
                       new(rows, top, dtype=torch.int64), new(rows, 4))
    else:
        out = Logprobs(*out)
        _want(out.logprob, (rows,), torch.float32, device, "out.logprob")
        _want(out.rank, (rows,), torch.int64, device, "out.rank")
        _want(out.entropy, (rows,), torch.float32, device, "out.entropy")
        _want(out.top_logprob, (rows, top), torch.float32, device, "out.top_logprob")
        _want(out.top_index, (rows, top), torch.int64, device, "out.top_index")
        _want(out.stats, (rows, 4), torch.float32, device, "out.stats")
    dt = DTYPES[logits.dtype]
    ws, ws_bytes = _workspace(workspace, "df11_logprobs_workspace_bytes", (dt, rows, vocab, top),
                              device, stream)
    codec._check(lib().df11_logprobs(
        logits.data_ptr(), dt, rows, vocab, stride, _ptr(tokens), top, temperature,
        _ptr(out.logprob), _ptr(out.rank), _ptr(out.entropy), _ptr(out.top_logprob),
        _ptr(out.top_index), _ptr(out.stats), _ptr(ws), ws_bytes, _handle(stream, device)),
        "df11_logprobs")
    return out


def logprobs_backward(logits, tokens, stats, grad_logprob=None, grad_entropy=None,
                      temperature: float = 1.0, out=None, stream=None):
    """The gradient of ``logits`` (its type) from the gradients of ``logprob``
    and ``entropy`` (float32, either may be None), with the ``stats`` that
    ``logprobs`` gave for the same logits, tokens and temperature.  ``out`` may
    be ``logits`` itself."""
    device = _gpu(logits, "logits")
    stride = _rows(logits, DTYPES, device, "logits")
    rows, vocab = logits.shape
    _want(tokens, (rows,), torch.int64, device, "tokens")
    _want(stats, (rows, 4), torch.float32, device, "stats")
    _want(grad_logprob, (rows,), torch.float32, device, "grad_logprob")
    _want(grad_entropy, (rows,), torch.float32, device, "grad_entropy")
    if out is None:
        out = _new((rows, vocab), logits.dtype, device, stream)
    grad_stride = _rows(out, (logits.dtype,), device, "out", logits.shape)
    codec._check(lib().df11_logprobs_backward(
        logits.data_ptr(), DTYPES[logits.dtype], rows, vocab, stride, _ptr(tokens),
        stats.data_ptr(), _ptr(grad_logprob), _ptr(grad_entropy), temperature, out.data_ptr(),
        grad_stride, _handle(stream, device)), "df11_logprobs_backward")
    return out


# ----------------------------------------------------------------- distillation
def distill_workspace_bytes(dtype, rows: int, vocab: int) -> int:
    return _bytes("df11_distill_workspace_bytes", DTYPES[dtype], rows, vocab)


def _teacher(teacher_index, teacher_logprob, rows, device):
    if teacher_index.dim() != 2:
        raise ValueError("teacher_index must be 2-d")
    shape = (rows, teacher_index.shape[1])
    _want(teacher_index, shape, torch.int64, device, "teacher_index")
    _want(teacher_logprob, shape, torch.float32, device, "teacher_logprob")
    return shape[1]


def distill(logits, teacher_index, teacher_logprob, tail: bool = True, temperature: float = 1.0,
            weight=None, grad=None, loss=None, stats=None, workspace=None, stream=None) -> Distill:
    """Divergence of the rows of ``logits`` (a student's, 2-d float32, bfloat16
    or float16 with contiguous rows) from a teacher's top log probabilities
    ``teacher_logprob`` (float32) at the places ``teacher_index`` (int64,
    negative: none): with ``tail`` the rest of the vocabulary is one more
    outcome, without it the teacher's probabilities are scaled to sum to one.

    With ``weight`` (float32, one per row) or ``grad`` (a tensor to fill, which
    may be ``logits`` itself) the gradient of sum(weight * loss) comes with the
    loss (weight None: ones); ``distill_backward`` gives it later otherwise."""
    device = _gpu(logits, "logits")
    stride = _rows(logits, DTYPES, device, "logits")
    rows, vocab = logits.shape
    top = _teacher(teacher_index, teacher_logprob, rows, device)
    _want(weight, (rows,), torch.float32, device, "weight")
    _want(loss, (rows,), torch.float32, device, "loss")
    _want(stats, (rows, 4), torch.float32, device, "stats")
    if weight is not None and grad is None:
        grad = _new((rows, vocab), logits.dtype, device, stream)
    grad_stride = 0 if grad is None else _rows(grad, (logits.dtype,), device, "grad", logits.shape)
    loss = _new((rows,), torch.float32, device, stream) if loss is None else loss
    stats = _new((rows, 4), torch.float32, device, stream) if stats is None else stats
    dt = DTYPES[logits.dtype]
    ws, ws_bytes = _workspace(workspace, "df11_distill_workspace_bytes", (dt, rows, vocab), device,
                              stream)
    codec._check(lib().df11_distill(
        logits.data_ptr(), dt, rows, vocab, stride, teacher_index.data_ptr(),
        teacher_logprob.data_ptr(), top, bool(tail), temperature, _ptr(weight), loss.data_ptr(),
        stats.data_ptr(), _ptr(grad), grad_stride, _ptr(ws), ws_bytes,
        _handle(stream, device)), "df11_distill")
    return Distill(loss, stats, grad)


def distill_backward(logits, teacher_index, teacher_logprob, stats, grad_loss=None,
                     tail: bool = True, temperature: float = 1.0, out=None, stream=None):
    """The gradient of ``logits`` from the gradient of ``loss`` (float32 per
    row, None: ones) and the ``stats`` that ``distill`` gave for the same
    arguments.  ``out`` may be ``logits`` itself."""
    device = _gpu(logits, "logits")
    stride = _rows(logits, DTYPES, device, "logits")
    rows, vocab = logits.shape
    top = _teacher(teacher_index, teacher_logprob, rows, device)
    _want(stats, (rows, 4), torch.float32, device, "stats")
    _want(grad_loss, (rows,), torch.float32, device, "grad_loss")
    if out is None:
        out = _new((rows, vocab), logits.dtype, device, stream)
    grad_stride = _rows(out, (logits.dtype,), device, "out", logits.shape)
    codec._check(lib().df11_distill_backward(
        logits.data_ptr(), DTYPES[logits.dtype], rows, vocab, stride, teacher_index.data_ptr(),
        teacher_logprob.data_ptr(), top, bool(tail), temperature, stats.data_ptr(),
        _ptr(grad_loss), out.data_ptr(), grad_stride, _handle(stream, device)),
        "df11_distill_backward")
    return out


# ------------------------------------------------------------ low-rank adapters
_BF16 = (torch.bfloat16,)
_Y = (torch.float32, torch.bfloat16)


def _adapters(x, a, b, scale, adapter):
    """(device, x's row stride, the call's shapes) of one set of adapters."""
    device = _gpu(x, "x")
    x_stride = _rows(x, _BF16, device, "x")
    tokens, cols = x.shape
    if a.dim() != 3 or b.dim() != 3 or b.shape[0] != a.shape[0] or b.shape[2] != a.shape[1]:
        raise ValueError("a must be (adapters, rank, cols) and b (adapters, rows, rank)")
    n, rank = a.shape[0], a.shape[1]
    rows = b.shape[1]
    _want(a, (n, rank, cols), torch.bfloat16, device, "a")
    _want(b, (n, rows, rank), torch.bfloat16, device, "b")
    _want(scale, (n,), torch.float32, device, "scale")
    _want(adapter, (tokens,), torch.int32, device, "adapter")
    return device, x_stride, (tokens, cols, rows, rank, n)


def lora_workspace_bytes(tokens: int, cols: int, rows: int, rank: int, adapters: int) -> int:
    return _bytes("df11_lora_workspace_bytes", tokens, cols, rows, rank, adapters)


def lora(x, a, b, scale, adapter, base=None, out=None, workspace=None, stream=None):
    """out[t] = base[t] + scale[i] * b[i] @ (a[i] @ x[t]) with i = adapter[t]
    (int32; any value outside 0..len(a)-1: base alone).

    x: bfloat16 (tokens, cols); a: bfloat16 (adapters, rank, cols); b: bfloat16
    (adapters, rows, rank); scale: float32 (adapters,) or None; base and out:
    (tokens, rows) float32, as ``codec.block_gemm`` gives its products, or
    bfloat16.  ``out`` may be ``base``; without either it is new, of base's
    type or float32."""
    device, x_stride, shapes = _adapters(x, a, b, scale, adapter)
    shape = (shapes[0], shapes[2])
    if out is None:
        out = _new(shape, torch.float32 if base is None else base.dtype, device, stream)
    out_stride = _rows(out, _Y, device, "out", shape)
    base_stride = 0 if base is None else _rows(base, (out.dtype,), device, "base", shape)
    ws, ws_bytes = _workspace(workspace, "df11_lora_workspace_bytes", shapes, device, stream)
    codec._check(lib().df11_lora(
        x.data_ptr(), x_stride, *shapes, a.data_ptr(), b.data_ptr(), _ptr(scale),
        adapter.data_ptr(), _ptr(base), base_stride, out.data_ptr(), out_stride, DTYPES[out.dtype],
        _ptr(ws), ws_bytes, _handle(stream, device)), "df11_lora")
    return out


def lora_backward_workspace_bytes(tokens: int, cols: int, rows: int, rank: int,
                                  adapters: int) -> int:
    return _bytes("df11_lora_backward_workspace_bytes", tokens, cols, rows, rank, adapters)


def lora_backward(x, a, b, scale, adapter, dy, dx_base=None, dx=None, da=None, db=None,
                  need_dx: bool = True, need_ab: bool = True, workspace=None,
                  stream=None) -> LoraGrads:
    """The gradients of ``lora`` for the gradient ``dy`` of its output (float32
    or bfloat16, (tokens, rows)): dx (bfloat16, added to ``dx_base`` where that
    is given; it may be ``dx_base`` itself), da and db (float32).  ``dx``,
    ``da``, ``db``: tensors to fill; ``need_dx`` or ``need_ab`` False leaves
    out dx, or da and db.  With da and db, ``dx`` must not be x or dy."""
    device, x_stride, shapes = _adapters(x, a, b, scale, adapter)
    tokens, cols, rows, rank, n = shapes
    dy_stride = _rows(dy, _Y, device, "dy", (tokens, rows))
    dx_stride = dxb_stride = 0
    if not need_dx:
        dx = dx_base = None
    else:
        if dx is None:
            dx = _new((tokens, cols), torch.bfloat16, device, stream)
        dx_stride = _rows(dx, _BF16, device, "dx", x.shape)
        if dx_base is not None:
            dxb_stride = _rows(dx_base, _BF16, device, "dx_base", x.shape)
    if not need_ab:
        da = db = None
    else:
        da = _new((n, rank, cols), torch.float32, device, stream) if da is None else da
        db = _new((n, rows, rank), torch.float32, device, stream) if db is None else db
        _want(da, (n, rank, cols), torch.float32, device, "da")
        _want(db, (n, rows, rank), torch.float32, device, "db")
    ws, ws_bytes = _workspace(workspace, "df11_lora_backward_workspace_bytes", shapes, device,
                              stream)
    codec._check(lib().df11_lora_backward(
        x.data_ptr(), x_stride, *shapes, a.data_ptr(), b.data_ptr(), _ptr(scale),
        adapter.data_ptr(), dy.data_ptr(), dy_stride, DTYPES[dy.dtype], _ptr(dx_base), dxb_stride,
        _ptr(dx), dx_stride, _ptr(da), _ptr(db), _ptr(ws), ws_bytes,
        _handle(stream, device)), "df11_lora_backward")
    return LoraGrads(dx, da, db)


# ------------------------------------------------- a paged cache of keys and values
# These calls have eleven tensors each, whose checks take longer than the kernels of a
# single token: what the tensors look like (not where they lie) is checked once and
# remembered.
def _look(t):
    return None if t is None else (t.shape, t.stride(), t.dtype, t.get_device())


def _is_contiguous(shape, stride):
    want = 1
    for n, s in zip(reversed(shape), reversed(stride)):
        if n != 1 and s != want:
            return False
        want *= n
    return True


def _as(look, shape, dtype, index, what):
    """_want for what a tensor looks like."""
    if look is not None and (look[0] != shape or look[2] != dtype or look[3] != index or
                             not (0 in shape or _is_contiguous(look[0], look[1]))):
        raise ValueError(f"{what} must be a contiguous {dtype} tensor of shape {tuple(shape)} on "
                         f"GPU {index}, not {look[2]} {tuple(look[0])} with strides {look[1]} on "
                         f"{look[3]}")


def _as_rows(look, dtypes, index, what, shape=None):
    """_rows for what a tensor looks like."""
    size, stride, dtype, where = look
    if len(size) != 2 or dtype not in dtypes or where != index or (
            shape is not None and size != shape):
        raise ValueError(f"{what} must be a 2-d tensor of {' or '.join(map(str, dtypes))}"
                         f"{'' if shape is None else ' and shape ' + str(tuple(shape))} on "
                         f"GPU {index}, not {dtype} {tuple(size)} on {where}")
    if size[1] > 1 and stride[1] != 1:
        raise ValueError(f"{what} must have contiguous rows")
    return stride[0] if size[0] > 1 else size[1]


def _cache_sizes(k, v, index):
    """What follows the addresses in df11_kv_cache."""
    shape, stride, dtype, where = k
    if len(shape) != 4 or dtype not in (torch.bfloat16, torch.float16):
        raise ValueError("cache.k must be (pages, kv_heads, page_size, head_dim), bfloat16 or "
                         f"float16, not {dtype} {tuple(shape)}")
    if v[0] != shape or v[2] != dtype:
        raise ValueError(f"cache.v must be as cache.k: {dtype} {tuple(shape)}, not {v[2]} "
                         f"{tuple(v[0])}")
    for (_, s, _, where), what in ((k, "cache.k"), (v, "cache.v")):
        if where != index:
            raise ValueError(f"{what} must be on GPU {index}, not {where}")
        if not _is_contiguous(shape[1:], s[1:]):
            raise ValueError(f"each page of {what} must be contiguous")
    return DTYPES[dtype], *shape, stride[0], v[1][0]


def _batch_sizes(start, length, table, prefix_table, index):
    """(sequences, width, table_stride) and pages of the prefix."""
    n = length[0][0] if len(length[0]) == 1 else -1
    _as(length, (n,), torch.int32, index, "batch.length")
    _as(start, (n + 1,), torch.int32, index, "batch.start")
    stride = _as_rows(table, (torch.int32,), index, "batch.table")
    if table[0][0] != n:
        raise ValueError(f"batch.table must have a row for each of {n} sequences")
    pages = 0
    if prefix_table is not None:
        pages = prefix_table[0].numel()
        _as(prefix_table, (pages,), torch.int32, index, "batch.prefix_table")
    return (n, table[0][1], stride), pages


def _heads(columns, dim, what):
    """Heads of `dim` values in the rows of a 2-d tensor."""
    heads, rest = divmod(columns, dim)
    if rest or not heads:
        raise ValueError(f"{what}'s rows must be heads of {dim} values, not {columns}")
    return heads


def _on_gpu(t, what):
    index = t.get_device()
    if index < 0:
        raise ValueError(f"{what} must be on a GPU, not {t.device}")
    if index != torch._C._cuda_getDevice():
        raise ValueError(f"{what} must be on the current GPU, not {t.device}")
    return index


def _raw_stream(stream, index):
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(index)
    return codec._handle(stream, torch.device("cuda", index))


def _check_prefix_len(n):
    if not 0 <= n < 2 ** 31:
        raise ValueError(f"batch.prefix_len must be from 0 to 2^31 - 1, not {n}")


def _pack(cache, batch, c, b, prefix_pages):
    """The two structs; `c` and `b` as _cache_sizes and _batch_sizes give them."""
    start, length, table, prefix_table, prefix_len = batch
    _check_prefix_len(prefix_len)
    return (_CACHE.pack(cache[0].data_ptr(), cache[1].data_ptr(), *c),
            _BATCH.pack(start.data_ptr(), length.data_ptr(), table.data_ptr(), *b,
                        0 if prefix_table is None else prefix_table.data_ptr(), prefix_pages,
                        prefix_len))


@functools.lru_cache(maxsize=1024)
def _append_sizes(index, q, k, v, inv_freq, q_out, cache_k, cache_v, *batch):
    c = _cache_sizes(cache_k, cache_v, index)
    b, prefix_pages = _batch_sizes(*batch, index)
    q_stride = _as_rows(q, DTYPES, index, "q")
    tokens, heads = q[0][0], _heads(q[0][1], c[4], "q")
    shape = (tokens, c[2] * c[4])
    k_stride = _as_rows(k, (q[2],), index, "k", shape)
    v_stride = _as_rows(v, (q[2],), index, "v", shape)
    rotary = 0
    if inv_freq is not None:
        rotary = 2 * inv_freq[0].numel()
        _as(inv_freq, (rotary // 2,), torch.float32, index, "inv_freq")
    out_stride = q[0][1]
    if q_out is not None:
        out_stride = _as_rows(q_out, (cache_k[2],), index, "q_out", q[0])
    return (c, b, prefix_pages, q_stride, k_stride, v_stride, DTYPES[q[2]], tokens, heads, rotary,
            out_stride)


def kv_append(q, k, v, inv_freq, cache: KVCache, batch: KVBatch, interleaved: bool = False,
              q_out=None, stream=None):
    """Rotates the rows of q and k by their positions and appends k and v to the
    cache; returns q_out, the rotated q of the cache's type.

    q: (tokens, heads * head_dim), k and v: (tokens, kv_heads * head_dim), float32
    as ``codec.block_gemm`` gives its products, bfloat16 or float16, rows
    contiguous.  A row's position is batch.prefix_len + its place among its
    sequence's own tokens; pair j of a head turns by position * inv_freq[j]
    (float32, half as many as values that turn; None: none do).  Pairs are j and
    j + len(inv_freq), or neighbours where ``interleaved``.  ``q_out`` may be q
    itself where the types are the same.  Rows behind the last sequence's are left
    as they are in q_out; a row without a place in its sequence's pages, or whose
    page is not one of the cache, is not appended.  Two rows must not share a
    token of a page."""
    index = _on_gpu(q, "q")
    start, length, table, prefix_table, _ = batch
    c, b, prefix_pages, q_stride, k_stride, v_stride, dtype, tokens, heads, rotary, out_stride = (
        _append_sizes(index, _look(q), _look(k), _look(v), _look(inv_freq), _look(q_out),
                      _look(cache[0]), _look(cache[1]), _look(start), _look(length), _look(table),
                      _look(prefix_table)))
    if q_out is None:
        q_out = _new(q.shape, cache[0].dtype, q.device, stream)
    pc, pb = _pack(cache, batch, c, b, prefix_pages)
    codec._check(lib().df11_kv_append(
        q.data_ptr(), q_stride, k.data_ptr(), k_stride, v.data_ptr(), v_stride, dtype, tokens,
        heads, _ptr(inv_freq), rotary, bool(interleaved), pc, pb, q_out.data_ptr(), out_stride,
        _raw_stream(stream, index)), "df11_kv_append")
    return q_out


def _attention_bytes(tokens, heads, c, b, prefix_pages, prefix_len):
    n = ctypes.c_uint64()
    codec._check(lib().df11_prefix_attention_workspace_bytes(
        tokens, heads, _CACHE.pack(0, 0, *c), _BATCH.pack(0, 0, 0, *b, 0, prefix_pages, prefix_len),
        ctypes.byref(n)), "df11_prefix_attention_workspace_bytes")
    return int(n.value)


def prefix_attention_workspace_bytes(tokens: int, heads: int, cache: KVCache,
                                     batch: KVBatch) -> int:
    """For this many rows of q; of cache and batch only the sizes count."""
    index = _on_gpu(cache.k, "cache.k")
    c = _cache_sizes(_look(cache.k), _look(cache.v), index)
    return _attention_bytes(tokens, heads, c, *_batch_sizes(*map(_look, batch[:4]), index),
                            batch.prefix_len)


@functools.lru_cache(maxsize=1024)
def _attention_sizes(index, prefix_len, q, out, lse, cache_k, cache_v, *batch):
    _check_prefix_len(prefix_len)
    c = _cache_sizes(cache_k, cache_v, index)
    b, prefix_pages = _batch_sizes(*batch, index)
    q_stride = _as_rows(q, (cache_k[2],), index, "q")
    tokens, heads = q[0][0], _heads(q[0][1], c[4], "q")
    out_stride = q[0][1] if out is None else _as_rows(out, (q[2],), index, "out", q[0])
    _as(lse, (tokens, heads), torch.float32, index, "lse")
    return (c, b, prefix_pages, q_stride, tokens, heads, out_stride, c[4] ** -0.5,
            _attention_bytes(tokens, heads, c, b, prefix_pages, prefix_len))


def prefix_attention(q, cache: KVCache, batch: KVBatch, scale: Optional[float] = None, out=None,
                     lse=None, need_lse: bool = False, workspace=None, stream=None) -> Attention:
    """Attention of q's rows (tokens, heads * head_dim, the cache's type, rows
    contiguous, as ``kv_append`` gives them) to the prefix that the batch's
    sequences share and to their own sequence's tokens up to themselves, which the
    cache already holds.  Consecutive heads / kv_heads query heads share a head of the
    cache.  Single and guessed tokens read the prefix together, prompts each for
    themselves; which it is goes by the sizes (rows for each sequence on average, the
    table's width), not by the lengths: prompts and single tokens of long contexts are
    faster in two calls, short contexts with a table not much wider than they are.

    scale: of the products q k before the softmax (None: head_dim ** -0.5).
    ``out`` may be q itself; ``lse`` (float32 (tokens, heads), given or with
    ``need_lse`` new) is the log of the sum of the exponentials.  Rows behind the
    last sequence's are left as they are in both.  A row that sees nothing has out
    0 and lse -inf; one that sees a page which is not of the cache has NaN."""
    index = _on_gpu(q, "q")
    start, length, table, prefix_table, prefix_len = batch
    c, b, prefix_pages, q_stride, tokens, heads, out_stride, usual, ws_bytes = _attention_sizes(
        index, prefix_len, _look(q), _look(out), _look(lse), _look(cache[0]), _look(cache[1]),
        _look(start), _look(length), _look(table), _look(prefix_table))
    if out is None:
        out = _new(q.shape, q.dtype, q.device, stream)
    if lse is None and need_lse:
        lse = _new((tokens, heads), torch.float32, q.device, stream)
    pc, pb = _pack(cache, batch, c, b, prefix_pages)
    if workspace is not None:
        workspace, ws_bytes = _workspace(workspace, None, None, q.device, stream)
    elif ws_bytes:
        workspace = _new((ws_bytes,), torch.uint8, q.device, stream)
    codec._check(lib().df11_prefix_attention(
        q.data_ptr(), q_stride, tokens, heads, usual if scale is None else scale, pc, pb,
        out.data_ptr(), out_stride, _ptr(lse), _ptr(workspace), ws_bytes,
        _raw_stream(stream, index)), "df11_prefix_attention")
    return Attention(out, lse)
