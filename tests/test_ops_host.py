"""What the operators' entry points refuse before anything is enqueued, and
their declarations (CPU only: addresses are numbers that nothing reads)."""
import ctypes
import os
import re

import pytest
import torch

from paper_2504_11651_amd import codec, ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, SMALL, UNSUPPORTED = -1, -3, -6
A = 1 << 20  # an aligned address


def test_library_exports_every_declared_operator():
    header = open(os.path.join(ROOT, "include", "df11_ops.h")).read()
    declared = set(re.findall(r"^int\s*(df11_\w+)\(", header, re.M))
    assert declared == set(ops.EXPORTS)
    for name in declared:
        assert len(getattr(ops.lib(), name).argtypes) == len(
            re.search(name + r"\((.*?)\);", header, re.S).group(1).split(","))
    for name, value in (("DF11_MAX_TOP", ops.MAX_TOP), ("DF11_MAX_RANK", ops.MAX_RANK)):
        assert re.search(rf"#define {name} (\d+)", header).group(1) == str(value)
    for i, name in enumerate(("F32", "BF16", "F16")):
        assert f"#define DF11_{name} {i}\n" in header


def logprobs(**change):
    a = dict(logits=A, dtype=0, rows=2, vocab=100, stride=100, tokens=A, top=4, tau=1.0, logprob=A,
             rank=A, entropy=A, top_logprob=A, top_index=A, stats=A, ws=A, ws_bytes=1 << 30, stream=None)
    assert set(change) <= set(a)
    return ops.lib().df11_logprobs(*(a | change).values())


@pytest.mark.parametrize("change, rc", [
    (dict(dtype=3), INVALID), (dict(vocab=0, top=0), INVALID), (dict(vocab=2 ** 31), INVALID),
    (dict(top=129, vocab=1000, stride=1000), INVALID), (dict(top=101), INVALID),
    (dict(stride=99), INVALID), (dict(logits=None), INVALID), (dict(logits=A + 2), INVALID),
    (dict(logits=A + 1, dtype=1), INVALID), (dict(tau=0.0), INVALID), (dict(tau=-1.0), INVALID),
    (dict(tau=float("nan")), INVALID), (dict(tau=float("inf")), INVALID), (dict(tau=1e-45), INVALID),
    (dict(tokens=None), INVALID), (dict(tokens=None, logprob=None), INVALID),
    (dict(top_logprob=None), INVALID), (dict(top_index=None), INVALID), (dict(stats=A + 4), INVALID),
    (dict(tokens=A + 4), INVALID), (dict(rows=(1 << 23) + 1), UNSUPPORTED),
    (dict(rows=1 << 62), UNSUPPORTED), (dict(rows=2 ** 63, vocab=16384, stride=16384), UNSUPPORTED),
    (dict(rows=0), 0), (dict(rows=0, logits=None), 0),
])
def test_logprobs_refusals(change, rc):
    assert logprobs(**change) == rc


def logprobs_backward(**change):
    a = dict(logits=A, dtype=0, rows=2, vocab=100, stride=100, tokens=A, stats=A, grad_logprob=A,
             grad_entropy=A, tau=1.0, grad=2 * A, grad_stride=100, stream=None)
    assert set(change) <= set(a)
    return ops.lib().df11_logprobs_backward(*(a | change).values())


@pytest.mark.parametrize("change, rc", [
    (dict(grad=None), INVALID), (dict(grad=A + 2), INVALID), (dict(grad_stride=99), INVALID),
    (dict(stats=None), INVALID), (dict(stats=A + 8), INVALID), (dict(tokens=None), INVALID),
    (dict(grad_logprob=None, grad_entropy=None), INVALID), (dict(grad=A, grad_stride=101), INVALID),
    (dict(tau=0.0), INVALID), (dict(rows=0), 0),
])
def test_logprobs_backward_refusals(change, rc):
    assert logprobs_backward(**change) == rc


def distill(**change):
    a = dict(logits=A, dtype=1, rows=2, vocab=100, stride=100, index=A, teacher=A, top=4, tail=1, tau=1.0,
             weight=A, loss=A, stats=A, grad=2 * A, grad_stride=100, ws=A, ws_bytes=1 << 30, stream=None)
    assert set(change) <= set(a)
    return ops.lib().df11_distill(*(a | change).values())


@pytest.mark.parametrize("change, rc", [
    (dict(top=0), INVALID), (dict(top=129), INVALID), (dict(index=None), INVALID),
    (dict(teacher=None), INVALID), (dict(loss=None), INVALID), (dict(stats=None), INVALID),
    (dict(index=A + 4), INVALID), (dict(stride=50), INVALID), (dict(grad_stride=50), INVALID),
    (dict(grad=2 * A + 1), INVALID), (dict(grad=A, grad_stride=128), INVALID),
    (dict(tau=float("nan")), INVALID), (dict(rows=(1 << 23) + 1), UNSUPPORTED), (dict(rows=0), 0),
])
def test_distill_refusals(change, rc):
    assert distill(**change) == rc


def distill_backward(**change):
    a = dict(logits=A, dtype=1, rows=2, vocab=100, stride=100, index=A, teacher=A, top=4, tail=1, tau=1.0,
             stats=A, grad_loss=A, grad=2 * A, grad_stride=100, stream=None)
    assert set(change) <= set(a)
    return ops.lib().df11_distill_backward(*(a | change).values())


@pytest.mark.parametrize("change, rc", [
    (dict(top=0), INVALID), (dict(top=129), INVALID), (dict(index=None), INVALID),
    (dict(stats=None), INVALID), (dict(grad=None), INVALID), (dict(grad=A, grad_stride=128), INVALID),
    (dict(dtype=7), INVALID), (dict(rows=0), 0),
])
def test_distill_backward_refusals(change, rc):
    assert distill_backward(**change) == rc


SHAPES = dict(tokens=4, cols=128, rows=64, rank=8, n=2)


def lora(**change):
    a = dict(x=A, x_stride=128, **SHAPES, a=A, b=A, scale=A, adapter=A, base=2 * A, base_stride=64, out=A,
             out_stride=64, dtype=0, ws=A, ws_bytes=1 << 30, stream=None)
    assert set(change) <= set(a)
    return ops.lib().df11_lora(*(a | change).values())


@pytest.mark.parametrize("change, rc", [
    (dict(cols=0), INVALID), (dict(rows=0), INVALID), (dict(rank=0), INVALID), (dict(n=0), INVALID),
    (dict(cols=96, x_stride=96), UNSUPPORTED), (dict(rows=72, out_stride=72), UNSUPPORTED),
    (dict(rank=4), UNSUPPORTED), (dict(rank=12), UNSUPPORTED), (dict(rank=136), UNSUPPORTED),
    (dict(tokens=2 ** 31), UNSUPPORTED), (dict(n=65536), UNSUPPORTED),
    (dict(x=None), INVALID), (dict(x=A + 8), INVALID), (dict(x_stride=120), INVALID),
    (dict(x_stride=132), INVALID), (dict(a=A + 2), INVALID), (dict(b=None), INVALID),
    (dict(adapter=None), INVALID), (dict(scale=A + 2), INVALID), (dict(out=None), INVALID),
    (dict(out=A + 4), INVALID), (dict(out_stride=66), INVALID), (dict(out_stride=60), INVALID),
    (dict(base=2 * A + 8), INVALID), (dict(base_stride=65), INVALID),
    (dict(base=A, base_stride=64, out_stride=128), INVALID), (dict(dtype=2), INVALID),
    (dict(dtype=1, out_stride=68), INVALID), (dict(ws_bytes=0), SMALL), (dict(ws=None), INVALID),
    (dict(ws=A + 4), INVALID), (dict(tokens=0), 0), (dict(tokens=0, x=None, ws=None, ws_bytes=0), 0),
])
def test_lora_refusals(change, rc):
    assert lora(**change) == rc


def lora_backward(**change):
    a = dict(x=A, x_stride=128, **SHAPES, a=A, b=A, scale=A, adapter=A, dy=A, dy_stride=64, dy_dtype=0,
             dx_base=2 * A, dx_base_stride=128, dx=A, dx_stride=128, da=A, db=A, ws=A, ws_bytes=1 << 30,
             stream=None)
    assert set(change) <= set(a)
    return ops.lib().df11_lora_backward(*(a | change).values())


@pytest.mark.parametrize("change, rc", [
    (dict(da=None), INVALID), (dict(db=None), INVALID), (dict(dx=None, da=None, db=None), INVALID),
    (dict(dy=None), INVALID), (dict(dy=A + 4), INVALID), (dict(dy_dtype=2), INVALID),
    (dict(dy_stride=56), INVALID), (dict(dx=A + 2), INVALID), (dict(dx_stride=100), INVALID),
    (dict(dx_base_stride=100), INVALID), (dict(dx_base=A, dx_base_stride=136), INVALID),
    (dict(da=A + 4), INVALID), (dict(db=A + 8), INVALID), (dict(ws_bytes=16), SMALL),
    (dict(ws=None), INVALID), (dict(rank=9), UNSUPPORTED), (dict(cols=65), UNSUPPORTED),
    (dict(scale=A + 1), INVALID), (dict(adapter=A + 2), INVALID),
])
def test_lora_backward_refusals(change, rc):
    assert lora_backward(**change) == rc


def test_workspace_sizes():
    assert ops.logprobs_workspace_bytes(torch.float32, 0, 1) >= 0
    assert ops.distill_workspace_bytes(torch.bfloat16, 5, 77) >= 0
    assert ops.lora_workspace_bytes(0, 64, 16, 8, 1) >= 0
    for fn, args in ((ops.logprobs_workspace_bytes, (torch.float32, 1, 10, 11)),
                     (ops.distill_workspace_bytes, (torch.float32, 1, 0)),
                     (ops.lora_workspace_bytes, (1, 64, 16, 7, 1)),
                     (ops.lora_backward_workspace_bytes, (1, 63, 16, 8, 1))):
        with pytest.raises(codec.DF11Error):
            fn(*args)
    for name in ("df11_logprobs_workspace_bytes", "df11_distill_workspace_bytes",
                 "df11_lora_workspace_bytes", "df11_lora_backward_workspace_bytes"):
        fn = getattr(ops.lib(), name)
        args = [1, 64, 64, 8, 1][:len(fn.argtypes) - 1]
        assert fn(*args, None) == INVALID
    assert ctypes.sizeof(ctypes.c_void_p) == 8


def test_host_tensors_are_refused():
    z = torch.zeros(2, 64)
    i, f = torch.zeros(2, dtype=torch.int64), torch.zeros(2)
    for call in (lambda: ops.logprobs(z, i), lambda: ops.logprobs_backward(z, i, torch.zeros(2, 4), f),
                 lambda: ops.distill(z, i[:, None], f[:, None]),
                 lambda: ops.distill_backward(z, i[:, None], f[:, None], torch.zeros(2, 4)),
                 lambda: ops.lora(z.bfloat16(), torch.zeros(1, 8, 64).bfloat16(),
                                  torch.zeros(1, 16, 8).bfloat16(), None, i.int())):
        with pytest.raises(ValueError, match="on a GPU"):
            call()
