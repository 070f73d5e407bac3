"""Calls on a named stream: what they allocate belongs to that stream, so that no
memory which the current stream still uses, or goes on to use, is written there."""
import pytest
import torch

from paper_2504_11651_amd import ops

from conftest import gpu_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs an MI355X")]


def owner(t):
    """The stream whose memory a tensor lies in."""
    for s in torch.cuda.memory_snapshot():
        if s["address"] <= t.data_ptr() < s["address"] + s["total_size"]:
            return s["stream"]
    raise AssertionError("not the allocator's")


def calls(stream):
    """Every operator with nothing given that it can allocate itself."""
    g = torch.Generator(device="cuda").manual_seed(1)
    z = torch.randn((5, 9001), generator=g, device="cuda")
    tokens = torch.arange(5, device="cuda")
    index = torch.arange(20, device="cuda").view(5, 4)
    logp = torch.full((5, 4), -1.5, device="cuda")
    ones = torch.ones(5, device="cuda")
    x = torch.randn((5, 128), generator=g, device="cuda").bfloat16()
    a = torch.randn((2, 8, 128), generator=g, device="cuda").bfloat16()
    b = torch.randn((2, 64, 8), generator=g, device="cuda").bfloat16()
    adapter = torch.tensor([0, 1, -1, 1, 0], dtype=torch.int32, device="cuda")
    dy = torch.randn((5, 64), generator=g, device="cuda")
    torch.cuda.synchronize()
    r = ops.logprobs(z, tokens, top=6, stream=stream)
    d = ops.distill(z, index, logp, weight=ones, stream=stream)
    out = [*r, ops.logprobs_backward(z, tokens, r.stats, ones, ones, stream=stream), d.loss, d.stats, d.grad,
           ops.distill_backward(z, index, logp, d.stats, stream=stream),
           ops.lora(x, a, b, None, adapter, stream=stream),
           *ops.lora_backward(x, a, b, None, adapter, dy, stream=stream)]
    torch.cuda.synchronize()
    return out


def test_outputs_lie_in_the_named_streams_memory():
    want = calls(None)
    for t in want:
        assert owner(t) == torch.cuda.current_stream().cuda_stream
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        got = calls(stream)
        for k, (p, q) in enumerate(zip(got, want)):
            assert owner(p) == side.cuda_stream and torch.equal(p, q), k


def test_the_current_stream_named_is_the_current_stream():
    for p, q in zip(calls(torch.cuda.current_stream()), calls(None)):
        assert owner(p) == torch.cuda.current_stream().cuda_stream and torch.equal(p, q)


def test_workspaces_lie_in_the_named_streams_memory(monkeypatch):
    seen = []
    real = ops._workspace

    def spy(given, *rest):
        ws = real(given, *rest)
        if ws[0] is not None:
            seen.append(owner(ws[0]))
        return ws

    monkeypatch.setattr(ops, "_workspace", spy)
    side = torch.cuda.Stream()
    calls(side)
    assert len(seen) == 4 and set(seen) == {side.cuda_stream}


def test_dropped_outputs_wait_for_both_streams():
    """What the current stream may still read is not handed out again before: a block
    of the named stream's memory is known to the allocator as used by both."""
    side = torch.cuda.Stream()
    t = calls(side)[0]
    torch.cuda.synchronize()
    where = t.data_ptr()
    # work of the current stream that is under way when the tensor is dropped
    big = torch.randn((4096, 4096), device="cuda")
    for _ in range(60):
        big = big @ big * 1e-2
    kept = t + big[0, 0]
    done = torch.cuda.Event()
    done.record()
    del t
    with torch.cuda.stream(side):
        again = [torch.empty(5, dtype=torch.float32, device="cuda") for _ in range(4)]
    if not done.query():
        assert all(x.data_ptr() != where for x in again)
    torch.cuda.synchronize()
    assert kept.shape == (5,)
