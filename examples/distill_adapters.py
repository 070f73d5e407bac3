"""Trains low-rank adapters over a frozen, compressed LM head, then serves them.

A teacher and a student share one LM head, which is kept compressed and decoded
losslessly on the GPU for its products.  The student sees the hidden states
mirrored along a few directions of its tenant, and each tenant's adapter learns to
undo it from the teacher's best alternatives alone:

  head products (codec.block_forward)
    teacher: ops.logprobs     its top log probabilities, all that is kept of it
    student: ops.lora         every tenant's adapter beside the shared product
             ops.distill      loss, and the gradient in place of the logits
             ops.lora_backward  the adapters' gradients -> Adam

and at the end one serving step for a batch of tenants' single tokens, with the
log probability and rank of the teacher's choice.

  python examples/distill_adapters.py [--vocab 8192 --hidden 1024 --steps 60]
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2504_11651_amd import codec, ops, synth  # noqa: E402


class Head:
    """A compressed LM head: logits of at most 64 rows of hidden states at a time."""

    def __init__(self, vocab, hidden, device):
        self.shape = (vocab, hidden)
        self.stream = codec.to_device(codec.encode(synth.lm_head(vocab, hidden)), device)
        self.weights = torch.empty(vocab * hidden, dtype=torch.bfloat16, device=device)
        self.mats = [(0, vocab, hidden)]
        need = codec.gemm_workspace_bytes(self.mats, codec.MAX_TOKENS)
        self.workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=device)
        codec.decode_block(self.stream, self.weights)

    def __call__(self, x):
        y = torch.empty((x.shape[0], self.shape[0]), dtype=torch.float32, device=x.device)
        for i in range(0, x.shape[0], codec.MAX_TOKENS):
            part = slice(i, min(x.shape[0], i + codec.MAX_TOKENS))
            # the first part decodes the head, the others multiply what it left
            call = codec.block_forward if i == 0 else codec.block_gemm
            call(self.stream if i == 0 else self.weights, *((self.weights,) if i == 0 else ()),
                 self.mats, [x[part]], [y[part]], self.workspace)
        return y


def hidden_states(rows, hidden, step, mirror, adapter):
    """The rows' hidden states, strong along their tenants' directions, and as the
    student sees them."""
    x = synth.activations(rows, hidden, 11, step)
    x = torch.from_numpy(x.view(np.int16)).to(mirror.device).view(torch.bfloat16).float()
    q = mirror[adapter.clamp(min=0).long()]  # rows x hidden x directions
    qt = q.transpose(1, 2).contiguous()
    x = x + 20.0 * ((x[:, None] @ q) @ qt)[:, 0]
    seen = x - 2.0 * ((x[:, None] @ q) @ qt)[:, 0] * (adapter >= 0)[:, None]
    return x.bfloat16(), seen.bfloat16()


def main(vocab=8192, hidden=1024, rank=16, tenants=3, rows=192, steps=60, top=32, rate=0.02,
         device="cuda"):
    device = torch.device(device, torch.cuda.current_device())
    g = torch.Generator(device="cpu").manual_seed(5)
    head = Head(vocab, hidden, device)
    mirror = torch.linalg.qr(torch.randn((tenants, hidden, rank // 4), generator=g)).Q.to(device)
    # requests of ragged lengths, each of one tenant; the last rows have none
    adapter = torch.randint(tenants, (rows,), generator=g).sort().values.int().to(device)
    adapter[-rows // 16:] = -1
    a = (torch.randn((tenants, rank, hidden), generator=g) * hidden ** -0.5).to(device)
    b = torch.zeros((tenants, vocab, rank), device=device)
    scale = torch.full((tenants,), 2.0, device=device)
    weight = (adapter >= 0).float() / (adapter >= 0).sum()
    moments = [[torch.zeros_like(p) for p in (a, b)] for _ in range(2)]
    losses = []
    for step in range(steps):
        x, seen = hidden_states(rows, hidden, step % 8, mirror, adapter)
        teacher = ops.logprobs(head(x), top=top)
        a16, b16 = a.bfloat16(), b.bfloat16()
        student = head(seen)
        ops.lora(seen, a16, b16, scale, adapter, base=student, out=student)
        kept = ops.distill(student, teacher.top_index, teacher.top_logprob, weight=weight,
                           grad=student)
        grads = ops.lora_backward(seen, a16, b16, scale, adapter, kept.grad, need_dx=False)
        losses.append((kept.loss * weight).sum())
        for p, d, m, v in zip((a, b), (grads.da, grads.db), *moments):
            m.mul_(0.9).add_(d, alpha=0.1)
            v.mul_(0.99).addcmul_(d, d, value=0.01)
            p.sub_(rate * 0.1 * (m / (1 - 0.9 ** (step + 1))) /
                   ((v / (1 - 0.99 ** (step + 1))).sqrt() + 1e-8))
        if step % 10 == 0 or step == steps - 1:
            print(f"step {step:3d}  loss {float(losses[-1]):.4f}", flush=True)

    # one token for each tenant, and one without an adapter
    who = torch.arange(-1, tenants, dtype=torch.int32, device=device)
    x, seen = hidden_states(tenants + 1, hidden, 99, mirror, who)
    best = ops.logprobs(head(x), top=1).top_index[:, 0].contiguous()
    logits = head(seen)
    ops.lora(seen, a.bfloat16(), b.bfloat16(), scale, who, base=logits, out=logits)
    served = ops.logprobs(logits, best, top=5)
    for t in range(tenants + 1):
        print(f"tenant {int(who[t]):2d}  the teacher's choice {int(best[t])}: log probability "
              f"{float(served.logprob[t]):.3f}, rank {int(served.rank[t])}, entropy "
              f"{float(served.entropy[t]):.3f}, best {served.top_index[t].tolist()}")
    return torch.stack(losses).tolist(), served


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("vocab", 8192), ("hidden", 1024), ("rank", 16), ("tenants", 3),
                        ("rows", 192), ("steps", 60), ("top", 32)):
        ap.add_argument(f"--{name}", type=int, default=value)
    ap.add_argument("--rate", type=float, default=0.02)
    main(**vars(ap.parse_args()))
