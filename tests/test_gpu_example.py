"""The example that uses the operators together, at a small size."""
import importlib.util
import os

import pytest
import torch

from conftest import gpu_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs an MI355X")]

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_adapters_learn_from_the_teacher(capsys):
    spec = importlib.util.spec_from_file_location(
        "distill_adapters", os.path.join(ROOT, "examples", "distill_adapters.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, served = example.main(vocab=2048, hidden=512, rows=96, steps=40, top=16)
    assert losses[-1] < 0.5 * losses[0] and all(x >= 0 for x in losses)
    # the token without an adapter is the teacher's own: its choice is the best one
    assert served.rank[0] == 0
    for rank, logprob, top in zip(served.rank, served.logprob, served.top_logprob):
        if rank < 5:
            assert logprob == top[rank]
    assert torch.isfinite(served.entropy).all() and "tenant  2" in capsys.readouterr().out
