"""GPU test of the example that runs the 4-bit products, their gradients, the
outer step, the functional distance and sampling together."""

import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


def test_workers_learn_output_layers_in_4_bits():
    import torch

    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "heads_in_4_bits.py")
    spec = importlib.util.spec_from_file_location("heads_in_4_bits", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    kw = dict(workers=3, vocab=777, width=200, tokens=70, rounds=4, inner_steps=6, lr=8.0)
    report = example.train(**kw)
    assert len(report) == 4
    assert abs(report[0]["loss"] - torch.tensor(777.0).log().item()) < 1e-4  # all logits are zero at first
    assert all(b["loss"] < a["loss"] for a, b in zip(report, report[1:]))
    for r in report:
        assert 0 < r["distance"] < 0.7  # at most log 2
        assert bool((r["tokens"] >= 0).all()) and bool((r["tokens"] < 777).all())
        assert bool((r["probs"] > 0).all()) and bool((r["probs"] <= 1).all())
    again = example.train(**kw)
    for a, b in zip(report, again):
        assert a["distance"] == b["distance"] and torch.equal(a["tokens"], b["tokens"])
        assert torch.equal(a["probs"], b["probs"])
