"""The example's training loop: boundary, loss, clipping and update together.
With moments in 8 bits it learns what it learns with 32."""
import importlib.util
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("train_last_stage", os.path.join(ROOT, "examples", "train_last_stage.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("bits", [8, 32])
def test_the_pipeline_learns(example, tc, bits):
    vocab = 500
    model = example.Pipeline(vocab=vocab, hidden=128, state_bits=bits)
    losses = [float(model.step(*example.batch(vocab, 2048, k))) for k in range(80)]
    assert all(math.isfinite(x) for x in losses)
    # it starts at chance and a next-token rule is learned to well under half of it
    assert abs(losses[0] - math.log(vocab)) < 1.0
    assert losses[-1] < 0.5 * math.log(vocab)
    assert tc.device_errors() == 0
    for params, opt in model.stages:
        assert opt.t == 80
        for p, w in zip(params, opt.w32):
            assert torch.equal(p.data, w.bfloat16())
