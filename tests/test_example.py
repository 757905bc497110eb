"""The example trains and serves: the gated layer, its gradients, the layer back and the optimiser together.

Bars.  Teacher and student start independent, so the relative loss starts near 2; the bar of a fall to 0.7 of that is the one of the
optimiser's own test.  One token alone and in a batch take the same products in another order: some 2^-24 of their terms in float32, a last
place of each of three roundings (the gated layer's result, the layer back's, the sum) in bfloat16."""
import importlib.util
import os

import pytest
import torch

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "gated_feed_forward.py")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype, bar", [pytest.param(torch.float32, 2e-6, id="f32"), pytest.param(torch.bfloat16, 2.0 ** -6, id="bf16")])
def test_trains_and_serves(dtype, bar):
    spec = importlib.util.spec_from_file_location("gated_feed_forward", PATH)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    block, losses = example.train(steps=80, dtype=dtype)
    assert torch.isfinite(losses).all() and losses[-5:].mean() < 0.7 * losses[:5].mean(), losses[::10]
    tokens = torch.randn(8, example.CHANNELS, device="cuda").to(dtype)
    together = example.serve(block, tokens)
    for i in (0, 7):
        assert (example.serve(block, tokens[i:i + 1])[0] - together[i]).float().norm() <= bar * together[i].float().norm()
