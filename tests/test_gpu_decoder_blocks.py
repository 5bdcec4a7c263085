"""The example decoder (examples/decoder_steps.py) with experts in e4m3 blocks of 128, chosen by groups: prompts, steps and a captured step."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROMPTS = [list(range(1, 70)), list(range(500, 533)), [7]]


def test_steps_eager_again_and_captured():
    spec = importlib.util.spec_from_file_location("decoder_steps", os.path.join(ROOT, "examples", "decoder_steps.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    model = example.Decoder(layers=2, d_model=512, d_ff=1024, experts=8, n_heads=8, n_kv_heads=2, vocab=1003, batch=3, max_tokens=256, page=32,
                            max_new=512, blocks=True)
    assert model.layers[0]["w1"].dtype == torch.float8_e4m3fn and tuple(model.layers[0]["w1_scale"].shape) == (8, 2, 8, 4)
    logits = model.prefill(PROMPTS)
    assert torch.isfinite(logits).all()
    plain = model.generate(PROMPTS, 12)
    again = model.generate(PROMPTS, 12)
    graph = model.generate(PROMPTS, 12, graph=True)
    assert torch.equal(plain, again) and torch.equal(plain, graph)
    assert (plain >= 0).all() and (plain < 1003).all() and plain.unique().numel() > 3
