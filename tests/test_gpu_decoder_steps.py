"""The example decoder (examples/decoder_steps.py): its operators together, as a program runs them."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("decoder_steps", os.path.join(ROOT, "examples", "decoder_steps.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def small(example, **kw):
    return example.Decoder(**{**dict(layers=2, d_model=512, d_ff=1024, experts=8, n_heads=8, n_kv_heads=2, vocab=1003, batch=3, max_tokens=256, page=32,
                                     max_new=512), **kw})


PROMPTS = [list(range(1, 70)), list(range(500, 533)), [7]]


def test_steps_see_what_a_prefill_of_the_same_tokens_sees(example):
    """Greedy decoding, then a prefill of prompt and answer in one: its logits choose the same next token, or one that is as good up to
    the roundings that tell the two ways apart (bf16 activations, scales of pages that grew token by token)."""
    model = small(example)
    tokens = model.generate(PROMPTS, 20, temperature=0.0)
    whole = [p + t[:-1] for p, t in zip(PROMPTS, tokens.tolist())]
    logits = model.prefill(whole).float()
    best = logits.max(1).values
    chosen = logits.gather(1, tokens[:, -1:].long().to(logits.device))[:, 0]
    # e4m3 keys and values: half a step is 2^-4 of an element; over 64 dimensions and two layers some per cent of the logits' spread
    assert (best - chosen <= 0.15 * logits.std(1)).all(), (best - chosen, logits.std(1))


def test_a_captured_step_gives_the_same_tokens(example):
    model = small(example)
    plain = model.generate(PROMPTS, 12)
    again = model.generate(PROMPTS, 12)
    graph = model.generate(PROMPTS, 12, graph=True)
    assert torch.equal(plain, again) and torch.equal(plain, graph)
    assert (plain >= 0).all() and (plain < 1003).all() and plain.unique().numel() > 3
