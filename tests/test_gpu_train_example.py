"""The training example: the operators together, with gradients through them, in both precisions of the optimiser's states."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("train_recurrence", os.path.join(ROOT, "examples", "train_recurrence.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("bits", [32, 8])
def test_training_learns_the_grammar(example, bits):
    """A uniform guess over the bytes costs log 256 = 5.5; the sentences' own choices, three of three words in some 27 bytes, about
    0.12 per byte."""
    losses, model = example.train(steps=60, width=128, bits=bits, say=lambda s: print(s, flush=True))
    assert losses[0] > 3.0
    assert sum(losses[-5:]) / 5 < 0.5 * losses[0] and losses[-1] < 1.5


def test_tokens_one_by_one_see_what_the_whole_sequence_sees(example):
    """The states that single tokens leave give the hidden states' logits of the whole sequence: the same next byte wherever one
    stands out by more than bf16's rounding over the blocks."""
    _, model = example.train(steps=20, width=128, bits=32, say=lambda s: None)
    text = model.write(b"the dog ", 30)
    assert len(text) > 12
    tokens = torch.tensor([list(text)], device="cuda")
    with torch.no_grad():
        logits = (model.hidden(tokens, torch.zeros_like(tokens, dtype=torch.bool)) @ model.embedding.t()).float()[0]
    for i in range(7, len(text) - 1):
        top = logits[i].topk(2)
        if top.values[0] - top.values[1] > 0.25:
            assert int(top.indices[0]) == text[i + 1], i
