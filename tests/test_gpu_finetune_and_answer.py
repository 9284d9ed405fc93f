"""The example that fine-tunes a network with clipped gradients and answers with its head in 8 bits."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_finetune_and_answer():
    spec = importlib.util.spec_from_file_location("finetune_and_answer",
                                                  os.path.join(ROOT, "examples", "finetune_and_answer.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    history, off = example.main(steps=6, size=100)
    # a step that follows the gradient of a smooth loss by a small length lowers it
    assert history[-1] < history[0]
    # codes of 8 bits are within half of 1/127 of a token's largest value: a few percent over two layers
    assert off < 0.05
