"""The example of a whole training step through the library learns."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("state", ["f32", "f8"])
def test_it_learns(state):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("train_lm",
                                                  os.path.join(ROOT, "examples", "train_lm.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    first, last, perplexity, floor = example.train(steps=120, workers=2, rows=32, length=8,
                                                   state=state)
    assert last < 0.8 * first          # from about log(vocabulary)
    assert perplexity > 0.9 * torch.tensor(floor).exp().item()
