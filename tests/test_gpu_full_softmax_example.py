"""The example runs its operators together: the loss falls, the norms are those of the gradients, answers are what was allowed."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "full_softmax.py")


def test_training_and_answers():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("full_softmax", PATH)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, norms, ids, probs = example.main(steps=60)
    assert all(x == x and x < 20 for x in losses) and min(norms) > 0
    assert sum(losses[-10:]) < sum(losses[:10])
    assert torch.all(ids >= 0) and torch.all(ids < 10_000) and torch.all(ids != torch.arange(8, device=ids.device))
    assert torch.all(probs > 0) and torch.all(probs <= 1)
