"""The example runs its operators together: walks begin where they were asked to, visit no node twice, end at goals, and their sums follow them."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "beam_walks.py")


def test_walks():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("beam_walks", PATH)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    w_in, walks, logp, sums = example.main(beams=5, num_starts=3, length=9)
    walks, logp, rows = walks.cpu(), logp.cpu(), w_in.double().cpu()
    assert tuple(walks.shape) == (3, 5, 9) and tuple(logp.shape) == (3, 5)
    assert torch.all(logp[:, :-1] >= logp[:, 1:]) and torch.all(logp <= 0) and torch.all(logp > float("-inf"))
    for s in range(3):
        assert len({tuple(w) for w in walks[s].tolist()}) == 5
        for k in range(5):
            walk = walks[s, k].tolist()
            nodes = [x for x in walk if x >= 0]
            assert nodes[0] == s and len(set(nodes)) == len(nodes) and walk == nodes + [-1] * (9 - len(nodes))
            assert all(x < 10_000 for x in nodes) and not any(100 <= x < 300 for x in nodes[1:-1])
            assert len(nodes) == 9 or 100 <= nodes[-1] < 300
            # at most eight additions in fp32, half a step of 2^-24 of a partial sum each
            bound = 8 * 2.0 ** -24 * rows[nodes].abs().sum(0)
            assert torch.all((sums[s, k].double().cpu() - rows[nodes].sum(0)).abs() <= bound)
