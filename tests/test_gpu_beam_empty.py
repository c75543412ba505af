"""A search from no starts: every call of it takes its empty inputs."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_search_from_no_starts():
    import beam_walks
    from paper_2407_15452_amd import binding as gs
    w = torch.randn(100, 64, generator=torch.Generator().manual_seed(1)).to(DEV)
    t = gs.gs_quantize_rows(w)
    walks, logp, sums = beam_walks.search(t, t, w, torch.zeros(0, dtype=torch.int32, device=DEV), torch.tensor([3], device=DEV), 4, 6)
    assert tuple(walks.shape) == (0, 4, 6) and tuple(logp.shape) == (0, 4) and sums.numel() == 0


def test_reorder_of_no_walks():
    from paper_2407_15452_amd import binding as gs
    none = torch.zeros(0, 4, dtype=torch.int32, device=DEV)
    walks, rows = torch.zeros(0, 9, dtype=torch.int32, device=DEV), torch.zeros(0, 5, device=DEV)
    gs.gs_beam_reorder([walks, rows], none, 4, nodes=none, columns=[8, None])
    gs.gs_beam_reorder([walks, rows], none, 7, outs=[walks.clone(), rows.clone()], nodes=none, columns=[8, None])
    torch.cuda.synchronize()
