"""Calls over no walks at all, as a search from no starts makes them: on the host, with tensors that say they are on a GPU."""
import ctypes as C

import pytest
import torch

from test_answers_host import A, B, P, gpu, gs, lib, reorder  # noqa: F401


@pytest.mark.parametrize("columns", [[1, None], [None, None], [3, None]])
@pytest.mark.parametrize("beams,width", [(3, 3), (4, 2)])
def test_reorder_of_no_walks(gs, monkeypatch, columns, beams, width):  # noqa: F811
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(gs, "_stream_of", lambda device: None)
    parents, nodes = gpu(torch.zeros(0, width, dtype=torch.int32)), gpu(torch.zeros(0, width, dtype=torch.int32))
    states = [gpu(torch.zeros(0, 4, dtype=torch.int32)), gpu(torch.zeros(0, 5, 3))]
    outs = [gpu(torch.zeros(0, 4, dtype=torch.int32)), gpu(torch.zeros(0, 5, 3))]
    gs.gs_beam_reorder(states, parents, beams, outs=outs, nodes=nodes, columns=columns)
    if beams == width:
        gs.gs_beam_reorder(states, parents, beams, nodes=nodes, columns=columns)
    with pytest.raises(ValueError):
        gs.gs_beam_reorder(states, parents, beams, outs=outs, nodes=nodes, columns=[4, None])


def test_reorder_of_no_walks_without_addresses(lib):  # noqa: F811
    assert reorder(lib, [(None, None, 16, 12), (None, None, 7, -1)], groups=0, parents=None, nodes=None) == 0
    assert reorder(lib, [(A, B, 16, 12)], groups=0, nodes=None) == 0
    assert reorder(lib, [(A, B, 16, 16)], groups=0) == -1 and reorder(lib, [(A, B, 16, 2)], groups=0) == -1
    assert reorder(lib, [(A, B, 16, 12)], groups=1, nodes=None) == -1 and reorder(lib, [(None, None, 16, 12)], groups=1) == -1
