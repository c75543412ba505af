"""Numbers that the binding passes on as 32 bits: beyond that they are refused, not cut off."""
import pytest
import torch

from test_answers_host import gpu, gs, lib  # noqa: F401


@pytest.mark.parametrize("width", [0, -1, 257, (1 << 32) + 4, -(1 << 32) + 4, 1 << 40])
def test_width(gs, monkeypatch, width):  # noqa: F811
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(gs, "_stream_of", lambda device: None)
    outs = dict(parents_out=gpu(torch.zeros(0, max(width, 0), dtype=torch.int32)), nodes_out=gpu(torch.zeros(0, max(width, 0), dtype=torch.int32)),
                logp_out=gpu(torch.zeros(0, max(width, 0))), ws=gpu(torch.zeros(512, dtype=torch.uint8)))
    with pytest.raises(ValueError):
        gs.gs_beam_select(gpu(torch.zeros(0, 9)), gpu(torch.zeros(0)), 3, width, **outs)


def test_workspaces_of_no_such_call(gs):  # noqa: F811
    assert gs.gs_beam_select_workspace_bytes(2, 4, 1000, 4) > 0
    for beams, width in ((4, (1 << 32) + 4), ((1 << 32) + 4, 4), (4, 257), (257, 4), (0, 4), (4, 0)):
        assert gs.gs_beam_select_workspace_bytes(2, beams, 1000, width) == 0
    assert gs.gs_scores_q8_workspace_bytes(5, 1000, (1 << 32) + 64) == 0
