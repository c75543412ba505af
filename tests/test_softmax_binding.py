"""What the binding of the full-softmax operators refuses by itself, without a GPU."""
import pytest
import torch


def test_gradients_are_asked_for_by_name():
    from paper_2407_15452_amd import binding as gs
    f, ids = torch.zeros(4, 8), torch.zeros(3, dtype=torch.int32)
    for name in ("both", "", "g_in"):
        with pytest.raises(ValueError):
            gs.gs_softmax_loss(f, f, ids, ids, want_grad=name)
    for name in ("in", "out", True, False):
        with pytest.raises(TypeError):                       # the tensors are not on the GPU
            gs.gs_softmax_loss(f, f, ids, ids, want_grad=name)
