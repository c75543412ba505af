"""gs_beam_reorder on states that take more workgroups than one launch has room for."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(scope="module")
def gs():
    from paper_2407_15452_amd import binding
    binding.lib()
    return binding


def some(rows, columns):
    x = torch.empty(rows, columns, dtype=torch.uint8, device=DEV)
    gen = torch.Generator(device=DEV).manual_seed(1)
    for r in range(rows):
        x[r].random_(0, 256, generator=gen)
    return x


def same(x, row, y, other):
    return all(torch.equal(x[row, lo:lo + (1 << 30)], y[other, lo:lo + (1 << 30)]) for lo in range(0, x.shape[1], 1 << 30))


def test_in_place(gs):
    """Rows of an odd number of bytes, 256 bytes a workgroup; a small state behind the large one."""
    state, small = some(4, (1 << 30) + 1), torch.arange(4 * 6, dtype=torch.int32, device=DEV).view(4, 6)
    before, small_before = state.clone(), small.clone()
    parents, nodes = torch.tensor([[1, 0, 3, 0]], dtype=torch.int32, device=DEV), torch.tensor([[7, 8, 9, 10]], dtype=torch.int32, device=DEV)
    gs.gs_beam_reorder([state, small], parents, 4, nodes=nodes, columns=[None, 5])
    for row, parent in enumerate(parents[0].tolist()):
        assert same(state, row, before, parent)
        assert torch.equal(small[row, :5], small_before[parent, :5]) and int(small[row, 5]) == 7 + row


def test_to_others(gs):
    """1 KB a workgroup, in bytes; a parent that is none."""
    state = some(2, (1 << 32) + 3)
    out = torch.full((5, state.shape[1]), 3, dtype=torch.uint8, device=DEV)
    parents = torch.tensor([[1, 0, -1, 1, 0]], dtype=torch.int32, device=DEV)
    gs.gs_beam_reorder([state], parents, 2, outs=[out])
    for row, parent in enumerate(parents[0].tolist()):
        assert bool((out[row, ::4099] == 3).all()) and bool((out[row, -4:] == 3).all()) if parent < 0 else same(out, row, state, parent)
