"""What the full-softmax operators and their binding refuse, on the host: pointers are made up and never followed."""
import ctypes as C
import os

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


def test_more_pairs_than_a_launch_takes():
    from paper_2407_15452_amd import binding, build
    if not os.path.exists(binding.LIB_PATH):
        build.build_lib()
    at = [C.c_void_p(256 * i) for i in range(10)]
    for dtype in (0, 1, 2):
        for dim in (8, 64, 256):
            for grads in ((at[7], at[8]), (None, at[8]), (at[7], None), (None, None)):
                for pairs in ((1 << 26) - 255, 1 << 26, (1 << 31) - 1):
                    assert binding.lib().gs_softmax_loss(
                        at[1], C.c_int64(100), at[2], C.c_int64(50), C.c_int32(dim), C.c_int32(dtype), at[3], at[4], C.c_int64(pairs), None,
                        C.c_float(1.0), at[6], *grads, C.c_float(1.0), at[9], C.c_size_t(1 << 62), None) == binding.GS_EOVERFLOW


class Elsewhere(torch.Tensor):
    """Says that it is on a GPU, of a number of its own."""
    is_cuda = property(lambda self: True)
    device = property(lambda self: torch.device("cuda", self.place))


def on_gpu(place, n=4):
    t = torch.zeros(n).as_subclass(Elsewhere)
    t.place = place
    return t


def test_gradients_of_one_device():
    from paper_2407_15452_amd import binding as gs
    a, b, other = on_gpu(0), on_gpu(0), on_gpu(1)
    assert gs.GradList([a, b], [None, on_gpu(0)]).device == torch.device("cuda", 0)
    for grads, outs in (([a, other], None), ([a, b], [other, None]), ([a, b], [None, other])):
        with pytest.raises(ValueError):
            gs.GradList(grads, outs)
