"""What gs_quantize_rows, gs_scores_q8, gs_beam_select, gs_beam_reorder and their binding refuse, and the sizes they ask for: on the
host, before anything is enqueued.  Pointers are made up and never followed."""
import ctypes as C
import math
import os

import pytest
import torch

P = [C.c_void_p(1 << 20 | 256 * i) for i in range(12)]
BIG = C.c_size_t(1 << 62)
EINVAL, EWORKSPACE, EOVERFLOW = -1, -2, -3


@pytest.fixture(scope="module")
def lib():
    from paper_2407_15452_amd import binding, build
    if not os.path.exists(binding.LIB_PATH):
        build.build_lib()
    return binding.lib()


@pytest.fixture(scope="module")
def gs(lib):
    from paper_2407_15452_amd import binding
    return binding


def at(a):
    return C.c_void_p(a)


def quantize(lib, **k):
    a = dict(table=P[1], nodes=50, dim=64, dtype=0, ids=P[2], n=5, count=P[3], q=P[4], scales=P[5])
    a.update(k)
    return lib.gs_quantize_rows(a["table"], C.c_int64(a["nodes"]), C.c_int32(a["dim"]), C.c_int32(a["dtype"]), a["ids"], C.c_int64(a["n"]), a["count"],
                                a["q"], a["scales"], None)


@pytest.mark.parametrize("bad", [dict(table=None), dict(q=None), dict(scales=None), dict(table=at(264)), dict(q=at(264)), dict(scales=at(258)),
                                 dict(nodes=0), dict(nodes=1 << 31), dict(n=-1), dict(n=1 << 31), dict(dim=0), dict(dim=-4), dict(dim=66),
                                 dict(dim=8196), dict(dim=68, dtype=1), dict(dim=68, dtype=2), dict(dtype=3), dict(dtype=-1), dict(ids=None),
                                 dict(ids=None, count=None), dict(ids=None, n=50),
                                 dict(ids=at(258)), dict(count=at(260))], ids=str)
def test_quantize_refuses(lib, bad):
    assert quantize(lib, **bad) == EINVAL


def test_no_rows(lib):
    assert quantize(lib, n=0) == 0


def test_pitches(lib, gs):
    assert [lib.gs_q8_pitch(C.c_int32(d)) for d in (0, -1, 8193, 1, 16, 17, 100, 8192)] == [0, 0, 0, 16, 16, 32, 112, 8192]
    assert [lib.gs_q8_scale_pitch(C.c_int32(d)) for d in (0, 8193, 1, 128, 129, 256, 257, 512, 513, 8192)] == [0, 0, 1, 1, 2, 2, 4, 4, 8, 64]
    for d in range(1, 8193, 7):
        assert gs.Table8.pitches(d) == (lib.gs_q8_pitch(C.c_int32(d)), lib.gs_q8_scale_pitch(C.c_int32(d)))
    for d in (0, -5, 8193):
        with pytest.raises(ValueError):
            gs.Table8.pitches(d)


def scores(lib, **k):
    a = dict(q_in=P[1], s_in=P[2], num_in=100, q_out=P[3], s_out=P[4], nodes=50, dim=64, centers=P[5], n=8, bias=P[6], scale=1.0, out=P[7], dtype=0,
             ws=P[9], ws_bytes=BIG)
    a.update(k)
    return lib.gs_scores_q8(a["q_in"], a["s_in"], C.c_int64(a["num_in"]), a["q_out"], a["s_out"], C.c_int64(a["nodes"]), C.c_int32(a["dim"]),
                            a["centers"], C.c_int64(a["n"]), a["bias"], C.c_float(a["scale"]), a["out"], C.c_int32(a["dtype"]), a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("bad", [dict(q_in=None), dict(q_out=None), dict(s_in=None), dict(s_out=None), dict(q_in=at(264)), dict(q_out=at(264)),
                                 dict(s_in=at(258)), dict(s_out=at(257)), dict(num_in=0), dict(num_in=1 << 31), dict(nodes=0), dict(nodes=1 << 31),
                                 dict(n=-1), dict(n=1 << 31), dict(dim=0), dict(dim=8193), dict(centers=None), dict(out=None), dict(ws=None),
                                 dict(ws=at(128)), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf), dict(dtype=3),
                                 dict(dtype=-1), dict(out=at(258)), dict(out=at(257), dtype=1), dict(bias=at(258)), dict(centers=at(258))], ids=str)
def test_scores_refuses(lib, bad):
    assert scores(lib, **bad) == EINVAL


def test_scores_of_more_than_a_launch_takes(lib):
    for n in (1 << 21, (1 << 31) - 1):
        for nodes, dim in ((1, 16), (50, 64), (1000, 1024)):
            for dtype in (0, 1, 2):
                assert scores(lib, n=n, nodes=nodes, dim=dim, dtype=dtype) == EOVERFLOW


def test_scores_workspace(lib):
    for nodes in (1, 50, 10_000, 1_000_000):
        for dim in (4, 64, 128, 200, 1024, 8192):
            got = []
            for n in (1, 2, 16, 17, 32, 33, 64, 65, 128, 129, 256, 257, 1000, 4096, 100_000):
                need = lib.gs_scores_q8_workspace_bytes(C.c_int64(n), C.c_int64(nodes), C.c_int32(dim))
                assert need > 0 and need % 256 == 0
                assert scores(lib, n=n, nodes=nodes, dim=dim, ws_bytes=C.c_size_t(need - 1)) == EWORKSPACE
                got.append(need)
            assert got == sorted(got)
    for bad in ((-1, 5, 64), (5, 0, 64), (5, 5, 0), (5, 5, 8193)):
        assert lib.gs_scores_q8_workspace_bytes(C.c_int64(bad[0]), C.c_int64(bad[1]), C.c_int32(bad[2])) == 0


def select(lib, **k):
    a = dict(scores=P[1], groups=3, beams=4, n=50, dtype=0, logp=P[2], ended=P[3], width=5, parents=P[4], nodes=P[5], out=P[6], ws=P[9], ws_bytes=BIG)
    a.update(k)
    return lib.gs_beam_select(a["scores"], C.c_int64(a["groups"]), C.c_int32(a["beams"]), C.c_int64(a["n"]), C.c_int32(a["dtype"]), a["logp"], a["ended"],
                              C.c_int32(a["width"]), a["parents"], a["nodes"], a["out"], a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("bad", [dict(scores=None), dict(logp=None), dict(parents=None), dict(nodes=None), dict(out=None), dict(ws=None), dict(ws=at(128)),
                                 dict(scores=at(258)), dict(scores=at(257), dtype=1), dict(logp=at(258)), dict(parents=at(258)), dict(nodes=at(257)),
                                 dict(out=at(259)), dict(groups=-1), dict(groups=1 << 31), dict(beams=0), dict(beams=257), dict(n=0), dict(n=1 << 31),
                                 dict(width=0), dict(width=257), dict(dtype=3), dict(dtype=-1)], ids=str)
def test_select_refuses(lib, bad):
    assert select(lib, **bad) == EINVAL


@pytest.mark.parametrize("more", [dict(out=at(1 << 20), logp=at(1 << 20), width=5), dict(out=at((1 << 20) + 44), logp=at(1 << 20)),
                                  dict(out=at((1 << 20) - 56), logp=at(1 << 20)), dict(out=at((1 << 20) + 4), logp=at(1 << 20), width=4)], ids=str)
def test_select_refuses_overlaps(lib, more):
    assert select(lib, **more) == EINVAL


def test_select_sizes(lib):
    assert select(lib, groups=0) == 0
    assert select(lib, groups=1 << 22, beams=1) == EOVERFLOW and select(lib, groups=1 << 14, beams=256) == EOVERFLOW
    assert select(lib, groups=4_000_000, beams=1, n=(1 << 31) - 1) == EOVERFLOW               # workgroups
    for dtype in (0, 1, 2):
        for beams, n, width in ((1, 1, 1), (4, 10_000, 4), (8, 1_000_000, 8), (256, 70_001, 256), (1, (1 << 31) - 1, 16)):
            got = []
            for groups in (1, 2, 3, 16, 64, 65, 100, 500, 1000, 4000):
                need = lib.gs_beam_select_workspace_bytes(C.c_int64(groups), C.c_int32(beams), C.c_int64(n), C.c_int32(width), C.c_int32(dtype))
                assert need > 0 and need % 256 == 0
                assert select(lib, groups=groups, beams=beams, n=n, width=width, dtype=dtype, ws_bytes=C.c_size_t(need - 1)) in (EWORKSPACE, EOVERFLOW)
                got.append(need)
            assert got == sorted(got)


def reorder(lib, states, groups=2, beams=3, width=3, parents=P[1], nodes=P[2], count=None):
    from paper_2407_15452_amd.binding import StateStruct
    array = (StateStruct * max(1, len(states)))(*[StateStruct(*s) for s in states])
    return lib.gs_beam_reorder(array, C.c_int32(len(states) if count is None else count), C.c_int64(groups), C.c_int32(beams), C.c_int32(width), parents,
                               nodes, None)


A, B = 1 << 30, 1 << 31


@pytest.mark.parametrize("states,more", [
    ([(None, B, 8, -1)], {}), ([(A, B, -1, -1)], {}), ([(A, B, 1 << 40, -1)], {}), ([(A, None, 8, -1)], dict(width=4)), ([(A, A, 8, -1)], dict(width=2)),
    ([(A, B, 8, -1)], dict(groups=-1)), ([(A, B, 8, -1)], dict(beams=0)), ([(A, B, 8, -1)], dict(beams=257)), ([(A, B, 8, -1)], dict(width=0)),
    ([(A, B, 8, -1)], dict(width=257)), ([(A, B, 8, -1)], dict(parents=None)), ([(A, B, 8, -1)], dict(parents=at(258))), ([(A, B, 8, -1)], dict(count=-1)),
    ([(A, B, 8, -2)], {}), ([(A, B, 8, 2)], {}), ([(A, B, 8, 8)], {}), ([(A, B, 10, 4)], {}), ([(A + 2, B, 8, 4)], {}), ([(A, B + 1, 8, 4)], {}),
    ([(A, B, 8, 4)], dict(nodes=None)), ([(A, B, 8, 4)], dict(nodes=at(258))),
    # overlaps: an output and its state, an output and another state, two outputs, a state moved in place and another's output
    ([(A, A + 8, 8, -1)], {}), ([(A, A - 8, 8, -1)], {}), ([(A, A + 47, 8, -1)], {}), ([(A, B, 8, -1), (B + 40, None, 8, -1)], {}),
    ([(A, B, 8, -1), (A + 4096, B + 47, 8, -1)], {}), ([(A, None, 8, -1), (B, A + 8, 8, -1)], {}), ([(A, None, 8, -1), (A, None, 8, -1)], {}),
    ([(A, None, 8, -1), (A + 40, None, 8, -1)], {}), ([(A, B, 8, -1)] * 2, {}),
    # an output and the choice itself
    ([(A, B, 8, -1)], dict(parents=at(B + 44))), ([(A, B, 8, -1)], dict(nodes=at(B - 20))), ([(A, None, 8, 4)], dict(parents=at(A)))], ids=str)
def test_reorder_refuses(lib, states, more):
    assert reorder(lib, states, **more) == EINVAL


def test_reorder_of_nothing(lib):
    assert reorder(lib, []) == 0 and reorder(lib, [(A, B, 8, 4)], groups=0) == 0 and reorder(lib, [(None, None, 0, -1)]) == 0
    assert reorder(lib, [(None, None, 0, -1)], width=7) == 0 and reorder(lib, [(None, None, 0, -1), (None, None, 0, -1)]) == 0
    assert lib.gs_beam_reorder(None, C.c_int32(1), C.c_int64(1), C.c_int32(1), C.c_int32(1), P[1], P[2], None) == EINVAL
    assert reorder(lib, [(A, B, 8, -1)], groups=1 << 21, beams=2) == EOVERFLOW


# ---- the binding, with tensors that say they are on a GPU --------------------------

class Elsewhere(torch.Tensor):
    is_cuda = property(lambda self: True)
    device = property(lambda self: torch.device("cuda", self.place))


def gpu(t, place=0):
    t = t.as_subclass(Elsewhere)
    t.place = place
    return t


def table8(gs, n=5, dim=64, place=0):
    pitch, scale_pitch = gs.Table8.pitches(dim)
    return gs.Table8(gpu(torch.zeros(n, pitch, dtype=torch.uint8).view(torch.float8_e4m3fn), place),
                  gpu(torch.zeros(n, scale_pitch, dtype=torch.uint8).view(torch.float8_e8m0fnu), place), dim)


def test_tables_are_checked(gs):
    data = gpu(torch.zeros(5, 64, dtype=torch.uint8).view(torch.float8_e4m3fn))
    scales = gpu(torch.zeros(5, 1, dtype=torch.uint8).view(torch.float8_e8m0fnu))
    assert gs.Table8(data, scales, 64).num_nodes == 5
    for bad in ((data, scales, 65), (data, scales, 48), (data[:4], scales, 64), (data, gpu(scales.expand(5, 2).contiguous()), 64),
                (data, gpu(torch.zeros(5, 1, dtype=torch.uint8).view(torch.float8_e8m0fnu), 1), 64)):
        with pytest.raises(ValueError):
            gs.Table8(*bad)
    for bad in ((data.view(torch.uint8), scales, 64), (data, scales.view(torch.uint8), 64), (torch.zeros(5, 64), scales, 64)):
        with pytest.raises(TypeError):
            gs.Table8(*bad)


def test_binding_refuses_shapes_and_devices(gs, monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    i32, f32 = torch.int32, torch.float32
    t, other, far = table8(gs), table8(gs, dim=80), table8(gs, place=1)
    ids = gpu(torch.zeros(3, dtype=i32))
    wide = gpu(torch.zeros(5, 64))
    with pytest.raises(ValueError):
        gs.gs_quantize_rows(wide, ids=ids)                                  # no copy to write to
    for out in (other, table8(gs, n=6), far):
        with pytest.raises(ValueError):
            gs.gs_quantize_rows(wide, ids=ids, out=out)
    with pytest.raises(ValueError):
        gs.gs_quantize_rows(gpu(torch.zeros(64)), out=t)
    for bad in (dict(t_out=other), dict(t_out=far), dict(bias=gpu(torch.zeros(4))), dict(centers=gpu(torch.zeros(3, dtype=i32), 1)),
                dict(out=gpu(torch.zeros(3, 4))), dict(out=gpu(torch.zeros(3, 5)), dtype=torch.bfloat16)):
        a = dict(t_in=t, t_out=t, centers=ids)
        a.update(bad)
        with pytest.raises(ValueError):
            gs.gs_scores_q8(**a)
    z, logp = gpu(torch.zeros(6, 9)), gpu(torch.zeros(6))
    for bad in (dict(beams=4), dict(beams=0), dict(logp=gpu(torch.zeros(5))), dict(logp=gpu(torch.zeros(6), 1)), dict(ended=gpu(torch.zeros(2, dtype=torch.bool))),
                dict(scores=gpu(torch.zeros(6))), dict(parents_out=gpu(torch.zeros(2, 3, dtype=i32))), dict(parents_out=gpu(torch.zeros(2, 4)))):
        a = dict(scores=z, logp=logp, beams=3, width=4)
        a.update(bad)
        with pytest.raises(ValueError):
            gs.gs_beam_select(**a)
    parents = gpu(torch.zeros(2, 3, dtype=i32))
    x = gpu(torch.zeros(6, 4, dtype=i32))
    for bad in (dict(parents=gpu(torch.zeros(6, dtype=i32))), dict(nodes=gpu(torch.zeros(2, 2, dtype=i32))), dict(outs=[x, x]), dict(columns=[0, 1]),
                dict(beams=2), dict(states=[gpu(torch.zeros(5, 4))]), dict(outs=[gpu(torch.zeros(6, 5, dtype=i32))]), dict(outs=[gpu(torch.zeros(6, 4))]),
                dict(columns=[4]), dict(columns=[-1]), dict(columns=[0]), dict(states=[gpu(torch.zeros(6, 4))], columns=[0], nodes=parents),
                dict(states=[gpu(torch.zeros(6, 4, dtype=i32), 1)])):
        a = dict(states=[x], parents=parents, beams=3)
        a.update(bad)
        with pytest.raises(ValueError):
            gs.gs_beam_reorder(**a)
    with pytest.raises(TypeError):
        gs.gs_beam_reorder([torch.zeros(6, 4)], torch.zeros(2, 3, dtype=i32), 3)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)             # another device than the tensors'
    for call in (lambda: gs.gs_quantize_rows(wide, out=t), lambda: gs.gs_scores_q8(t, t, ids, out=gpu(torch.zeros(3, 5))),
                 lambda: gs.gs_beam_reorder([x], parents, 3)):
        with pytest.raises(ValueError):
            call()
