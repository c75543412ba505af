"""gs_clip_grads where a workgroup takes several units of work, over the borders of tensors, formats and alignments.

Bounds: the norm to 1e-14 as in test_gpu_clip.py.  The factor is fp64 and so is the product: it is off by the norm's 1e-14 and
three roundings of 2^-53.  fp32 elements are then rounded once, 2^-24; 16-bit ones to fp32 (2^-24) and to their format (u)."""
import math

import pytest
import torch

from test_gpu_clip import DEV, gs, norm_of, tensors  # noqa: F401

pytestmark = pytest.mark.gpu


def check_tight(got, was, factor):
    for g, w in zip(got, was):
        want = w.cpu().double() * factor
        u = torch.finfo(g.dtype).eps / 2
        more = 0.0 if g.dtype == torch.float32 else 2.0 ** -24 * (1 + u)
        least = 2.0 ** -25 if g.dtype == torch.float16 else 2.0 ** -149 if g.dtype == torch.float32 else 2.0 ** -134
        assert torch.all((g.cpu().double() - want).abs() <= (u + more + 1.1e-14) * want.abs() + least)


# 1024 workgroups share the units, 32 KB each, the last of a tensor less
@pytest.mark.parametrize("fmts", [("f32",), ("bf16",), ("f32", "bf16", "f16")], ids="-".join)
@pytest.mark.parametrize("sizes", [[7_000_003, 6_000_001, 7_000_000], [3 + i % 50 for i in range(3000)] + [1_000_003, 5, 2_000_001, 1, 900_000],
                                   [1_500_000] + [16_385, 1, 0, 33_000] * 100 + [8_000_000]], ids=["three", "small-then-large", "mixed"])
@pytest.mark.parametrize("shift", [0, 1])
def test_units_of_several_tensors(gs, sizes, fmts, shift):  # noqa: F811
    grads = tensors(sizes, fmts, shift=shift)
    was = [t.clone() for t in grads]
    norm = norm_of(grads)
    outs = [torch.full_like(t, 7.0) for t in grads]
    got = gs.gs_clip_grads(gs.GradList(grads, outs), 0.3 * norm)
    assert abs(got.item() - norm) <= 1e-14 * norm
    check_tight(outs, was, 0.3)
    assert gs.gs_clip_grads(gs.GradList(grads, outs), 2 * norm).item() == got.item()                 # copied
    assert all(torch.equal(a, b) for a, b in zip(outs, was)) and all(torch.equal(a, b) for a, b in zip(grads, was))
    assert gs.gs_clip_grads(grads, 0.3 * norm).item() == got.item()
    check_tight(grads, was, 0.3)


@pytest.mark.parametrize("fmt", ["f32", "bf16", "f16"])
def test_elements_are_scaled_in_64_bits(gs, fmt):  # noqa: F811
    """Factors that are no floats: one rounding for an fp32 element, where a factor of fp32 would make three of them."""
    for seed, part in ((1, 0.1), (2, 1 / 3), (3, 0.7)):
        grads = tensors([50_001, 77], (fmt,), seed=seed)
        was = [t.clone() for t in grads]
        gs.gs_clip_grads(grads, part * norm_of(grads))
        check_tight(grads, was, part)


def test_a_tensor_beyond_31_bits(gs):  # noqa: F811
    n = (1 << 31) + 1029
    x = torch.full((n,), 0.5, dtype=torch.bfloat16, device=DEV)
    x[-1], x[1 << 31] = 3.0, -2.0
    norm = math.sqrt((n - 2) * 0.25 + 13.0)
    got = gs.gs_clip_grads([x[3:], x[:3]], norm / 2)
    assert abs(got.item() - norm) <= 1e-14 * norm
    assert float(x[-1]) == 1.5 and float(x[1 << 31]) == -1.0
    x[-1] = x[1 << 31] = 0.25
    assert all(bool((x[lo:lo + (1 << 28)] == 0.25).all()) for lo in range(0, n, 1 << 28))
