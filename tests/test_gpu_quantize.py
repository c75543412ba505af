"""gs_quantize_rows against its definition, computed here in 64 bits over the list of the format's values: every byte equal."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def gs():
    from paper_2407_15452_amd import binding
    binding.lib()
    return binding


# the positive values of e4m3 by their byte: 0x00 to 0x7e; 3 bits of fraction, exponent bias 7
VALUES = np.array([(m / 8) * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)][:127])


def nearest(x):
    """Bytes of the values nearest to |x| <= 448, ties to the even byte, with the sign."""
    a = np.abs(x)
    hi = np.clip(np.searchsorted(VALUES, a), 1, 126)
    lo = hi - 1
    below, above = a - VALUES[lo], VALUES[hi] - a
    at = np.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)
    return (at | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def definition(x, rows=None):
    """(data, scales) bytes of the rows of x, in 64 bits."""
    n, dim = x.shape
    pitch, blocks = -(-dim // 16) * 16, -(-dim // 128)
    data = np.zeros((n, pitch), np.uint8)
    scales = np.zeros((n, blocks if blocks <= 2 else -(-blocks // 4) * 4), np.uint8)
    for b in range(blocks):
        part = x[:, 128 * b:128 * b + 128]
        fine = np.isfinite(part).all(axis=1)
        most = np.where(fine, np.abs(np.where(np.isfinite(part), part, 0)).max(axis=1), 1.0)
        power = np.full(n, -127)
        for e in range(-127, 121):                       # the least power of two with most <= 448 * 2^e
            power[most > np.ldexp(448.0, e)] = e + 1
        scales[:, b] = np.where(fine, power + 127, 255)
        data[:, 128 * b:128 * b + part.shape[1]] = np.where(fine[:, None], nearest(np.where(fine[:, None], np.ldexp(part, -power[:, None]), 0)), 0)
    return data, scales


def check(gs, table, got, rows=None, before=None):
    data, scales = definition(table.double().cpu().numpy())
    if rows is not None:
        keep = np.ones(len(data), bool)
        keep[rows] = False
        data[keep], scales[keep] = before[0][keep], before[1][keep]
    assert np.array_equal(got.scales.view(torch.uint8).cpu().numpy(), scales)
    mine = got.data.view(torch.uint8).cpu().numpy()
    assert np.array_equal(mine & 127, data & 127)
    assert np.array_equal((mine ^ data)[(data & 127) != 0], np.zeros(((data & 127) != 0).sum(), np.uint8))      # signs, but of zeros


@pytest.mark.parametrize("dtype", list(TORCH))
@pytest.mark.parametrize("n,dim", [(1, 8), (1, 64), (3, 120), (1000, 128), (77, 136), (50, 200), (5, 256), (9, 264), (33, 520), (300, 1024), (2, 8192), (70_001, 16)])
def test_whole_table(gs, dtype, n, dim):
    gen = torch.Generator().manual_seed(n * 10_000 + dim)
    x = torch.randn(n, dim, generator=gen) * torch.exp(2 * torch.randn(n, 1, generator=gen))
    x = x.to(TORCH[dtype]).to(DEV)
    check(gs, x, gs.gs_quantize_rows(x))


@pytest.mark.parametrize("n,dim", [(7, 4), (5, 12), (600, 100), (11, 132), (3, 8188)])
def test_columns_of_fp32_by_four(gs, n, dim):
    x = torch.randn(n, dim, generator=torch.Generator().manual_seed(dim)).to(DEV)
    check(gs, x, gs.gs_quantize_rows(x))


@pytest.mark.parametrize("dtype", list(TORCH))
def test_every_power_and_its_borders(gs, dtype):
    """Rows whose largest value is 448 times a power of two, the next above, the next below; ties between two of the format's values."""
    t = TORCH[dtype]
    least, most = (-149, 119) if dtype == "f32" else (-133, 119) if dtype == "bf16" else (-24, 7)
    rows = []
    for e in range(least - 9, most + 1):
        top = torch.tensor(448.0, dtype=torch.float64).mul(2.0 ** e).to(t)
        if not torch.isfinite(top) or top == 0:
            continue
        for edge in (top, torch.nextafter(top.float(), torch.tensor(torch.inf)).to(t) if dtype == "f32" else top * (1 + torch.finfo(t).eps),
                     top * (1 - torch.finfo(t).eps)):
            if not torch.isfinite(edge):
                continue
            steps = torch.linspace(-1, 1, 123, dtype=torch.float64) * float(edge)
            ties = float(top) / 448.0 * torch.tensor([17 * 16.0, 19 * 8.0, 2.0 ** -10, 3 * 2.0 ** -10, -(2.0 ** -10)], dtype=torch.float64)
            row = torch.cat([steps.to(t), ties.to(t)])
            row[0] = edge
            rows.append(row)
    x = torch.stack(rows).to(DEV)
    check(gs, x, gs.gs_quantize_rows(x))


@pytest.mark.parametrize("dtype", list(TORCH))
def test_nothing_infinite_and_none(gs, dtype):
    x = torch.randn(12, 400, generator=torch.Generator().manual_seed(3)).to(TORCH[dtype])
    x[0] = 0
    x[1] = -0.0
    x[2, 130] = torch.inf
    x[3, 0] = -torch.inf
    x[4, 399] = torch.nan
    x[5, :128] = torch.nan
    x[6, 128:256] = 0
    x[7] = torch.finfo(TORCH[dtype]).max
    x[8] = torch.finfo(TORCH[dtype]).tiny
    x[9] = torch.finfo(TORCH[dtype]).smallest_normal / 2
    x = x.to(DEV)
    got = gs.gs_quantize_rows(x)
    check(gs, x, got)
    assert got.scales.view(torch.uint8)[2].tolist()[1] == 255 and got.scales.view(torch.uint8)[2].tolist()[0] != 255


@pytest.mark.parametrize("dtype", list(TORCH))
def test_rows_by_their_ids(gs, dtype):
    n, dim = 500, 200
    gen = torch.Generator().manual_seed(5)
    old, x = (torch.randn(n, dim, generator=gen).to(TORCH[dtype]).to(DEV) for _ in range(2))
    ids = torch.tensor([3, 499, 0, 77, 77, -1, 500, 2 ** 31 - 1, -2 ** 31, 250], dtype=torch.int32, device=DEV)
    for count, rows in ((None, [3, 499, 0, 77, 250]), (4, [3, 499, 0, 77]), (0, []), (-5, []), (100, [3, 499, 0, 77, 250])):
        copy = gs.gs_quantize_rows(old)
        before = copy.data.view(torch.uint8).cpu().numpy().copy(), copy.scales.view(torch.uint8).cpu().numpy().copy()
        device_count = None if count is None else torch.tensor([count], dtype=torch.int64, device=DEV)
        assert gs.gs_quantize_rows(x, ids=ids, count=device_count, out=copy) is copy
        check(gs, x, copy, rows, before)


def test_rows_that_a_step_changed(gs):
    """With the ids and the count of gs_unique_ids the copy is that of the whole table."""
    n, dim = 3000, 64
    x = torch.randn(n, dim, generator=torch.Generator().manual_seed(8)).to(DEV)
    copy = gs.gs_quantize_rows(x)
    touched = torch.randint(0, n, (700,), generator=torch.Generator().manual_seed(9), dtype=torch.int32).to(DEV)
    ids, count = gs.gs_unique_ids(touched, n)[:2]
    gs.gs_put_rows(x, ids, torch.randn(700, dim, generator=torch.Generator().manual_seed(10)).to(DEV), 1.0, count=count)
    gs.gs_quantize_rows(x, ids=ids, count=count, out=copy)
    whole = gs.gs_quantize_rows(x)
    assert torch.equal(copy.data.view(torch.uint8), whole.data.view(torch.uint8))
    assert torch.equal(copy.scales.view(torch.uint8), whole.scales.view(torch.uint8))


def test_offsets_beyond_31_bits(gs):
    """2.2 GB of bytes from 4.4 GB of halves: the last rows, and rows around byte 2^31 and 2^32."""
    n, dim = 275_000, 8000
    x = torch.zeros(n, dim, dtype=torch.float16, device=DEV)
    rows = [0, 134_217, 134_218, 268_434, 268_435, 268_436, n - 1]
    part = torch.randn(len(rows), dim, generator=torch.Generator().manual_seed(2)).half().to(DEV)
    x[rows] = part
    got = gs.gs_quantize_rows(x)
    data, scales = definition(part.double().cpu().numpy())
    assert np.array_equal(got.data.view(torch.uint8)[rows].cpu().numpy() & 127, data & 127)
    assert np.array_equal(got.scales.view(torch.uint8)[rows].cpu().numpy(), scales)
    assert int((got.data.view(torch.uint8)[1:1000] != 0).sum()) == 0
