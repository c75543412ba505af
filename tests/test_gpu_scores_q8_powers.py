"""gs_scores_q8 on rows whose blocks have very different powers of two, against products in 64 bits; tolerances as in
test_gpu_scores_q8.py.  Every block has a part of its own, so that no sum overflows: in some the centres and nodes meet with powers
whose product is ordinary, in the others one side has a large power and the other one zeros (whose scale is the least, 2^-127)."""
import pytest
import torch

from test_gpu_scores_q8 import DEV, INF, TORCH, check, gs  # noqa: F401

pytestmark = pytest.mark.gpu


def bytes_of(rows, columns, gen):
    """e4m3 values of every size, no NaN."""
    x = torch.randint(0, 256, (rows, columns), generator=gen, dtype=torch.uint8)
    return torch.where((x & 0x7f) == 0x7f, x & 0xfb, x)


def table(gs, rows, dim, live, high, zero, parts, seed, far=0.4):
    """Blocks of part "live" have the power `live`, those of part `zero` are zeros; the rest has the power `high`, or (1 - far of the rows)
    that of the live ones."""
    gen = torch.Generator().manual_seed(seed)
    t = gs.Table8.empty(rows, dim, DEV)
    data = torch.zeros(rows, t.data.shape[1], dtype=torch.uint8)
    data[:, :dim] = bytes_of(rows, dim, gen)
    scales = torch.zeros(rows, t.scales.shape[1], dtype=torch.uint8)
    spread = torch.rand(rows, generator=gen) < far
    for b, part in enumerate(parts):
        if part == zero:
            data[:, b * 128:(b + 1) * 128] = 0
            continue
        power = torch.full((rows,), live)
        if part != "live":
            power = torch.where(spread, high, live)
        scales[:, b] = (power + 127).clamp(0, 254).to(torch.uint8)
    t.data.view(torch.uint8).copy_(data)
    t.scales.view(torch.uint8).copy_(scales)
    return t


def both(gs, dim, center, node, parts, nodes, seed=1):
    """center, node: (power of the live blocks, of the high ones)."""
    t_in = table(gs, 60, dim, *center, "node", parts, seed)
    t_out = table(gs, nodes, dim, *node, "center", parts, seed + 1)
    return t_in, t_out


def parts_of(dim, order):
    blocks = -(-dim // 128)
    names = {"c": ["live", "center"], "n": ["node", "live"], "cn": ["center", "live", "node"], "nc": ["live", "node", "live", "center"]}[order]
    return [names[b % len(names)] for b in range(blocks)]


POWERS = {                                       # of centres and of nodes: live, high
    "20": ((0, 20), (0, 20)), "54": ((0, 54), (0, 54)), "60": ((0, 60), (0, 60)), "65": ((0, 65), (0, 66)), "75": ((0, 75), (0, 75)),
    "119": ((0, 119), (0, 119)), "c124": ((-24, 100), (24, 25)), "c125": ((-25, 100), (25, 25)), "c126": ((-26, 100), (26, 26)),
    "c127": ((-27, 100), (27, 27)), "c130": ((-30, 100), (30, 30)), "c200": ((-81, 119), (81, 100)), "n124": ((24, 25), (-24, 100)),
    "n125": ((25, 25), (-25, 100)), "n126": ((26, 26), (-26, 100)), "n127": ((27, 27), (-27, 100)), "n130": ((30, 30), (-30, 100)),
    "n200": ((81, 100), (-81, 119)), "zeros": ((0, 0), (0, 0)), "zeros large": ((100, 100), (-100, -100)), "zeros small": ((-100, -100), (100, 100)),
    "n least": ((119, 119), (-127, 100)), "c least": ((-127, 100), (119, 119)), "all": ((-127, 127), (119, 127)),
}


@pytest.mark.parametrize("name", list(POWERS))
@pytest.mark.parametrize("dim,order", [(256, "c"), (256, "n"), (200, "c"), (136, "n"), (384, "cn"), (260, "cn"), (640, "nc"), (1100, "cn")])
def test_blocks_far_apart(gs, dim, order, name):  # noqa: F811
    center, node = POWERS[name]
    t_in, t_out = both(gs, dim, center, node, parts_of(dim, order), 257)
    gen = torch.Generator().manual_seed(5)
    for centers in (1, 32, 33, 130, 300):
        ids = torch.randint(0, 60, (centers,), generator=gen, dtype=torch.int32).to(DEV)
        for dtype in TORCH:
            check(gs, t_in, t_out, ids, scale=2.0 ** -12, dtype=dtype)


@pytest.mark.parametrize("dim,order", [(256, "c"), (256, "n"), (384, "cn"), (640, "nc")])
@pytest.mark.parametrize("center,node", [((13, 73), (-127, -100)), ((73, 73), (-119, -99)), ((-119, -99), (73, 73)), ((-10, 60), (-100, -90)),
                                         ((-100, -90), (-10, 60)), ((60, 119), (0, 60))])
def test_small_and_large_scores(gs, dim, order, center, node):  # noqa: F811
    """Scores far from 1, beside blocks that meet zeros."""
    t_in, t_out = both(gs, dim, center, node, parts_of(dim, order), 300, seed=7)
    for centers in (20, 40, 200):
        check(gs, t_in, t_out, (torch.arange(centers, dtype=torch.int32) % 60).to(DEV))


@pytest.mark.parametrize("dim,order", [(256, "c"), (256, "n"), (384, "cn"), (1100, "nc")])
@pytest.mark.parametrize("name", ["60", "c200", "n200"])
def test_rows_far_apart_among_others(gs, dim, order, name):  # noqa: F811
    """One centre and one node with such blocks; NaN, masked nodes and centres that are no rows beside them."""
    center, node = POWERS[name]
    parts = parts_of(dim, order)
    t_in, t_out = both(gs, dim, (center[0], center[0]), (node[0], node[0]), parts, 3001)
    one_in, one_out = both(gs, dim, center, node, parts, 60, seed=3)
    for t, one, at in ((t_in, one_in, 17), (t_out, one_out, 1033)):
        row = int(one.scales.view(torch.uint8).amax(1).argmax())
        t.data.view(torch.uint8)[at] = one.data.view(torch.uint8)[row]
        t.scales.view(torch.uint8)[at] = one.scales.view(torch.uint8)[row]
    t_in.scales.view(torch.uint8)[5, -(-dim // 128) - 1] = 255
    t_out.scales.view(torch.uint8)[7, 0] = 255
    bias = torch.randn(3001, generator=torch.Generator().manual_seed(2)).to(DEV)
    bias[::9] = -INF
    for centers in (40, 300):
        ids = (torch.arange(centers, dtype=torch.int32) % 62).to(DEV)
        for dtype in TORCH:
            check(gs, t_in, t_out, ids, bias=bias, scale=2.0 ** -12, dtype=dtype)


@pytest.mark.parametrize("centers", [1, 32, 33, 300])
@pytest.mark.parametrize("dim", [256, 384])
def test_least_powers_that_count(gs, centers, dim):  # noqa: F811
    """Nodes' blocks of the least scale, 2^-127, that are no zeros, beside ordinary ones; and so for centres."""
    parts = ["node", "live", "center"][-(-dim // 128) * -1:]
    for center, node in (((119, 0), (-127, 0)), ((-127, 0), (119, 0))):
        t_in, t_out = both(gs, dim, center, node, parts, 500, seed=11)
        check(gs, t_in, t_out, (torch.arange(centers, dtype=torch.int32) % 60).to(DEV))
