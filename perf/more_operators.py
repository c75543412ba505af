"""Answers from 8-bit tables, and the best walks by beam search, as cases that can be timed.

A table that only answers can be kept in 8 bits: rows of e4m3 values with a power of two for each block of 128 columns.  Two
operators make and use such tables: rows are quantised (all of them, or the ones that a training step has changed), and centres
are scored against every node.  Two more turn scores into walks: the best continuations of a group's walks over all of them and
all nodes are selected, and what is kept for each walk follows the choice.  Each case is one call.  ``run`` computes it in
elementary torch operations, or, where ``own`` is true, with the entry points of ``paper_2407_15452_amd.binding``; both take the
same inputs.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
INF = float("inf")
BLOCK = 128


def _pitch(dim):
    """Columns of a stored row: a multiple of 16."""
    return (dim + 15) // 16 * 16


def _scale_pitch(dim):
    """Scales of a stored row: 1, 2 or a multiple of 4."""
    blocks = (dim + BLOCK - 1) // BLOCK
    return blocks if blocks <= 2 else (blocks + 3) // 4 * 4


def _quantize(nodes, rows, dim, dtype, **more):
    """rows: how many rows, chosen by their ids, are quantised again; 0: the whole table."""
    return {"op": "quantize", "nodes": nodes, "rows": rows, "dim": dim, "dtype": dtype, **more}


def _scores(centers, nodes, dim, dtype, bias=False, **more):
    return {"op": "scores", "centers": centers, "nodes": nodes, "dim": dim, "dtype": dtype, "bias": bias, **more}


def _select(groups, beams, nodes, width, dtype, **more):
    return {"op": "select", "groups": groups, "beams": beams, "nodes": nodes, "width": width, "dtype": dtype, **more}


def _reorder(groups, beams, width, states, columns, **more):
    """states: how many tensors of `columns` fp32 values per walk, beside the walks themselves."""
    return {"op": "reorder", "groups": groups, "beams": beams, "width": width, "states": states, "columns": columns, **more}


def listed():
    return [
        # the rows that a small training step has changed, quantised again in their 8-bit copy: latency counts
        _quantize(10_000, 256, 128, "f32", name="quantize-rows"),
        # a table of a million nodes, whole, after training
        _quantize(1_000_000, 0, 128, "bf16", name="quantize-1m"),
        # one query against a million nodes, as a recommender answers it: one read of the table
        _scores(1, 1_000_000, 128, "f32", name="q8-one"),
        # a batch of queries with popularity offsets, some nodes no answers: as many scores as fit the memory of the next step
        _scores(256, 1_000_000, 128, "f32", bias=True, name="q8-256"),
        # ragged: rows of 200, an odd number of nodes, fp16 scores
        _scores(777, 50_021, 200, "f16", bias=True, name="q8-ragged"),
        # rows made of features (text, images) beside the graph's: wide ones, bfloat16 scores
        _scores(4096, 50_000, 1024, "bf16", name="q8-wide"),
        # the widest and the most of them: what the matrix instructions take
        _scores(8192, 32_768, 2048, "bf16", name="q8-most"),
        # one search of four walks on the smallest graph: latency
        _select(1, 4, 10_000, 4, "f32", name="select-one"),
        # the first step of many searches: one walk each, the sixteen best nodes, bfloat16 scores with many equal ones
        _select(256, 1, 100_003, 16, "bf16", name="select-first"),
        # a later step of eight searches over a large graph; walks that have ended among them
        _select(8, 8, 1_000_000, 8, "f32", name="select-8x8"),
        # what one search keeps: its walks and a row for each
        _reorder(1, 4, 4, 1, 128, name="reorder-one"),
        # many searches with much kept for each walk, such as every row it has passed
        _reorder(64, 8, 8, 6, 32_768, name="reorder-many"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(["quantize", "scores", "scores", "scores", "select", "select", "reorder"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    nodes = _log(rng, 64, 1_000_000)
    dim = 8 * _log(rng, 1, 256)
    if op == "quantize":
        dim = dim if dtype != "f32" else 4 * _log(rng, 2, 512)
        nodes = min(nodes, 128_000_000 // dim)
        return _quantize(nodes, 0 if rng.random() < 0.5 else _log(rng, 1, nodes), dim, dtype)
    if op == "scores":
        nodes = min(nodes, 512_000_000 // dim)
        most = min(8192, 256_000_000 // nodes, 8192 * 32_768 * 2048 // (nodes * dim))
        return _scores(_log(rng, 1, max(1, most)), nodes, dim, dtype, bias=rng.random() < 0.4)
    beams, width = _log(rng, 1, 32), _log(rng, 1, 64)
    if op == "select":
        return _select(_log(rng, 1, max(1, min(512, 64_000_000 // (beams * nodes)))), beams, nodes, width, dtype)
    groups, states, columns = _log(rng, 1, 256), rng.randint(1, 8), _log(rng, 1, 65_536)
    return _reorder(max(1, min(groups, 100_000_000 // (states * columns * max(beams, width)))), beams, width, states, columns)


def _uniform(gen, *shape):
    return torch.rand(*shape, generator=gen, device=DEV)


def _rows(gen, n, dim):
    """Trained rows: of different lengths, as nodes are of different degrees."""
    x = torch.randn(n, dim, generator=gen, device=DEV)
    return x * (math.sqrt(2.0 / math.sqrt(dim)) * torch.exp(0.5 * torch.randn(n, 1, generator=gen, device=DEV)))


def _power_of_two(power):
    """2^power as fp32, by its bits: power from -126 to 127."""
    return ((power.int() + 127) << 23).view(torch.float32)


def _plain_quantize(x):
    """Rows in 8 bits: e4m3 values [n, pitch] and exponents e8m0 [n, scale pitch], by blocks of 128 columns.  The scale of a block is
    the least power of two by which its largest value is at most 448; NaN (with zeros) where a block holds infinity or NaN."""
    n, dim = x.shape
    blocks = (dim + BLOCK - 1) // BLOCK
    x = torch.nn.functional.pad(x.float(), (0, blocks * BLOCK - dim)).view(n, blocks, BLOCK)
    most = x.abs().amax(dim=2)
    fine = torch.isfinite(x).all(dim=2)
    part, power = torch.frexp(torch.where(fine, most, 1.0))
    power = (power - torch.where(part <= 0.875, 9, 8)).masked_fill(most == 0, -127).clamp(min=-127)
    q = (x * _power_of_two(-power)[:, :, None]).masked_fill(~fine[:, :, None], 0.0)
    q = q.view(n, blocks * BLOCK)[:, :_pitch(dim)].contiguous().to(E4M3)
    scales = torch.where(fine, power + 127, 255).to(torch.uint8)
    return q, torch.nn.functional.pad(scales, (0, _scale_pitch(dim) - blocks)).view(E8M0)


def _table8(gen, n, dim):
    q, scales = [], []
    for lo in range(0, n, 65_536):                                # in pieces: the wide ones take much memory
        part = _plain_quantize(_rows(gen, min(65_536, n - lo), dim))
        q.append(part[0].view(torch.uint8))
        scales.append(part[1].view(torch.uint8))
    return torch.cat(q).view(E4M3), torch.cat(scales).view(E8M0)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s = dict(case)
    if case["op"] == "quantize":
        n, dim = case["nodes"], case["dim"]
        s["table"] = _rows(gen, n, dim).to(DTYPES[case["dtype"]])
        s["ids"] = None
        if case["rows"]:
            s["ids"] = torch.sort(torch.randperm(n, generator=gen, device=DEV)[:case["rows"]]).values.to(torch.int32)
        old = _plain_quantize(s["table"][:1])                     # what the copy holds beforehand
        s["q"] = old[0].view(torch.uint8).repeat(n, 1).view(E4M3)
        s["scales"] = old[1].view(torch.uint8).repeat(n, 1).view(E8M0)
    elif case["op"] == "scores":
        n, dim, rows = case["nodes"], case["dim"], max(1, min(case["nodes"], 100_000))
        s["q_in"], s["scales_in"] = _table8(gen, rows, dim)
        s["q_out"], s["scales_out"] = _table8(gen, n, dim)
        s["centers"] = (_uniform(gen, case["centers"]) * rows).to(torch.int32).clamp_(max=rows - 1)
        s["bias"] = None
        if case["bias"]:                                          # offsets by popularity; three nodes in ten are no answers
            out = _uniform(gen, n) < 0.3
            out[n // 2] = False
            s["bias"] = (0.5 * torch.randn(n, generator=gen, device=DEV)).masked_fill(out, -INF)
        s["scale"] = 1.0
    elif case["op"] == "select":
        g, b, n = case["groups"], case["beams"], case["nodes"]
        z = 2.0 * torch.randn(g * b, n, generator=gen, device=DEV)
        z.masked_fill_(_uniform(gen, g * b, n) < 0.1, -INF)       # nodes that are no answers
        s["scores"] = z.to(DTYPES[case["dtype"]])
        logp = -20.0 * _uniform(gen, g, b)
        ended = _uniform(gen, g, b) < 0.1
        if b > 1:
            logp[:, 1:].masked_fill_(_uniform(gen, g, b - 1) < 0.05, -INF)      # fewer walks than places so far
            ended[:, 0] = False
        s["logp"] = logp.reshape(-1).contiguous()
        s["ended"] = ended.reshape(-1).contiguous() if b > 1 else None
    else:
        g, b, k, length = case["groups"], case["beams"], case["width"], 80
        s["column"] = 40
        walks = torch.randint(0, 1_000_000, (g * b, length), generator=gen, device=DEV, dtype=torch.int32)
        walks[:, s["column"]:] = -1
        s["states"] = [walks] + [torch.randn(g * b, case["columns"], generator=gen, device=DEV) for _ in range(case["states"])]
        s["outs"] = [torch.zeros(g * k, *x.shape[1:], dtype=x.dtype, device=DEV) for x in s["states"]]
        s["parents"] = (_uniform(gen, g, k) ** 2 * b).to(torch.int32).clamp_(max=b - 1)     # good walks go on in several ways
        s["nodes"] = torch.randint(0, 1_000_000, (g, k), generator=gen, device=DEV, dtype=torch.int32)
    return s


def _own(s):
    from paper_2407_15452_amd import binding as gs
    if s["op"] == "quantize":
        t = gs.Table8(s["q"], s["scales"], s["dim"])
        gs.gs_quantize_rows(s["table"], ids=s["ids"], out=t)
        return {"q": t.data, "scales": t.scales}
    if s["op"] == "scores":
        a, b = gs.Table8(s["q_in"], s["scales_in"], s["dim"]), gs.Table8(s["q_out"], s["scales_out"], s["dim"])
        return {"scores": gs.gs_scores_q8(a, b, s["centers"], bias=s["bias"], scale=s["scale"], dtype=DTYPES[s["dtype"]])}
    if s["op"] == "select":
        parents, nodes, logp = gs.gs_beam_select(s["scores"], s["logp"], s["beams"], s["width"], ended=s["ended"])
        return {"parents": parents, "nodes": nodes, "logp": logp}
    gs.gs_beam_reorder(s["states"], s["parents"], s["beams"], outs=s["outs"], nodes=s["nodes"], columns=[s["column"]] + [None] * (len(s["states"]) - 1))
    return {"states": s["outs"]}


def _plain_rows(q, scales, dim):
    """8-bit rows as the fp32 values that they stand for."""
    at = torch.arange(dim, device=DEV) // BLOCK
    return q.float()[:, :dim] * scales.float()[:, at]


def _plain_scores(s):
    picked = s["centers"].long()
    h = _plain_rows(s["q_in"].view(torch.uint8)[picked].view(E4M3), s["scales_in"].view(torch.uint8)[picked].view(E8M0), s["dim"])
    z = h @ _plain_rows(s["q_out"], s["scales_out"], s["dim"]).T
    if s["scale"] != 1.0:
        z = z * s["scale"]
    if s["bias"] is not None:
        z = z + s["bias"]
    return z.to(DTYPES[s["dtype"]])


def _plain_select(s):
    g, b, n, k = s["groups"], s["beams"], s["nodes"], s["width"]
    z = s["scores"].double()
    top = z.amax(dim=1, keepdim=True)
    lse = top + torch.log(torch.exp(z - top).sum(dim=1, keepdim=True))
    z, ids = torch.sort(z, dim=1, descending=True, stable=True)      # equal scores: the lowest node first
    z, ids = z[:, :k], ids[:, :k]
    logp = s["logp"].double()[:, None]
    total = torch.where(z > -INF, logp + (z - lse), -INF)
    if s["ended"] is not None:                                       # a walk that has ended stays as it is
        first = torch.arange(z.shape[1], device=DEV)[None, :] == 0
        ended = s["ended"][:, None]
        total = torch.where(ended, torch.where(first, logp, -INF), total)
        ids = torch.where(ended, -1, ids)
    per = total.shape[1]
    total, ids = total.view(g, b * per), ids.view(g, b * per)
    total, at = torch.sort(total, dim=1, descending=True, stable=True)
    total, at = total[:, :k], at[:, :k]
    there = total > -INF
    parents = torch.where(there, at // per, -1)
    nodes = torch.where(there, ids.gather(1, at), -1)
    short = k - total.shape[1]                                       # fewer candidates than places
    pad = torch.nn.functional.pad
    return {"parents": pad(parents, (0, short), value=-1).to(torch.int32), "nodes": pad(nodes, (0, short), value=-1).to(torch.int32),
            "logp": pad(total, (0, short), value=-INF).float()}


def _plain_reorder(s):
    first = s["beams"] * torch.arange(s["groups"], device=DEV)[:, None]
    rows = (first + s["parents"].long()).reshape(-1)
    [o.copy_(x[rows]) for x, o in zip(s["states"], s["outs"])]
    s["outs"][0][:, s["column"]] = s["nodes"].reshape(-1)
    return {"states": s["outs"]}


def run(state):
    if own:
        return _own(state)
    if state["op"] == "quantize":
        if state["ids"] is None:
            q, scales = _plain_quantize(state["table"])
            return {"q": q, "scales": scales}
        rows = state["ids"].long()
        q, scales = _plain_quantize(state["table"][rows])
        state["q"].view(torch.uint8)[rows] = q.view(torch.uint8)
        state["scales"].view(torch.uint8)[rows] = scales.view(torch.uint8)
        return {"q": state["q"], "scales": state["scales"]}
    if state["op"] == "scores":
        return {"scores": _plain_scores(state)}
    return _plain_select(state) if state["op"] == "select" else _plain_reorder(state)


def work(case):
    if case["op"] == "quantize":
        n = case["rows"] or case["nodes"]
        row = _pitch(case["dim"]) + _scale_pitch(case["dim"])
        return {"bytes": n * (case["dim"] * BYTES[case["dtype"]] + row + (4 if case["rows"] else 0)), "flops": 0}
    if case["op"] == "scores":
        m, n, d = case["centers"], case["nodes"], case["dim"]
        row = _pitch(d) + _scale_pitch(d)
        return {"bytes": (min(m, n, 100_000) + n) * row + 4 * m + (4 * n if case["bias"] else 0) + m * n * BYTES[case["dtype"]],
                "flops": 2 * m * n * d}
    if case["op"] == "select":
        rows = case["groups"] * case["beams"]
        return {"bytes": rows * (case["nodes"] * BYTES[case["dtype"]] + 5) + 12 * case["groups"] * case["width"], "flops": 0}
    row = 4 * (80 + case["states"] * case["columns"])
    return {"bytes": case["groups"] * ((min(case["beams"], case["width"]) + case["width"]) * row + 8 * case["width"]), "flops": 0}


def _exact_quantize(s):
    """Block by block, in numpy: the least power of two by which the largest value is at most 448; the values, not rounded, in its units."""
    x = s["table"].double().cpu().numpy()
    n, dim = x.shape
    rows = np.arange(n) if s["ids"] is None else s["ids"].cpu().numpy()
    q = s["q"].double().cpu().numpy()
    scales = s["scales"].double().cpu().numpy()
    q[rows], scales[rows] = 0.0, 2.0 ** -127
    for b in range((dim + BLOCK - 1) // BLOCK):
        part = x[rows, b * BLOCK:(b + 1) * BLOCK]
        with np.errstate(divide="ignore"):
            power = np.ceil(np.log2(np.abs(part).max(axis=1) / 448.0))
        unit = 2.0 ** np.maximum(power, -127)
        q[rows, b * BLOCK:b * BLOCK + part.shape[1]] = part / unit[:, None]
        scales[rows, b] = unit
    return {"q": torch.from_numpy(q), "scales": torch.from_numpy(scales)}


def _exact_scores(s):
    """A block's values times its power of two, in 64 bits, block by block."""
    out = 0.0
    for b in range((s["dim"] + BLOCK - 1) // BLOCK):
        cut = slice(b * BLOCK, min(s["dim"], (b + 1) * BLOCK))
        both = []
        for q, scales in ((s["q_in"], s["scales_in"]), (s["q_out"], s["scales_out"])):
            both.append(q[:, cut].to(torch.float64) * scales[:, b:b + 1].to(torch.float64))
        out = out + both[0].index_select(0, s["centers"].long()) @ both[1].t().contiguous()
    out = s["scale"] * out
    return {"scores": out if s["bias"] is None else out + s["bias"].double()}


def _exact_select(s):
    """Group by group, in numpy: all candidates above the last that is taken, put in order."""
    g, b, n, k = s["groups"], s["beams"], s["nodes"], s["width"]
    parents, nodes, logp = np.full((g, k), -1, np.int32), np.full((g, k), -1, np.int32), np.full((g, k), -np.inf)
    ended = None if s["ended"] is None else s["ended"].cpu().numpy()
    before = s["logp"].double().cpu().numpy()
    for i in range(g):
        found = []
        for j in range(b):
            r = i * b + j
            if before[r] == -np.inf:
                continue
            if ended is not None and ended[r]:
                found.append((-before[r], j, 0.0, -1))
                continue
            z = s["scores"][r].double()
            p = (before[r] + torch.log_softmax(z, 0)).cpu().numpy()
            z = z.cpu().numpy()
            cut = np.partition(z, n - k)[n - k] if k < n else -np.inf
            at = np.flatnonzero((z >= cut) & (z > -np.inf))
            at = at[np.argsort(-z[at], kind="stable")][:k]
            found += [(-p[a], j, -z[a], a) for a in at]
        for t, (p, j, _, a) in enumerate(sorted(found)[:k]):
            parents[i, t], nodes[i, t], logp[i, t] = j, a, -p
    return {"parents": parents, "nodes": nodes, "logp": logp}


def _exact_reorder(s):
    group = torch.arange(s["groups"], device=DEV).repeat_interleave(s["width"])
    states = [torch.index_select(x, 0, group * s["beams"] + s["parents"].flatten()) for x in s["states"]]
    states[0] = torch.cat([states[0][:, :s["column"]], s["nodes"].view(-1, 1), states[0][:, s["column"] + 1:]], dim=1)
    return {"states": states}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "quantize":
        return _exact_quantize(s)
    if case["op"] == "scores":
        return _exact_scores(s)
    return _exact_select(s) if case["op"] == "select" else _exact_reorder(s)
