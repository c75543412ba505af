"""The full-softmax operators around the embedding tables, as cases that can be timed.

Skip-gram's objective is a softmax over every node; negative sampling stands in for it.  Four operators work on that
objective itself: the loss of a batch of (centre, context) pairs with the gradients of both tables, the scores of centres
against every node, the choice of a node from scores by given random numbers, and the global norm of gradients with
clipping.  Each case is one call.  ``run`` computes it in elementary torch operations, or, where ``own`` is true, with the
entry points of ``paper_2407_15452_amd.binding``; both take the same inputs.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
INF = float("inf")


def _loss(pairs, nodes, dim, dtype, grad=True, bias=False, **more):
    return {"op": "loss", "pairs": pairs, "nodes": nodes, "dim": dim, "dtype": dtype, "grad": grad, "bias": bias, **more}


def _scores(pairs, nodes, dim, dtype, bias=False, **more):
    return {"op": "scores", "pairs": pairs, "nodes": nodes, "dim": dim, "dtype": dtype, "bias": bias, **more}


def _sample(rows, nodes, dtype, top_k=False, top_p=False, min_p=False, **more):
    return {"op": "sample", "rows": rows, "nodes": nodes, "dtype": dtype, "top_k": top_k, "top_p": top_p, "min_p": min_p, **more}


def _clip(tensors, elements, dtype, reached=True, **more):
    return {"op": "clip", "tensors": tensors, "elements": elements, "dtype": dtype, "reached": reached, **more}


def listed():
    return [
        # one pair of the benchmark's smallest graph, loss alone: a look at one held-out edge, latency counts
        _loss(1, 10_000, 64, "f32", grad=False, name="loss-one"),
        # the benchmark's smallest workload: 65,536 pairs of a batch, 10,000 nodes, fp32 tables
        _loss(65_536, 10_000, 64, "f32", name="loss-64k-f32"),
        # a graph of a million nodes, bfloat16 tables, the batch of a large training step
        _loss(4096, 1_000_000, 128, "bf16", name="loss-1m-bf16"),
        # ragged: only some nodes may be answers (items of a user-item graph), popularity offsets, fp16 rows of 200
        _loss(777, 50_021, 200, "f16", bias=True, name="loss-ragged-f16"),
        # one query against a million nodes, as a recommender answers it: one read of the table
        _scores(1, 1_000_000, 128, "bf16", name="scores-one"),
        # a batch of queries: as many scores as fit the memory of the next step
        _scores(256, 1_000_000, 128, "bf16", bias=True, name="scores-256"),
        # one answer from the smallest graph, every filter set
        _sample(1, 10_000, "f32", True, True, True, name="sample-one"),
        # a batch of answers over a large graph, nucleus alone: the filter that has to weigh every node
        _sample(256, 100_003, "bf16", top_p=True, name="sample-nucleus"),
        # the largest batch of scores, every filter set by row
        _sample(64, 1_000_000, "f32", True, True, True, name="sample-64"),
        # the gradients of the smallest workload's step: two blocks of rows, clipped
        _clip(2, 4_834_304, "f32", name="clip-two"),
        # both tables of a million nodes, bfloat16, limit not reached: the norm is all that is computed
        _clip(2, 256_000_000, "bf16", reached=False, name="clip-below"),
        # the parameters of a model on top of the tables: many tensors of all sizes, at all alignments
        _clip(301, 20_000_003, "f32", name="clip-many"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["loss", "loss", "scores", "sample", "sample", "clip"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    dim = 4 * rng.randint(2, 64) if dtype == "f32" else 8 * rng.randint(1, 32)
    nodes = _log(rng, 64, 1_000_000)
    if op == "loss":
        most = 4096 * 1_000_000 * 128 // (nodes * dim)
        return _loss(_log(rng, 1, max(1, min(65_536, most))), nodes, dim, dtype, grad=rng.random() < 0.75, bias=rng.random() < 0.4)
    if op == "scores":
        return _scores(_log(rng, 1, min(4096, 256_000_000 // nodes)), nodes, dim, dtype, bias=rng.random() < 0.4)
    if op == "sample":
        return _sample(_log(rng, 1, min(4096, 64_000_000 // nodes)), nodes, dtype, *(rng.random() < 0.5 for _ in range(3)))
    tensors = _log(rng, 1, 400)
    return _clip(tensors, max(tensors, _log(rng, 1, 128_000_000)), dtype, reached=rng.random() < 0.7)


def _uniform(gen, *shape):
    return torch.rand(*shape, generator=gen, device=DEV)


def _bias(gen, nodes):
    """Offsets by popularity; three nodes in ten are no answers, and one node always is."""
    bias = 0.5 * torch.randn(nodes, generator=gen, device=DEV)
    out = _uniform(gen, nodes) < 0.3
    out[nodes // 2] = False
    return bias.masked_fill(out, -INF)


def _tables(case, gen):
    """Mid-training rows: scores of about N(0, 2^2)."""
    d, t = case["dim"], DTYPES[case["dtype"]]
    sigma = math.sqrt(2.0 / math.sqrt(d))
    rows = max(1, min(case["nodes"], 100_000))
    w_in = (sigma * torch.randn(rows, d, generator=gen, device=DEV)).to(t)
    w_out = (sigma * torch.randn(case["nodes"], d, generator=gen, device=DEV)).to(t)
    centers = (_uniform(gen, case["pairs"]) * rows).to(torch.int32).clamp_(max=rows - 1)
    return w_in, w_out, centers


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s = dict(case)
    if case["op"] in ("loss", "scores"):
        s["w_in"], s["w_out"], s["centers"] = _tables(case, gen)
        s["bias"] = _bias(gen, case["nodes"]) if case["bias"] else None
        s["scale"] = 1.0
        if case["op"] == "loss":
            n, nodes = case["pairs"], case["nodes"]
            t = (_uniform(gen, n) ** 2 * nodes).to(torch.int64).clamp_(max=nodes - 1)       # popular nodes more often
            if s["bias"] is not None:
                t = torch.where(torch.isinf(s["bias"][t]), nodes // 2, t)
            if n > 1:
                t = t.masked_fill(_uniform(gen, n) < 0.02, -1)                            # walks that ended early
            s["contexts"] = t.to(torch.int32)
            s["grad_scale"] = 1.0 / n
    elif case["op"] == "sample":
        rows, nodes = case["rows"], case["nodes"]
        z = 2.0 * torch.randn(rows, nodes, generator=gen, device=DEV)
        z.masked_fill_(_uniform(gen, rows, nodes) < 0.1, -INF)
        s["scores"] = z.to(DTYPES[case["dtype"]])
        s["uniforms"] = _uniform(gen, rows)
        greedy = _uniform(gen, rows) < 0.1
        s["temperature"] = (0.5 + _uniform(gen, rows)).masked_fill(greedy, 0.0)
        k = (_uniform(gen, rows) * math.log(1000.0)).exp().to(torch.int32)
        s["top_k"] = torch.where(_uniform(gen, rows) < 0.1, 0, k) if case["top_k"] else None   # 0: this row has no such limit
        s["top_p"] = 0.7 + 0.29 * _uniform(gen, rows) if case["top_p"] else None
        s["min_p"] = 0.1 * _uniform(gen, rows) if case["min_p"] else None
    else:
        n, total, t = case["tensors"], case["elements"], DTYPES[case["dtype"]]
        cuts = torch.sort((_uniform(gen, n - 1) ** 3 * total).to(torch.int64).clamp_(max=total)).values.tolist() if n > 2 else [total // 2] * (n - 1)
        ends = list(zip([0] + cuts, cuts + [total]))
        s["flat"] = (0.02 * torch.randn(total, generator=gen, device=DEV)).to(t)
        s["out"] = torch.empty_like(s["flat"]) if case["reached"] else s["flat"]
        s["grads"] = [s["flat"][a:b] for a, b in ends]
        s["outs"] = [s["out"][a:b] for a, b in ends]
        s["max_norm"] = 0.02 * math.sqrt(total) * (0.25 if case["reached"] else 100.0)
        if own:                                    # the list of its gradients that a program builds once
            from paper_2407_15452_amd import binding as gs
            s["list"] = gs.GradList(s["grads"], s["outs"] if case["reached"] else None)
    return s


def _own(s):
    from paper_2407_15452_amd import binding as gs
    if s["op"] == "loss":
        loss, g_in, g_out = gs.gs_softmax_loss(s["w_in"], s["w_out"], s["centers"], s["contexts"], bias=s["bias"], scale=s["scale"],
                                               grad_scale=s["grad_scale"], want_grad=s["grad"])
        return {"loss": loss, "g_in": g_in, "g_out": g_out}
    if s["op"] == "scores":
        return {"scores": gs.gs_scores(s["w_in"], s["w_out"], s["centers"], bias=s["bias"], scale=s["scale"])}
    if s["op"] == "sample":
        ids, probs = gs.gs_sample_scores(s["scores"], s["uniforms"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                                         min_p=s["min_p"])
        return {"ids": ids, "probs": probs}
    norm = gs.gs_clip_grads(s["list"], s["max_norm"])
    return {"norm": norm, "grads": s["out"]}


def _plain_scores(s, h, c):
    z = h @ c.T
    if s["scale"] != 1.0:
        z = z * s["scale"]
    return z if s["bias"] is None else z + s["bias"]


def _plain_rows(s):
    h, c = s["w_in"][s["centers"].long()].float(), s["w_out"].float()
    if s["bias"] is not None:
        c = c.masked_fill(torch.isinf(s["bias"])[:, None], 0.0)
    return h, c


def _plain_loss(s):
    h, c = _plain_rows(s)
    z = _plain_scores(s, h, c)
    t = s["contexts"].long()
    used = t >= 0
    at = t.clamp(min=0)[:, None]
    m = z.amax(dim=1, keepdim=True)
    hit = z.gather(1, at)
    e = torch.exp(z - m)
    del z
    total = e.sum(dim=1, keepdim=True)
    loss = torch.where(used, (m + torch.log(total) - hit)[:, 0], 0.0)
    g_in = g_out = None
    if s["grad"]:
        p = e / total
        del e
        p.scatter_add_(1, at, torch.full_like(hit, -1.0))
        p = p * torch.where(used, s["grad_scale"] * s["scale"], 0.0)[:, None]
        g_in = (p @ c).to(s["w_in"].dtype)
        g_out = (p.T @ h).to(s["w_out"].dtype)
    return {"loss": loss, "g_in": g_in, "g_out": g_out}


def _plain_sample(s):
    z = s["scores"].float()
    rows, n = z.shape
    order = torch.sort(z, dim=1, descending=True, stable=True)
    z, ids = order.values.double(), order.indices
    del order
    place = torch.arange(n, device=DEV)[None, :]
    temperature = s["temperature"].double()[:, None]
    top = z[:, :1]
    e = torch.where(z == top, 1.0, torch.exp((z - top) / temperature)).masked_fill(torch.isinf(z) & (z < 0), 0.0)
    e = torch.where(temperature == 0.0, (place == 0).double(), e)
    keep = z > -INF
    if s["top_k"] is not None:
        k = s["top_k"].long()[:, None]
        keep = keep & ((place < k) | (k <= 0))
    if s["top_p"] is not None:
        kept = e.masked_fill(~keep, 0.0)
        before = kept.cumsum(dim=1) - kept
        keep = keep & ((before < s["top_p"].double()[:, None] * kept.sum(dim=1, keepdim=True)) | (place == 0))
        del kept, before
    if s["min_p"] is not None:
        keep = keep & (e >= s["min_p"].double()[:, None])
    e = torch.zeros_like(e).scatter_(1, ids, e.masked_fill(~keep, 0.0))
    del z, ids, keep
    total = e.sum(dim=1, keepdim=True)
    over = (e.cumsum(dim=1) > s["uniforms"].double()[:, None] * total) & (e > 0)
    at = torch.where(over, place, n).amin(dim=1)
    last = torch.where(e > 0, place, -1).amax(dim=1)
    at = torch.where(at < n, at, last)
    prob = torch.where(at >= 0, e.gather(1, at.clamp(min=0)[:, None])[:, 0] / total[:, 0], 0.0)
    return {"ids": at.to(torch.int32), "probs": prob.float()}


def _plain_clip(s):
    norm = torch.stack([g.double().square().sum() for g in s["grads"]]).sum().sqrt()
    factor = torch.clamp(s["max_norm"] / norm, max=1.0).float()
    [o.copy_(g.float() * factor) for g, o in zip(s["grads"], s["outs"])]
    return {"norm": norm.reshape(1), "grads": s["out"]}


def run(state):
    if own:
        return _own(state)
    if state["op"] == "loss":
        return _plain_loss(state)
    if state["op"] == "scores":
        return {"scores": _plain_scores(state, *_plain_rows(state))}
    return _plain_sample(state) if state["op"] == "sample" else _plain_clip(state)


def work(case):
    if case["op"] in ("loss", "scores"):
        b, n, d, size = case["pairs"], case["nodes"], case["dim"], BYTES[case["dtype"]]
        rows = min(b, n, 100_000) * d * size + n * d * size + 4 * b + (4 * n if case["bias"] else 0)
        if case["op"] == "scores":
            return {"bytes": rows + 4 * b * n, "flops": 2 * b * n * d}
        if not case["grad"]:
            return {"bytes": rows + 8 * b, "flops": 2 * b * n * d}
        return {"bytes": rows + 8 * b + (b + n) * d * size, "flops": 6 * b * n * d}
    if case["op"] == "sample":
        return {"bytes": case["rows"] * (case["nodes"] * BYTES[case["dtype"]] + 28), "flops": 0}
    size = case["elements"] * BYTES[case["dtype"]]
    return {"bytes": size * (2 if case["reached"] else 1), "flops": 2 * case["elements"]}


def _exact_tables(s):
    h, c = s["w_in"].double().index_select(0, s["centers"].long()), s["w_out"].double()
    b = torch.zeros(c.shape[0], dtype=torch.float64, device=DEV) if s["bias"] is None else s["bias"].double()
    c = torch.where((b == -INF)[:, None], 0.0, c)
    return h, c, b


def _exact_loss(s):
    """Rows in blocks; log sum exp and the softmax by torch's own in 64 bits."""
    h, c, b = _exact_tables(s)
    n = h.shape[0]
    block = max(1, 100_000_000 // c.shape[0])
    loss = torch.zeros(n, dtype=torch.float64, device=DEV)
    g_in, g_out = torch.zeros_like(h), torch.zeros_like(c)
    for lo in range(0, n, block):
        x = h[lo:lo + block]
        t = s["contexts"][lo:lo + block].long()
        z = s["scale"] * (x @ c.t().contiguous()) + b
        i = torch.nonzero(t >= 0)[:, 0]
        loss[lo + i] = torch.logsumexp(z[i], 1) - z[i, t[i]]
        if s["grad"]:
            g = torch.softmax(z, 1)
            g[i, t[i]] -= 1
            g[t < 0] = 0
            g *= s["scale"] * s["grad_scale"]
            g_in[lo:lo + block] = g @ c
            g_out += g.t().contiguous() @ x
    return {"loss": loss, "g_in": g_in if s["grad"] else None, "g_out": g_out if s["grad"] else None}


def _exact_sample(s):
    """Row by row in numpy: sorted, cut, and searched in the order of the ids."""
    rows = s["scores"].shape[0]
    ids, probs = np.full(rows, -1, np.int32), np.zeros(rows)
    host = {k: s[k].cpu().numpy().astype(np.float64) for k in ("uniforms", "temperature", "top_k", "top_p", "min_p") if s[k] is not None}
    for r in range(rows):
        z = s["scores"][r].double().cpu().numpy()
        may = np.flatnonzero(z > -np.inf)
        if not may.size:
            continue
        rank = may[np.argsort(-z[may], kind="stable")]
        if host["temperature"][r] == 0:
            ids[r], probs[r] = rank[0], 1.0
            continue
        w = np.exp((z[rank] - z[rank[0]]) / host["temperature"][r])
        if "top_k" in host and host["top_k"][r] > 0:
            rank, w = rank[:int(host["top_k"][r])], w[:int(host["top_k"][r])]
        if "top_p" in host:
            before = np.concatenate([[0.0], np.cumsum(w)[:-1]])
            m = max(1, int((before < host["top_p"][r] * w.sum()).sum()))
            rank, w = rank[:m], w[:m]
        if "min_p" in host:
            m = int((w >= host["min_p"][r]).sum())
            rank, w = rank[:m], w[:m]
        back = np.argsort(rank)
        rank, w = rank[back], w[back]
        sums = np.cumsum(w)
        j = min(int(np.searchsorted(sums, host["uniforms"][r] * w.sum(), side="right")), w.size - 1)
        ids[r], probs[r] = rank[j], w[j] / w.sum()
    return {"ids": ids, "probs": probs}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "loss":
        return _exact_loss(s)
    if case["op"] == "scores":
        h, c, b = _exact_tables(s)
        return {"scores": s["scale"] * (h @ c.t().contiguous()) + b}
    if case["op"] == "sample":
        return _exact_sample(s)
    x = s["flat"].double()
    norm = torch.linalg.vector_norm(x)
    return {"norm": norm.reshape(1), "grads": x * min(1.0, s["max_norm"] / float(norm))}
