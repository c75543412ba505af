"""Skip-gram by its full softmax: training steps and answers, on one GPU.

A walk corpus of the smallest workload (10,000 nodes) is trained without negative samples: ``gs_softmax_loss`` gives the loss
of every pair over all nodes with both tables' gradients, ``gs_clip_grads`` bounds their norm, ``gs_table_mult_add`` takes the
step.  Then nodes are asked for a neighbour: ``gs_scores`` against every node, ``gs_sample_scores`` draws one by temperature,
top-k and top-p.

    python examples/full_softmax.py [steps]
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2407_15452_amd import binding as gs, inputs  # noqa: E402


def corpus(wl, device="cuda:0"):
    """Shuffled (centre, context) pairs of the workload's walks."""
    src, dst, _ = inputs.edge_list(wl, "cpu")
    g = gs.gs_csr_build(src.to(device), dst.to(device), None, wl.num_nodes, gs.GS_SYMMETRIZE | gs.GS_DROP_SELF_LOOPS | gs.GS_DEDUPE)
    starts = inputs.walk_starts(wl.num_nodes, 0, wl.num_nodes).to(device)
    walks = gs.gs_random_walk(g, None, starts, wl.walk_len, wl.walk_seed)
    centers, contexts, n = gs.gs_make_pairs(walks, wl.window)
    order = torch.randperm(n, generator=torch.Generator().manual_seed(1)).to(device)
    return centers[:n][order], contexts[:n][order]


def train(w_in, w_out, centers, contexts, batch, steps, lr, max_norm):
    """Steps of gradient descent; returns the mean losses, one per step, and the norms before clipping."""
    losses, norms = [], []
    g_w = torch.empty_like(w_in)
    ws = torch.empty(gs.gs_softmax_loss_workspace_bytes(batch, *w_out.shape), dtype=torch.uint8, device=w_in.device)
    g_in, g_out = torch.empty(batch, w_in.shape[1], device=w_in.device), torch.empty_like(w_out)
    grads = gs.GradList([g_w, g_out])              # both stay where they are
    for k in range(steps):
        lo = k * batch % (centers.numel() - batch + 1)
        c, t = centers[lo:lo + batch].contiguous(), contexts[lo:lo + batch].contiguous()
        loss, _, _ = gs.gs_softmax_loss(w_in, w_out, c, t, grad_scale=1.0 / batch, g_in=g_in, g_out=g_out, ws=ws)
        g_w.zero_().index_add_(0, c.long(), g_in)  # a row per pair: pairs of one centre add up (in an order that may differ from run to run)
        norms.append(gs.gs_clip_grads(grads, max_norm))
        gs.gs_table_mult_add(w_in, g_w, -lr)
        gs.gs_table_mult_add(w_out, g_out, -lr)
        losses.append(loss.mean())
    return torch.stack(losses).tolist(), torch.cat(norms).tolist()


def answer(w_in, w_out, nodes, uniforms, temperature=0.8, top_k=50, top_p=0.95):
    """A neighbour for each of `nodes`, by the given random numbers; a node is no answer to itself."""
    z = gs.gs_scores(w_in, w_out, nodes)
    z.scatter_(1, nodes.long()[:, None], float("-inf"))
    each = lambda v, t=torch.float32: torch.full((nodes.numel(),), v, dtype=t, device=nodes.device)  # noqa: E731
    return gs.gs_sample_scores(z, uniforms, temperature=each(temperature), top_k=each(top_k, torch.int32), top_p=each(top_p))


def main(steps=200):
    wl = inputs.WORKLOADS[0]
    centers, contexts = corpus(wl)
    w_in, w_out = (t.cuda() for t in inputs.random_tables(wl.num_nodes, wl.dim, seed=1, scale=0.2))
    losses, norms = train(w_in, w_out, centers, contexts, batch=8192, steps=steps, lr=200.0, max_norm=0.05)
    for k in range(0, steps, max(1, steps // 10)):
        print(f"step {k}: loss/pair {losses[k]:.4f}, norm {norms[k]:.4f}")
    nodes = torch.arange(8, dtype=torch.int32, device="cuda")
    ids, probs = answer(w_in, w_out, nodes, torch.rand(8, generator=torch.Generator().manual_seed(2)).cuda())
    print("answers", ids.tolist(), "probabilities", [round(p, 4) for p in probs.tolist()])
    return losses, norms, ids, probs


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 200)
