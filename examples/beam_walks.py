"""The most probable walks of a model, by beam search over 8-bit tables, on one GPU.

A random model of the smallest workload (10,000 nodes): ``gs_quantize_rows`` makes 8-bit copies of its tables.  Then, step by step,
``gs_scores_q8`` scores every node as the successor of each walk's last one, ``gs_beam_select`` keeps the best continuations, and
``gs_beam_reorder`` lets the walks and the sums of their rows follow the choice.  A walk ends at a goal; a node is not visited twice.

    python examples/beam_walks.py [beams]
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2407_15452_amd import binding as gs, inputs  # noqa: E402


def search(t_in, t_out, w_in, starts, goals, beams, length, scale=1.0):
    """Walks [starts, beams, length] (-1 behind the goal), their log-probabilities, and the sums of their nodes' rows of w_in."""
    groups, dev = starts.numel(), starts.device
    walks = starts.repeat_interleave(beams)[:, None].repeat(1, length)     # the start in places yet to come: masked as any visited node
    sums = gs.gs_get_rows(w_in, walks[:, 0].contiguous())
    logp = torch.full((groups, beams), float("-inf"), device=dev)
    logp[:, 0] = 0.0                                                       # one walk per start at first
    is_goal = torch.zeros(t_out.num_nodes + 1, dtype=torch.bool, device=dev)
    is_goal[goals.long()] = True
    ended = torch.zeros(groups * beams, dtype=torch.bool, device=dev)
    z = torch.empty(groups * beams, t_out.num_nodes, dtype=torch.bfloat16, device=dev)
    for t in range(1, length):
        gs.gs_scores_q8(t_in, t_out, walks[:, t - 1].contiguous(), scale=scale, dtype=z.dtype, out=z)   # of ended walks NaN: not looked at
        z.scatter_(1, walks.long().clamp(min=0), float("-inf"))
        parents, nodes, logp = gs.gs_beam_select(z, logp.reshape(-1), beams, beams, ended=ended)
        gs.gs_beam_reorder([walks, sums], parents, beams, nodes=nodes, columns=[t, None])
        new = nodes.reshape(-1).long()
        ended = (new < 0) | is_goal[new]
        rows = gs.gs_get_rows(w_in, nodes.reshape(-1).clamp(min=0))
        sums += torch.where((new >= 0)[:, None], rows, 0.0)
    return walks.view(groups, beams, length), logp, sums.view(groups, beams, w_in.shape[1])


def main(beams=8, num_starts=4, length=12):
    wl = inputs.WORKLOADS[0]
    w_in, w_out = (t.cuda() for t in inputs.random_tables(wl.num_nodes, wl.dim, seed=1, scale=0.8))
    t_in, t_out = gs.gs_quantize_rows(w_in), gs.gs_quantize_rows(w_out)
    starts = torch.arange(num_starts, dtype=torch.int32, device="cuda")
    goals = torch.arange(100, 300, dtype=torch.int32, device="cuda")
    walks, logp, sums = search(t_in, t_out, w_in, starts, goals, beams, length)
    for s in range(num_starts):
        best = [x for x in walks[s, 0].tolist() if x >= 0]
        print(f"from {s}: log-probability {logp[s, 0].item():.3f}", best)
    return w_in, walks, logp, sums


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 8)
