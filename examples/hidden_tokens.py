"""Trains a small GGNN to predict hidden node labels from their neighbourhood,
then answers for a few nodes: `python examples/hidden_tokens.py [steps]`.

The graph is one of the package's synthetic program graphs.  A node's label is
made of one to three subtokens of a 500-token vocabulary: the first is shared by
twenty nodes that follow one another in the reordered graph, the others are
drawn, so that a hidden node's neighbours tell what it is called.
"""
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import numpy as np  # noqa: E402

from ggnn_synth import backbone_graph, draw_params, scramble_graph  # noqa: E402
from paper_1906_11786_amd.driver import BandedGGNN, compile_graphs  # noqa: E402
from paper_1906_11786_amd.tokens import NodeTokens, token_lists  # noqa: E402


def main(steps: int = 60, n: int = 2000, B: int = 64, E: int = 3, H: int = 64, T: int = 3, V: int = 500,
         dt: str = "bf16"):
    import torch
    g = scramble_graph(5, 0, backbone_graph(5, 0, n, E, span_mean=6.0, max_span=B))[0]
    comp = compile_graphs([g], B, E, reorder=True)
    params = draw_params(5, comp.n_real, comp.n_pad, H, E, dt)
    rng = np.random.default_rng(0)
    first = (np.arange(n) // 20) % V                     # shared by twenty neighbours
    lists = [[int(first[i])] + list(rng.integers(0, V, rng.integers(0, 3))) for i in range(n)]
    hidden = rng.permutation(n)[:n // 6]
    shown = [[] if h else x for h, x in zip(np.isin(np.arange(n), hidden), lists)]
    model = BandedGGNN(comp, H, T, dt, params)
    table = rng.standard_normal((V, H)) / np.sqrt(H)
    if dt == "bf16":
        table = torch.from_numpy(table).to(torch.bfloat16).double().numpy()
    tok = NodeTokens(model, table, *token_lists(shown, comp.n_pad), scale=np.sqrt(H), p_in=0.1, p_out=0.1, seed=7)
    tok.setup_training(hidden, first[hidden], lr=0.5, momentum=0.9)
    losses = []
    for i in range(steps):
        tok.train_step()
        losses.append(float(tok.loss.mean()))
        if i % 20 == 0 or i == steps - 1:
            print(f"step {i}: mean loss {losses[-1]:.3f}", flush=True)
    out = tok.evaluate(hidden[:8], first[hidden[:8]])
    print("nodes  ", list(map(int, hidden[:8])))
    print("targets", list(map(int, first[hidden[:8]])))
    print("answers", out["best"].tolist())
    return losses


if __name__ == "__main__":
    main(*(int(a) for a in sys.argv[1:2]))
