"""A small GGNN learns hidden node labels from a larger one's best answers, then
answers under rules: `python examples/distill_tokens.py [steps]`.

The graph and its labels are those of hidden_tokens.py.  The teacher trains on the
labels of half of the hidden nodes; for all hidden nodes it leaves its eight
best tokens with their logits, on which the student trains beside the known labels.
At the end the student answers for a few nodes: freely, then with its first answers
counted as seen, and with half of the vocabulary masked.
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


def main(steps: int = 60, n: int = 2000, B: int = 64, E: int = 3, T: int = 3, V: int = 500, dt: str = "bf16"):
    import torch
    g = scramble_graph(5, 0, backbone_graph(5, 0, n, E, span_mean=6.0, max_span=B))[0]
    comp = compile_graphs([g], B, E, reorder=True)
    rng = np.random.default_rng(0)
    first = (np.arange(n) // 20) % V                     # shared by twenty neighbours
    lists = [[int(first[i])] + list(rng.integers(0, V, rng.integers(0, 3))) for i in range(n)]
    hidden = rng.permutation(n)[:n // 6]
    shown = [[] if h else x for h, x in zip(np.isin(np.arange(n), hidden), lists)]
    known = np.where(np.arange(len(hidden)) % 2 == 0, first[hidden], -1)

    def make(H, seed):
        params = draw_params(seed, comp.n_real, comp.n_pad, H, E, dt)
        table = np.random.default_rng(seed).standard_normal((V, H)) / np.sqrt(H)
        table = torch.from_numpy(table).to(torch.bfloat16).double().numpy()
        return NodeTokens(BandedGGNN(comp, H, T, dt, params), table, *token_lists(shown, comp.n_pad), scale=np.sqrt(H),
                          p_in=0.1, p_out=0.1, seed=7)

    teacher, student = make(64, 5), make(32, 6)
    teacher.setup_training(hidden, known, lr=0.5, momentum=0.9)
    for _ in range(steps):
        teacher.train_step()
    answers = teacher.top(hidden, 8, temperature=2.0)
    student.setup_training(hidden, known, lr=0.5, momentum=0.9, teacher=answers, temperature=2.0, soft=0.5)
    losses = []
    for i in range(steps):
        student.train_step()
        losses.append((float(student.loss.mean()), float(student.soft_loss.mean())))
        if i % 20 == 0 or i == steps - 1:
            print(f"step {i}: mean cross entropy {losses[-1][0]:.3f}, distillation {losses[-1][1]:.3f}", flush=True)
    asked = hidden[:6]
    free = student.top(asked, 3)
    seen = [free["token"][:r, 0].tolist() for r in range(len(asked))]   # what the rows before answered
    ruled = student.top(asked, 3, student.rules(len(asked), seen=seen, repetition=1.5, presence=1.0))
    half = np.zeros((1, V), bool)
    half[0, :V // 2] = True
    masked = student.top(asked, 3, student.rules(len(asked), allowed=half, allowed_of=np.zeros(len(asked), int)))
    print("targets     ", first[asked].tolist())
    for name, out in (("free", free), ("unlike before", ruled), ("first half", masked)):
        print(f"{name:13s}", out["token"].tolist())
    return losses, free, ruled, masked


if __name__ == "__main__":
    main(*(int(a) for a in sys.argv[1:2]))
