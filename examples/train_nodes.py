"""Trains a node classifier on a synthetic partition: messages and aggregation by LayerStep, two layers by DenseLayer with products in 8 bits and dropout, learned rows for the nodes
by Embedding, log probabilities by ClassLoss.

    python examples/train_nodes.py [--config c0] [--hidden 64] [--classes 7] [--steps 60] [--rate 0.02]

The classes are those that another layer, of unknown weights, makes likeliest; three in ten nodes have theirs given.  Prints the mean of -log p, over the nodes with a given class and over the others."""
from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_2306_01381_amd import binding as B  # noqa: E402
from paper_2306_01381_amd.dense import ClassLoss, DenseLayer, Embedding  # noqa: E402
from paper_2306_01381_amd.layer import LayerStep  # noqa: E402
from paper_2306_01381_amd.synth import CONFIGS, make_partition  # noqa: E402


class NodeClassifier:
    """logits = layer_2(layer_1(x) + rows of the nodes)."""

    def __init__(self, n_rows: int, n_in: int, n_hidden: int, n_classes: int, device="cuda:0", drop: float = 0.3):
        self.first = DenseLayer(n_rows, n_in, n_hidden, device, seed=1, bits=8, drop=drop)
        self.nodes = Embedding(n_rows, n_hidden, n_rows, device, seed=2, scale=0.1)
        self.second = DenseLayer(n_rows, n_hidden, n_classes, device, seed=3, bits=8)
        self.loss = ClassLoss(n_rows, n_classes, device)
        self.hidden = torch.empty_like(self.first.y)

    def forward(self, x: torch.Tensor, ids: torch.Tensor, training: bool = True) -> torch.Tensor:
        torch.add(self.first.forward(x, training), self.nodes.forward(ids, training), out=self.hidden)
        return self.second.forward(self.hidden, training)

    def backward(self, logits: torch.Tensor, targets: torch.Tensor, n_given: int) -> torch.Tensor:
        """The gradient of what the two layers have between them; the layers keep their parameters' gradients."""
        between = self.second.backward(self.loss.backward(logits, targets, n_given))
        self.first.backward(between, wants_dx=False)
        return between

    def update(self, between: torch.Tensor, rate: float) -> None:
        self.first.update(rate, norm_rate=rate)
        self.second.update(rate, norm_rate=rate)
        self.nodes.descend(between, 10 * rate)


def train(config: str = "c0", n_hidden: int = 64, n_classes: int = 7, steps: int = 60, rate: float = 0.02, device: str = "cuda:0", say=lambda *a: None):
    """The mean of -log p of the given classes before every step and after the last, without dropout at the end."""
    p = make_partition(CONFIGS[config])
    aggregation = LayerStep(p, device, seed=1)
    model = NodeClassifier(p.n_rows, p.cfg.dim, n_hidden, n_classes, device)
    aggregation.run(B.SERIAL)
    torch.cuda.current_stream().wait_stream(aggregation.stream_msg)
    gen = torch.Generator(device=device).manual_seed(2)
    unknown = torch.randn(n_classes, p.cfg.dim, generator=gen, device=device)
    classes = (aggregation.out @ unknown.t()).argmax(1).int()
    given = torch.rand(p.n_rows, generator=gen, device=device) < 0.3
    targets = torch.where(given, classes, -1).int()
    hidden_from_training = torch.where(given, -1, classes).int()
    n_given = int(given.sum())
    ids = torch.arange(p.n_rows, dtype=torch.int32, device=device)
    losses = []
    for step in range(steps + 1):
        logits = model.forward(aggregation.out, ids, training=step < steps)
        losses.append(-model.loss.forward(logits, targets).sum() / n_given)
        if step < steps:
            between = model.backward(logits, targets, n_given)
            model.update(between, rate * (1 - step / steps))
        if step % 10 == 0:
            say(f"step {step:4d}  mean -log p {losses[-1].item():.4f}")
    others = -model.loss.forward(logits, hidden_from_training).sum() / max(p.n_rows - n_given, 1)
    say(f"of the nodes whose class was not given: {others.item():.4f}")
    return torch.stack(losses).tolist()


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--config", default="c0", choices=sorted(c for c in CONFIGS if not CONFIGS[c].backward), help="a synthetic partition of synth.py")
    ap.add_argument("--hidden", type=int, default=64)
    ap.add_argument("--classes", type=int, default=7)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--rate", type=float, default=0.02)
    a = ap.parse_args()
    train(a.config, a.hidden, a.classes, a.steps, a.rate, say=lambda *words: print(*words, flush=True))
