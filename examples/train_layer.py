"""Trains one GNN layer on a synthetic partition: messages and aggregation by LayerStep, the dense half by DenseLayer.

    python examples/train_layer.py [--config c0] [--out 64] [--steps 100] [--rate 0.05]

The layer learns rows that another layer, of unknown weights, makes of the same aggregated features.  Prints the mean squared error as it falls."""
from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_2306_01381_amd import binding as B  # noqa: E402
from paper_2306_01381_amd.dense import DenseLayer  # noqa: E402
from paper_2306_01381_amd.layer import LayerStep  # noqa: E402
from paper_2306_01381_amd.synth import CONFIGS, make_partition  # noqa: E402


def train(config: str = "c0", n_out: int = 64, steps: int = 100, rate: float = 0.05, device: str = "cuda:0", say=lambda *a: None):
    """The mean squared error before every step and after the last."""
    p = make_partition(CONFIGS[config])
    aggregation = LayerStep(p, device, seed=1)
    layer = DenseLayer(p.n_rows, p.cfg.dim, n_out, device, seed=1)
    gen = torch.Generator(device=device).manual_seed(2)
    unknown = torch.randn(n_out, p.cfg.dim, generator=gen, device=device)
    target, errors = None, []
    for step in range(steps + 1):
        aggregation.run(B.SERIAL)
        torch.cuda.current_stream().wait_stream(aggregation.stream_msg)
        if target is None:
            z = aggregation.out @ unknown.t()
            target = torch.nn.functional.layer_norm(z, (n_out,))
        y = layer.forward(aggregation.out)
        off = y - target
        errors.append(off.square().mean())
        if step % 10 == 0:
            say(f"step {step:4d}  mean squared error {errors[-1].item():.4f}")
        if step < steps:
            layer.backward(off.mul_(2.0 / off.numel()), wants_dx=False)
            layer.update(rate * (1 - step / steps))
            aggregation.stream_msg.wait_stream(torch.cuda.current_stream())
    return torch.stack(errors).tolist()


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--config", default="c0", choices=sorted(c for c in CONFIGS if not CONFIGS[c].backward), help="a synthetic partition of synth.py")
    ap.add_argument("--out", type=int, default=64, help="columns of the layer's result")
    ap.add_argument("--steps", type=int, default=100)
    ap.add_argument("--rate", type=float, default=0.05)
    a = ap.parse_args()
    train(a.config, a.out, a.steps, a.rate, say=lambda *words: print(*words, flush=True))
