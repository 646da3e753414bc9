"""The dense half of a layer: owns the device memory of y = layer_norm(x W^T), its gradients and its weights' updates, next to LayerStep, whose
aggregated rows it takes.

The products run on 4-bit copies of their operands (MX blocks): x and W to nearest, the gradient of the product stochastically, so that the
gradients are unbiased for the rounded operands.  The weights themselves stay in fp32 and move along their orthogonalised momentum.
Everything computational happens inside libadaqp; this module only owns memory and queues its calls on torch's current stream.
"""
from __future__ import annotations

import itertools
import math
from typing import Optional

import torch

from . import binding as B

# (a, b, c) of the update's steps: five times s -> a s + b s^3 + c s^5 takes singular values from a hundredth of the norm on to between 0.68 and 1.14.
UPDATE_STEPS = ((3.4445, -4.7750, 2.0315),) * 5

_layers = itertools.count()
_APART = 0x9E3779B97F4A7C15                         # odd, about 2^64 over the golden ratio: multiples of it by near numbers lie far apart


def rows_of_lines(n_rows: int, n_cols: int, device, dtype=torch.float32) -> torch.Tensor:
    """An uninitialised [n_rows, n_cols] matrix whose rows cover whole 128-byte lines."""
    line = 128 // dtype.itemsize
    return torch.empty(n_rows, -(-n_cols // line) * line, dtype=dtype, device=device)[:, :n_cols]


class DenseLayer:
    def __init__(self, n_rows: int, n_in: int, n_out: int, device="cuda:0", seed: Optional[int] = None, eps: float = 1e-5, weight: Optional[torch.Tensor] = None):
        """`seed`: of the weights and of the numbers that round gradients; layers that are trained together need different ones.  None: how many
        layers were made without one before this."""
        if seed is None:
            seed = next(_layers)
        self.n_rows, self.n_in, self.n_out, self.eps = n_rows, n_in, n_out, eps
        self.seed = seed * _APART % 2 ** 64         # of the rounding numbers; every step takes two more
        self.device = torch.device(device)
        if weight is None:
            gen = torch.Generator().manual_seed(seed)
            weight = torch.randn(n_out, n_in, generator=gen) / math.sqrt(n_in)
        if tuple(weight.shape) != (n_out, n_in):
            raise ValueError(f"weight is {tuple(weight.shape)}, {(n_out, n_in)} is wanted")
        dev = self.device
        self.weight = weight.to(dev, torch.float32).contiguous()
        self.gamma, self.beta = torch.ones(n_out, device=dev), torch.zeros(n_out, device=dev)
        self.z, self.y, self.dz = (rows_of_lines(n_rows, n_out, dev) for _ in range(3))
        self.dx = rows_of_lines(n_rows, n_in, dev)
        self.stats = torch.empty(n_rows, 2, device=dev)
        self.dweight, self.momentum, self.direction = (torch.zeros(n_out, n_in, device=dev) for _ in range(3))
        self.dgamma, self.dbeta = torch.empty(n_out, device=dev), torch.empty(n_out, device=dev)
        # 4-bit copies: x by rows (forward) and by columns (dW), W by rows (forward) and by columns (dx), dz both ways (dx, dW)
        self.x4, self.xt4 = B.mx4_empty(n_rows, n_in, dev), B.mx4_empty(n_in, n_rows, dev)
        self.w4, self.wt4 = B.mx4_empty(n_out, n_in, dev), B.mx4_empty(n_in, n_out, dev)
        self.dz4, self.dzt4 = B.mx4_empty(n_rows, n_out, dev), B.mx4_empty(n_out, n_rows, dev)
        need = max(B.adaqp_mx4_matmul_workspace_bytes(n_rows, n_out, n_in), B.adaqp_mx4_matmul_workspace_bytes(n_rows, n_in, n_out),
                   B.adaqp_mx4_matmul_workspace_bytes(n_out, n_in, n_rows), B.adaqp_layernorm_workspace_bytes(n_rows, n_out),
                   B.adaqp_orthogonalize_workspace_bytes(1, n_out, n_in), 1)
        self.workspace = torch.empty(need, dtype=torch.uint8, device=dev)       # of one call at a time: they follow one another on a stream
        self.steps = 0
        self.trained_on = False                     # whether xt4 is of the last forward's x
        self._quantize_weight()

    def _quantize_weight(self) -> None:
        B.adaqp_mx4_quantize(self.weight, self.n_in, B.MX4_NEAREST, 0, self.w4, self.wt4)

    def forward(self, x: torch.Tensor, training: bool = True) -> torch.Tensor:
        """y of x [n_rows, n_in].  `training`: backward may follow, so that the columns' form of x is made in the same pass."""
        self.trained_on = False
        B.adaqp_mx4_quantize(x, self.n_in, B.MX4_NEAREST, 0, self.x4, self.xt4 if training else None)
        B.adaqp_mx4_matmul(self.x4, self.w4, self.n_in, self.z, self.workspace)
        B.adaqp_layernorm_forward(self.z, self.n_out, self.gamma, self.beta, self.eps, self.y, self.stats)
        self.trained_on = training
        return self.y

    def backward(self, dy: torch.Tensor, wants_dx: bool = True) -> Optional[torch.Tensor]:
        """dx of the last forward(), and the parameters' gradients in dweight, dgamma and dbeta.  Raises if that was none for training."""
        if not self.trained_on:
            raise RuntimeError("backward() needs a forward(training=True) before it: there is no columns' form of x")
        B.adaqp_layernorm_backward(self.z, dy, self.n_out, self.stats, self.gamma, self.dz, self.dgamma, self.dbeta, self.workspace)
        self.steps += 1
        B.adaqp_mx4_quantize(self.dz, self.n_out, B.MX4_STOCHASTIC, self.seed + 2 * self.steps, self.dz4 if wants_dx else None, self.dzt4)
        B.adaqp_mx4_matmul(self.dzt4, self.xt4, self.n_rows, self.dweight, self.workspace)
        if not wants_dx:
            return None
        B.adaqp_mx4_matmul(self.dz4, self.wt4, self.n_out, self.dx, self.workspace)
        return self.dx

    def update(self, rate: float, momentum: float = 0.95, norm_rate: float = 0.0) -> None:
        """Moves the weights against their orthogonalised momentum, gamma and beta against their gradients."""
        self.momentum.mul_(momentum).add_(self.dweight)
        B.adaqp_orthogonalize(self.momentum, self.direction, UPDATE_STEPS, 1e-7, self.workspace)
        self.weight.add_(self.direction, alpha=-rate * math.sqrt(max(1.0, self.n_out / self.n_in)))
        self.gamma.add_(self.dgamma, alpha=-norm_rate)
        self.beta.add_(self.dbeta, alpha=-norm_rate)
        self._quantize_weight()
