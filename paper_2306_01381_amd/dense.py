"""The dense half of a layer: owns the device memory of y = dropout(layer_norm(x W^T)), its gradients and its weights' updates, next to LayerStep, whose
aggregated rows it takes; the rows that a network learns for its nodes (Embedding) and what it is trained on (ClassLoss).

The products run on 4-bit copies of their operands (MX blocks): x and W to nearest, the gradient of the product stochastically, so that the
gradients are unbiased for the rounded operands; or on 8-bit copies (bits=8), all to nearest, W by tiles, so that both directions multiply with the same values.  Products come
out in fp32: those of 8 bits are exact in it, at the rate of bf16's instructions and not the twice as fast ones that bf16 outputs take.
The weights themselves stay in fp32 and move along their orthogonalised momentum.
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
    def __init__(self, n_rows: int, n_in: int, n_out: int, device="cuda:0", seed: Optional[int] = None, eps: float = 1e-5, weight: Optional[torch.Tensor] = None,
                 bits: int = 4, drop: float = 0.0):
        """`seed`: of the weights and of the numbers that round gradients and drop elements; layers that are trained together need different ones.  None: how many
        layers were made without one before this.  `bits`: of the products' operands, 4 or 8.  `drop`: the share of y's elements that training drops."""
        if bits not in (4, 8):
            raise ValueError(f"products have operands of 4 or 8 bits, not of {bits}")
        if not 0.0 <= drop < 1.0:
            raise ValueError(f"a share of {drop} cannot be dropped")
        self.bits, self.drop = bits, drop
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
        # copies of 4 (or 8) bits: x by rows (forward) and by columns (dW), W by rows (forward) and by columns (dx), dz both ways (dx, dW)
        empty, product_bytes = (B.mx4_empty, B.adaqp_mx4_matmul_workspace_bytes) if bits == 4 else (B.f8_empty, B.adaqp_f8_matmul_workspace_bytes)
        self.x4, self.xt4 = empty(n_rows, n_in, dev), empty(n_in, n_rows, dev)
        self.w4, self.wt4 = empty(n_out, n_in, dev), empty(n_in, n_out, dev)
        self.dz4, self.dzt4 = empty(n_rows, n_out, dev), empty(n_out, n_rows, dev)
        need = max(product_bytes(n_rows, n_out, n_in), product_bytes(n_rows, n_in, n_out), product_bytes(n_out, n_in, n_rows),
                   B.adaqp_layernorm_workspace_bytes(n_rows, n_out), B.adaqp_orthogonalize_workspace_bytes(1, n_out, n_in), 1)
        self.workspace = torch.empty(need, dtype=torch.uint8, device=dev)       # of one call at a time: they follow one another on a stream
        self.steps = 0
        self.drops = 0                              # forwards that dropped; the seed of their choices is self.seed + self.drops, by another generator tag than the rounding's
        self.dropped = 0.0                          # the share that the last forward for training dropped
        self.trained_on = False                     # whether xt4 is of the last forward's x
        self._quantize_weight()

    def _quantize_weight(self) -> None:
        if self.bits == 4:
            B.adaqp_mx4_quantize(self.weight, self.n_in, B.MX4_NEAREST, 0, self.w4, self.wt4)
        else:
            B.adaqp_f8_quantize(self.weight, self.n_in, B.F8_TILES, self.w4, self.wt4)

    def _product(self, a, b, k: int, out: torch.Tensor) -> None:
        (B.adaqp_mx4_matmul if self.bits == 4 else B.adaqp_f8_matmul)(a, b, k, out, self.workspace)

    def forward(self, x: torch.Tensor, training: bool = True) -> torch.Tensor:
        """y of x [n_rows, n_in].  `training`: backward may follow, so that the columns' form of x is made in the same pass."""
        self.trained_on = False
        if self.bits == 4:
            B.adaqp_mx4_quantize(x, self.n_in, B.MX4_NEAREST, 0, self.x4, self.xt4 if training else None)
        else:
            B.adaqp_f8_quantize(x, self.n_in, B.F8_ROWS, self.x4, self.xt4 if training else None)
        self._product(self.x4, self.w4, self.n_in, self.z)
        B.adaqp_layernorm_forward(self.z, self.n_out, self.gamma, self.beta, self.eps, self.y, self.stats)
        if training:
            self.dropped = self.drop
        if training and self.dropped > 0.0:
            self.drops += 1
            B.adaqp_dropout(self.y, self.n_out, self.dropped, self.seed + self.drops, self.y)
        self.trained_on = training
        return self.y

    def backward(self, dy: torch.Tensor, wants_dx: bool = True) -> Optional[torch.Tensor]:
        """dx of the last forward(), and the parameters' gradients in dweight, dgamma and dbeta.  Raises if that was none for training."""
        if not self.trained_on:
            raise RuntimeError("backward() needs a forward(training=True) before it: there is no columns' form of x")
        if self.dropped > 0.0:
            B.adaqp_dropout(dy, self.n_out, self.dropped, self.seed + self.drops, self.dz)
            dy = self.dz
        B.adaqp_layernorm_backward(self.z, dy, self.n_out, self.stats, self.gamma, self.dz, self.dgamma, self.dbeta, self.workspace)
        self.steps += 1
        if self.bits == 4:
            B.adaqp_mx4_quantize(self.dz, self.n_out, B.MX4_STOCHASTIC, self.seed + 2 * self.steps, self.dz4 if wants_dx else None, self.dzt4)
        else:
            B.adaqp_f8_quantize(self.dz, self.n_out, B.F8_ROWS, self.dz4 if wants_dx else None, self.dzt4)
        self._product(self.dzt4, self.xt4, self.n_rows, self.dweight)
        if not wants_dx:
            return None
        self._product(self.dz4, self.wt4, self.n_out, self.dx)
        return self.dx

    def update(self, rate: float, momentum: float = 0.95, norm_rate: float = 0.0) -> None:
        """Moves the weights against their orthogonalised momentum, gamma and beta against their gradients."""
        self.momentum.mul_(momentum).add_(self.dweight)
        B.adaqp_orthogonalize(self.momentum, self.direction, UPDATE_STEPS, 1e-7, self.workspace)
        self.weight.add_(self.direction, alpha=-rate * math.sqrt(max(1.0, self.n_out / self.n_in)))
        self.gamma.add_(self.dgamma, alpha=-norm_rate)
        self.beta.add_(self.dbeta, alpha=-norm_rate)
        self._quantize_weight()


class Embedding:
    """Rows of a table that is learned, one for each id that a batch names."""

    def __init__(self, n_entries: int, dim: int, n_ids: int, device="cuda:0", seed: int = 0, scale: float = 1.0, table: Optional[torch.Tensor] = None):
        """`n_ids`: of a batch.  `scale`: what the table's rows are multiplied by."""
        dev = torch.device(device)
        if table is None:
            table = torch.randn(n_entries, dim, generator=torch.Generator().manual_seed(seed))
        if tuple(table.shape) != (n_entries, dim):
            raise ValueError(f"table is {tuple(table.shape)}, {(n_entries, dim)} is wanted")
        self.n_entries, self.dim, self.n_ids, self.scale = n_entries, dim, n_ids, scale
        self.table, self.out = rows_of_lines(n_entries, dim, dev), rows_of_lines(n_ids, dim, dev)
        self.table.copy_(table)
        self.dtable: Optional[torch.Tensor] = None
        self.sorted_ids, self.order = (torch.empty(n_ids, dtype=torch.int32, device=dev) for _ in range(2))
        need = max(B.adaqp_embedding_sort_workspace_bytes(n_ids, n_entries), B.adaqp_embedding_backward_workspace_bytes(n_ids, dim), 1)
        self.workspace = torch.empty(need, dtype=torch.uint8, device=dev)
        self.trained_on = False                     # whether sorted_ids and order are of the last forward's ids

    def forward(self, ids: torch.Tensor, training: bool = True) -> torch.Tensor:
        """The rows of ids [n_ids] (int32; zeros for those outside the table).  `training`: their gradient may follow, so that they are sorted."""
        self.trained_on = False
        B.adaqp_embedding_forward(self.table, self.dim, ids, self.scale, self.out)
        if training:
            B.adaqp_embedding_sort(ids, self.n_entries, self.sorted_ids, self.order, self.workspace)
        self.trained_on = training
        return self.out

    def _gradient(self, dy: torch.Tensor, scale: float, accumulate: bool, to: torch.Tensor) -> None:
        if not self.trained_on:
            raise RuntimeError("a gradient needs a forward(training=True) before it: the ids are not sorted")
        B.adaqp_embedding_backward(dy, self.dim, self.sorted_ids, self.order, scale, accumulate, to, self.workspace)

    def backward(self, dy: torch.Tensor) -> torch.Tensor:
        """The whole table's gradient, of the last forward()."""
        if self.dtable is None:
            self.dtable = rows_of_lines(self.n_entries, self.dim, self.table.device)
        self._gradient(dy, self.scale, False, self.dtable)
        return self.dtable

    def descend(self, dy: torch.Tensor, rate: float) -> None:
        """Moves the rows that the last forward() named, and only them, against their gradient."""
        self._gradient(dy, -rate * self.scale, True, self.table)


class ClassLoss:
    """The mean of -log p of the given classes, over the rows that have one, and its gradient."""

    def __init__(self, n_rows: int, n_classes: int, device="cuda:0"):
        dev = torch.device(device)
        self.n_rows, self.n_classes = n_rows, n_classes
        self.logp, self.entropy, self.stats = torch.empty(n_rows, device=dev), torch.empty(n_rows, device=dev), torch.empty(n_rows, 2, device=dev)
        self.dlogits = rows_of_lines(n_rows, n_classes, dev)
        self.workspace = torch.empty(max(B.adaqp_logprob_workspace_bytes(n_rows, n_classes, 0), 1), dtype=torch.uint8, device=dev)

    def forward(self, logits: torch.Tensor, targets: torch.Tensor) -> torch.Tensor:
        """log p of the targets (int32; 0 for rows whose target is no class), and their rows' entropy in `entropy`."""
        B.adaqp_logprob_forward(logits, self.n_classes, targets, self.logp, self.entropy, self.stats, None, None, self.workspace)
        return self.logp

    def backward(self, logits: torch.Tensor, targets: torch.Tensor, n_given: int) -> torch.Tensor:
        """The logits' gradient of -sum(logp) / n_given, after forward() of the same.  n_given: rows whose target is a class; with 0, the sum of no row, the gradient is zeros."""
        if n_given < 0:
            raise ValueError(f"{n_given} rows cannot have a class")
        B.adaqp_logprob_backward(logits, self.n_classes, targets, self.stats, None, None, None, -1.0 / n_given if n_given else 0.0, self.dlogits)
        return self.dlogits

    def likeliest(self, logits: torch.Tensor, n: int):
        """(log p, classes) [n_rows, n] of each row's n likeliest classes."""
        top_logp = torch.empty(self.n_rows, n, device=logits.device)
        top_class = torch.empty(self.n_rows, n, dtype=torch.int32, device=logits.device)
        work = torch.empty(max(B.adaqp_logprob_workspace_bytes(self.n_rows, self.n_classes, n), 1), dtype=torch.uint8, device=logits.device)
        B.adaqp_logprob_forward(logits, self.n_classes, None, None, None, None, top_logp, top_class, work)
        return top_logp, top_class
