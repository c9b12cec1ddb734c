"""`torch.autograd` front end of the C ABI: a linear layer whose backward pass is
Algorithm 1 (low-rank backpropagation on the selected Walsh-Hadamard bases).

Only the backward pass is the library's: the forward product `y = x W^T + b` is a
plain matrix product and is left to torch (in one call, the bias added in the product's
epilogue, where x, weight and bias are of one type and autocast is off; else as a product
and a sum).  The layer takes the token grid
explicit, x of shape (B, H, W, Cin), or, with `grid=(H, W)`, a token sequence
(B, n + H*W, Cin) whose first n tokens (class tokens) are not part of the grid:
those take exact backpropagation (Eq. 2), and the grid tokens are handed to the
library as a strided view of the sequence, without a copy.  The bias (absent
from the paper's Eq. 1) is optional.
"""
from __future__ import annotations

from typing import Sequence, Tuple

import torch

from . import binding as _b


class LbpLinearFunction:
    """y = x W^T (+ b);  backward: Algorithm 1 on the selected bases.

    With `save_projected` the forward pass keeps x_hat = p(x) (Eq. 3) instead of
    x: r / k^2 of the activation's elements stay alive until the backward pass,
    which then starts at the second step of Algorithm 1.  Called as a
    `torch.autograd.Function` is; forward and backward are native
    (csrc/torch_binding.cpp)."""

    @staticmethod
    def apply(x: torch.Tensor, weight: torch.Tensor, bias, k: int, bases: Sequence[Tuple[int, int]],
              save_projected: bool, grid=None) -> torch.Tensor:
        H, W = (0, 0) if grid is None else (int(grid[0]), int(grid[1]))
        return _b._native().linear(x, weight, bias, int(k), [tuple(p) for p in bases], bool(save_projected), H, W)


class LbpLinear(torch.nn.Module):
    """Linear layer over a (B, H, W, C) token grid with LBP-WHT backward.

    `bases` is an ordered list of 0-based (i, j) sequency pairs, e.g. from
    `lbp_select_bases(k, SEL_L1, m)` (Eq. 8) or `lbp_select_lhe` (Sec. 3.2).

    `activation` (one of `ACTIVATIONS`), `dropout` (the probability, drawn from torch's
    generator of the device while the module is in training mode) and the `residual` given
    to a call are applied in the product's epilogue.  Such a call wants CUDA tensors of one
    dtype, fp32 or bf16.  Under autocast x, weight and bias are cast to its type, as by torch's
    own linear layer; a residual of another type keeps it and is added to the result by
    torch's rules (fp32 onto bf16: fp32).  A backward pass
    can be captured into a graph like that of torch's own layers, and under the same
    condition: no graph of earlier, uncaptured passes over the same parameters is alive.
    There is no forward-mode derivative: an operand with a tangent is refused.
    """

    activation, dropout = None, 0.0     # (also of modules stored before there were these)

    def __init__(self, in_features: int, out_features: int, k: int,
                 bases: Sequence[Tuple[int, int]], device=None, dtype=None, bias: bool = False,
                 save_projected: bool = False, grid=None, activation=None, dropout: float = 0.0):
        super().__init__()
        if activation is not None and activation not in _b.ACTIVATIONS:
            raise ValueError(f"activation is one of {_b.ACTIVATIONS}, got {activation!r}")
        if not 0.0 <= float(dropout) <= 1.0:
            raise ValueError(f"dropout is a probability, got {dropout}")
        w = torch.empty((out_features, in_features), device=device, dtype=dtype)
        torch.nn.init.normal_(w, std=in_features ** -0.5)
        self.weight = torch.nn.Parameter(w)
        self.bias = (torch.nn.Parameter(torch.zeros(out_features, device=device, dtype=dtype))
                     if bias else None)
        self.k, self.bases = int(k), [tuple(p) for p in bases]
        self.save_projected = bool(save_projected)
        self.grid = None if grid is None else (int(grid[0]), int(grid[1]))
        self.activation, self.dropout = (None if activation == "none" else activation), float(dropout)

    def forward(self, x: torch.Tensor, residual: torch.Tensor | None = None) -> torch.Tensor:
        H, W = self.grid or (0, 0)
        p = float(self.dropout) if self.training else 0.0
        if self.activation is not None or p > 0.0 or residual is not None:
            return _b._native().layer(x, self.weight, self.bias, residual, self.k, self.bases, self.save_projected,
                                      H, W, self.activation, p)
        return _b._native().linear(x, self.weight, self.bias, self.k, self.bases, self.save_projected, H, W)
