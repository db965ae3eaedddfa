"""Rotations learned for rows that are kept in 4 bits, one for every region (or one for all: a single group).

A row x is kept as the 4-bit values of R x, R the rotation of its region.  For given values v the orthogonal R with the least
sum of ||R x - v||^2 is the orthogonal factor of sum v x^T, and for a given R the nearest values are the rounded ones, so that
the two are found in turn (the alternation by which a rotation in front of a product quantiser is learned, Section 4, OPQ).
Every step is one of the library's operators: the rows' products with their region's matrix, rounding to 4 bits and back,
the regions' cross-covariances (the gradient of that product), and their orthogonal factors by Newton-Schulz steps.
"""
from __future__ import annotations

import torch

from . import binding as B

# towards the orthogonal factor: 12 steps take singular values from 2e-3 of the Frobenius norm to 1
POLAR = [(1.875, -1.25, 0.375)] * 12


@torch.no_grad()
def learn(x: torch.Tensor, offsets: torch.Tensor, rounds: int = 8, hold: float = 0.05, start: torch.Tensor | None = None):
    """Rotations [G, D, D] fp32 for the rows x [n, D] fp32, group by group at ``offsets`` [G + 1], and the mean squared error of their 4-bit
    values after every round.  ``hold`` (of a cross-covariance's norm over sqrt(D)) draws towards the rotation of the round before, which
    decides where a region has fewer rows than components."""
    D, G = x.shape[1], offsets.shape[0] - 1
    R = torch.eye(D, device=x.device).expand(G, D, D).contiguous() if start is None else start
    errors = []
    for step in range(rounds + 1):
        y = B.ivf_grouped_product(x, R, offsets)
        v = B.ivf_mx4_expand(B.ivf_mx4_quantise(y))
        errors.append((y - v).square().sum(1).mean())
        if step < rounds:
            M = B.ivf_grouped_gradient(v, x, offsets)
            weight = hold * M.flatten(1).norm(dim=1) / D ** 0.5 + 1e-30
            R = B.ivf_orthogonalise(M + weight[:, None, None] * R, POLAR, eps=0.0)   # (a region without rows keeps its rotation)
    return R, torch.stack(errors)


@torch.no_grad()
def keep(x: torch.Tensor, R: torch.Tensor, offsets: torch.Tensor) -> B.Mx4Rows:
    """The rows x, rotated by their groups' matrices, in 4 bits."""
    return B.ivf_mx4_quantise(B.ivf_grouped_product(x, R, offsets))
