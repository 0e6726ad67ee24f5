"""Attention under changed scores in 64 bits from its definition, and how far an output of the
GPU's may lie from it.

Tolerance of one output of the kernels: it is rounded once to bf16 (half a step, 2^-8 of it).  Weights
are rounded to bf16, each by at most 2^-8 of itself, and the normaliser sums the rounded ones; a score's
error of `dl` moves its weight by as much.  With p the exact weights and every one off by a factor of at
most 1 + x, the output moves by at most x sum_j p_j |v_j - out| (to first order; 1 + 2^-7 covers
the rest), and that sum is at most dev = sqrt(sum_j p_j v_j^2 - out^2).  So
  tol = 2^-8 |out| + (2^-8 + dl) (1 + 2^-7) dev + 1e-6 max |v|    (the sums' own rounding in fp32).
A score q.k / sqrt d is a sum of d products in fp32, off by at most d 2^-24 sum |q_c k_c| / sqrt d; a cap's
tanh by 2^-20 of the cap; scaling, bias, reference and the exponential add a few steps (2^-22 together) of
the logits' size, of which only those within some 64 of the row's largest have weight; and a bias is
that of a tile's first key, up to 128 slopes, and what its 63 others add, from which the d products' sum
starts: (d 63 + 128) 2^-24 < 2^-10.9 slopes.
"""
from __future__ import annotations

import torch

HALF = 2.0 ** -8  # half a step of bf16


def change(a, cap, bias):
    """Scores a in 64 bits, capped and biased."""
    if cap:
        a = cap * torch.tanh(a / cap)
    return a if bias is None else a + bias


def attend(q, k, v, vis, cap=0.0, bias=None):
    """Rows q [rows, d] over keys k, v [keys, d] where vis [rows, keys]: (out, log-sum-exp, dev, dl)."""
    q, k, v = (x.double() for x in (q, k, v))
    d = q.shape[1]
    a = change(q @ k.T / d ** 0.5, cap, bias)
    none = torch.full_like(a, float("-inf"))
    a = torch.where(vis, a, none)
    some = vis.any(1)
    top = torch.where(some, a.max(1).values if a.shape[1] else a.new_zeros(len(a)), a.new_zeros(len(a)))
    p = torch.exp(a - top[:, None])
    z = p.sum(1)
    p = p / torch.where(z > 0, z, torch.ones_like(z))[:, None]
    out = p @ v
    dev = (p @ v ** 2 - out ** 2).clamp(min=0).sqrt()
    sums = d * 2.0 ** -24 * float((q.abs() @ k.abs().T).max()) / d ** 0.5 if a.numel() else 0.0
    size = float(top.abs().max()) if len(top) else 0.0
    slope = float((bias[:, 1:] - bias[:, :-1]).abs().max()) if bias is not None and bias.shape[1] > 1 else 0.0
    dl = 2 * (sums + cap * 2.0 ** -20 + 2.0 ** -22 * (2 * size + 64) + slope * (63 * d + 128) * 2.0 ** -24)
    return out, torch.where(z > 0, top + torch.log(z), torch.full_like(z, float("-inf"))), dev, dl


def tolerance(out, dev, dl, top):
    return HALF * out.abs() + (HALF + dl) * (1 + 2.0 ** -7) * dev + 1e-6 * top


def slopes_of(Hq):
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / Hq) for h in range(Hq)])
