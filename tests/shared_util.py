"""Attention in 64 bits with the bounds of the kernels' roundings, for the tests of packed prompts and
shared documents (plain torch on the CPU, written from the formulas)."""
from __future__ import annotations

import math

import torch

STEP = {"bf16": torch.finfo(torch.bfloat16).eps / 2, "f32": torch.finfo(torch.float32).eps / 2}
HALF = torch.finfo(torch.float16).eps / 2
U32 = torch.finfo(torch.float32).eps / 2


def attend64(q, k, v, scale, seen, dtype):
    """q [n][D], k, v [m][D] (float64), seen [n][m]: the softmax attention, its log-sum-exp, and how far the
    kernels' results may be off, element by element.

    Scores: products of D terms summed in float32 (D roundings of at most the sum of the absolute products),
    scaled and exponentiated in the base-2 domain (a few roundings of the score itself): e_z.  The weights'
    relative error is 2 e_z (numerator and normaliser) plus the float32 sums over the keys, each key one
    rounding.  bf16: a weight is rounded to bf16 before it meets the values, a split part's row to fp16 relative
    to its largest value, so A = sum of weight * |v| is off by STEP + HALF of itself (the row's largest value
    for the latter).  Then the output's own rounding.
    """
    n = q.shape[0]
    if k.shape[0] == 0:
        z = torch.zeros_like(q)
        return z, torch.full((n,), -math.inf, dtype=torch.float64), z, torch.zeros(n, dtype=torch.float64)
    z = (q @ k.T) * scale
    # what a row does not see is not looked at (it may hold anything)
    z = torch.where(seen, z, torch.full_like(z, -math.inf))
    lse = torch.logsumexp(z, dim=-1)
    p = torch.where(seen, torch.exp(z - lse[:, None]), torch.zeros_like(z))
    p = torch.where(seen.any(-1, keepdim=True), p, torch.zeros_like(p))
    out = (p[:, :, None] * v[None]).where(seen[:, :, None], torch.zeros((), dtype=torch.float64)).sum(1) if not torch.isfinite(v).all() else p @ v
    a = p @ v.nan_to_num(0, 0, 0).abs()
    big = torch.where(seen, (q.abs() @ k.nan_to_num(0, 0, 0).abs().T) * scale, torch.zeros_like(z)).amax(-1)
    e_z = 2 * U32 * (q.shape[1] * big + 4 * big + 4)
    e_sum = (k.shape[0] + 16) * U32
    rel = 2 * e_z + 2 * e_sum
    tol = rel[:, None] * a + STEP[dtype] * out.abs()
    if dtype == "bf16":
        tol = tol + STEP["bf16"] * a + HALF * a.amax(-1, keepdim=True)
    tol_lse = e_z + e_sum + 4 * U32 * lse.abs()
    return out, lse, tol, tol_lse


def check(name, got, want, tol):
    """Same places finite, equal where not (NaN with NaN), within tol elsewhere."""
    got, want = got.double().cpu(), want.double()
    fine = torch.isfinite(want)
    assert torch.equal(fine, torch.isfinite(got)), f"{name}: finite in other places: {(fine != torch.isfinite(got)).sum().item()} of {fine.numel()}"
    assert torch.equal(torch.isnan(want), torch.isnan(got)), f"{name}: NaN in other places"
    inf = torch.isinf(want)
    assert torch.equal(want[inf], got[inf]), f"{name}: infinities differ"
    off = torch.where(fine, (got - want).abs() - tol.double().expand_as(want), torch.full_like(want, -1.0))
    at = int(off.argmax())
    assert off.max() <= 0, f"{name}: off by {(got - want).abs().flatten()[at]:.3g} at {at}, {tol.expand_as(want).flatten()[at]:.3g} allowed"
