"""Paged caches for the tests, and rotation and attention in 64 bits with the bounds of the kernels' roundings (plain
torch on the CPU, written from the formulas)."""
from __future__ import annotations

import math

import torch

from paper_2402_04617_amd import infllm as F
from tests.shared_util import HALF, STEP, U32

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def params(Hq, Hkv, D, dtype, scale=1.0):
    return F.params(Hq, Hkv, D, 0, 1, 1, 1, 0, dtype=dtype, sm_scale=scale)


class Cache:
    """Pages of `n` sequences of `lens` tokens: every slot that no token takes, and spare pages, hold `fill`; table
    entries past a sequence's pages are 1 << 30."""

    def __init__(self, lens, Hkv, D, page, dtype, order="heads", seed=0, fill=math.nan, spare=2, device="cuda"):
        g = torch.Generator().manual_seed(seed)
        counts = [-(-x // page) for x in lens]
        n = sum(counts) + spare
        perm = torch.randperm(n, generator=g)
        self.page, self.order, self.lens, self.D, self.Hkv = page, order, list(lens), D, Hkv
        self.keys = [torch.randn((x, Hkv, D), generator=g).to(DT[dtype]) for x in lens]
        self.values = [torch.randn((x, Hkv, D), generator=g).to(DT[dtype]) for x in lens]
        self.table = torch.full((len(lens), max(1, max(counts, default=1))), 1 << 30, dtype=torch.int32)
        k = torch.full((n, page, Hkv, D), fill, dtype=DT[dtype])
        v = k.clone()
        at = 0
        for i, c in enumerate(counts):
            self.table[i, :c] = perm[at:at + c].to(torch.int32)
            at += c
            for cache, rows in ((k, self.keys[i]), (v, self.values[i])):
                for x in range(c):
                    part = rows[x * page:(x + 1) * page]
                    cache[int(self.table[i, x]), :len(part)] = part
        self.host_table = self.table.clone()
        if order == "heads":                       # [n][Hkv][page][D]
            self.k, self.v = (x.transpose(1, 2).contiguous().to(device) for x in (k, v))
            self.struct = F.pages(self.k, self.v, page)
        elif order == "tokens":                    # [n][page][Hkv][D]
            self.k, self.v = k.to(device), v.to(device)
            self.struct = F.pages(self.k, self.v, page, Hkv * page * D, Hkv * D, D)
        else:                                      # k and v side by side, a gap behind each row: [n][2][page][Hkv][D + 8]
            kv = torch.full((n, 2, page, Hkv, D + 8), fill, dtype=DT[dtype])
            kv[:, 0, ..., :D], kv[:, 1, ..., :D] = k, v
            self.kv = kv.to(device)
            self.k, self.v = self.kv[:, 0, ..., :D], self.kv[:, 1, ..., :D]
            self.struct = F.pages(self.k, self.v, page, 2 * page * Hkv * (D + 8), Hkv * (D + 8), D + 8)
        self.table = self.table.to(device)

    def slots(self, cache):
        """[page][slot][head][D] on the host."""
        return (cache.transpose(1, 2) if self.order == "heads" else cache).cpu()


def attend64(q, k, v, scale, seen, dtype, cap=0.0, bias=None, slope=0.0):
    """q [n][D], k, v [m][D] (float64), seen [n][m], bias [n][m] (to be added): the softmax attention, its
    log-sum-exp, and how far the kernels' results may be off, element by element.

    The score of a key: a product of D terms in float32 (D roundings of at most the sum of the absolute products),
    scaled; the cap 's derivative is at most 1 and its own formula a few roundings of the cap and of the score; the
    bias a few roundings of itself and of the bias across a tile of 64 keys; the base-2 exponential's argument a few
    roundings of the score.  That is the relative error e of the key's weight, and the sum of weight * e the
    normaliser's.  Then the float32 sums over the keys, each key one rounding.  bf16: a weight is rounded to bf16
    before it meets the values, a split part's row to fp16 relative to its largest value.  Then the output's own
    rounding.
    """
    z = (q @ k.T) * scale
    raw = (q.abs() @ k.nan_to_num(0, 0, 0).abs().T) * scale
    e = U32 * (2 * q.shape[1] * raw + 8 * (raw + 1))
    if cap:
        z = cap * torch.tanh(z / cap)
        e = e + 16 * U32 * cap
    if bias is not None:
        z = z + bias
        e = e + 8 * U32 * (bias.abs() + 64 * abs(slope))
    inf = torch.full_like(z, -math.inf)
    z = torch.where(seen, z, inf)
    some = seen.any(-1)
    lse = torch.logsumexp(z, dim=-1)
    p = torch.where(seen, torch.exp(z - lse[:, None]), torch.zeros_like(z))
    p = torch.where(some[:, None], p, torch.zeros_like(p))
    zero = torch.zeros((), dtype=torch.float64)
    out = torch.stack([torch.where(s[:, None], w[:, None] * v, zero).sum(0) for s, w in zip(seen, p)]) \
        if not torch.isfinite(v).all() else p @ v
    av = v.nan_to_num(0, 0, 0).abs()
    e = torch.where(seen, e, torch.zeros_like(e))
    pe = p.nan_to_num(0, 0, 0) * e.nan_to_num(0, 0, 0)
    a = p.nan_to_num(0, 0, 0) @ av
    e_norm = pe.sum(-1)
    e_sum = (k.shape[0] + 16) * U32
    tol = 2 * (pe @ av) + 2 * (e_norm + 2 * e_sum)[:, None] * a + STEP[dtype] * out.abs()
    if dtype == "bf16":
        tol = tol + STEP["bf16"] * a + HALF * a.amax(-1, keepdim=True)
    return out, lse, tol, 2 * e_norm + e_sum + 4 * U32 * lse.abs()


def seen_by(past, new, window=0, n_init=0):
    pos, t = torch.arange(past, past + new)[:, None], torch.arange(past + new)[None]
    seen = t <= pos
    if window:
        seen &= (t > pos - window) | (t < n_init)
    return seen


def rotate64(x, at, theta, interleaved, magnitude, norm, weight, eps, dtype):
    """x [token][head][D] (float64), at [token] (int64): normed and rotated, and how far a result in float32 rounded
    once may be off.

    The norm: a float32 sum of D squares (at most D roundings of it, halved by the root), the root, a quotient and
    two products: (D / 2 + 6) roundings of the value.  The rotation: an angle formed in float64 (two roundings of
    it), cosines and sines rounded to float32 with the magnitude, two products and a sum: 5 roundings of the sum of
    their absolute values.
    """
    D = x.shape[-1]
    e = torch.zeros((), dtype=torch.float64)
    if norm:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
        if weight is not None:
            x = x * weight
        e = (D / 2 + 6) * U32 * x.abs()
    n = len(theta)
    first = torch.arange(n) * (2 if interleaved else 1)
    second = first + (1 if interleaved else n)
    angle = at.double()[:, None] * torch.tensor(theta, dtype=torch.float64)
    off = (angle.abs() * 4 * 2.0 ** -53)[:, None] * abs(magnitude)
    c, s = (angle.cos() * magnitude)[:, None], (angle.sin() * magnitude)[:, None]
    y, tol = x.clone(), (e + torch.zeros_like(x))
    a, b = x[..., first], x[..., second]
    ea, eb = tol[..., first].clone(), tol[..., second].clone()
    y[..., first], y[..., second] = a * c - b * s, a * s + b * c
    both = a.abs() + b.abs()
    tol[..., first] = ea * c.abs() + eb * s.abs() + 5 * U32 * ((a * c).abs() + (b * s).abs()) + off * both
    tol[..., second] = ea * s.abs() + eb * c.abs() + 5 * U32 * ((a * s).abs() + (b * c).abs()) + off * both
    return y, tol + STEP[dtype] * y.abs()
