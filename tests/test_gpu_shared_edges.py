"""Prompts and shared documents where their code takes another way (GPU): lookups longer than what a workgroup keeps
of them, several launches that each split their longest prompts, and bits that a bad value elsewhere does not move."""
import math

import pytest
import torch

from paper_2402_04617_amd import infllm as F
from tests.gpu_util import log
from tests.shared_util import attend64, check
from tests.test_gpu_prefix import Case, params
from tests.test_gpu_prompt import attend, make, verify

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,D,init,block,k_m,n_q", [
    ("bf16", 64, 16, 8, 1300, 1), ("bf16", 128, 3, 5, 1100, 3), ("bf16", 64, 0, 8, 1026, 40),
    ("f32", 64, 16, 4, 2300, 1), ("f32", 128, 3, 3, 2050, 20),
])
def test_long_lookups(dtype, D, init, block, k_m, n_q):
    """More entries than LDS holds (1,024 and 2,048), skipped ones on both sides of that; then a value that is not
    finite in a unit that some rows look up behind it."""
    log(f"[prefix] {dtype} D={D} {k_m} units of {block}, n_q={n_q}")
    B, length = 2, init + (k_m + 60) * block + 100 + 7
    c = Case(params(4, 2, D, dtype, local=100, init=init, block=block, topk=k_m), B, n_q, length, (9, 0), seed=k_m)
    assert c.part.n_units >= k_m
    g = torch.Generator().manual_seed(n_q)
    for b in range(B):
        for h in range(2):
            at = torch.randint(k_m, (k_m // 9,), generator=g).cuda()
            c.idx[b, h, at] = torch.tensor([-1, c.part.n_units, 2 ** 31 - 1], dtype=torch.int32).cuda()[at % 3]
    c.idx[0, 0, -2:] = torch.tensor([-5, c.part.n_units - 1], dtype=torch.int32)
    u = c.part.n_units - 1  # (the last entry of continuation 0, kv head 0; its rows may hold NaN so far)
    rows = slice(init + u * block, init + (u + 1) * block)
    for t in (c.k, c.v):
        t[0, rows] = torch.randn((block, D), generator=g).to(c.dt)
    c.run()
    c.verify()
    c.v[0, rows, 7] = math.inf
    c.run()
    c.verify()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompt_launches_that_split(dtype):
    """Two launches of 256 and fewer sequences, each with prompts whose keys are split, in one workspace."""
    lens = [1, 0, 2000] + [1 + i % 3 for i in range(254)] + [1700, 0, 3, 1650, 64]
    p = F.params(2, 1, 64, 0, 4096, 128, 4, 0, dtype, sm_scale=0.125)
    full = [n for n in lens if n]
    sizes = [F.infllm_prompt_workspace_bytes(p, x) for x in (full[:256], full[256:], lens)]
    log(f"[prompt] {dtype} {len(full)} sequences, workspaces {sizes}")
    assert len(full) > 256 and min(sizes) > 0 and sizes[2] == max(sizes)
    q, k, v, out, qs, ks, os, views = make(lens, 2, 1, 64, dtype, "tokens")
    lse = attend(p, lens, q, k, v, out, qs, ks, os)
    verify(lens, views, out, lse, 2, 1, "tokens", dtype, 0.125)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prefix_bits_beside_bad_values(dtype):
    """Values that are not finite leave the bits of other kv heads, and of other continuations where they are a
    continuation's own."""
    c = Case(params(6, 3, 128, dtype), 3, 4, 1500, (7, 100, 60))
    c.run()
    clean, lse = c.out.clone(), c.lse.clone()
    log(f"[prefix] {dtype} bits beside bad values")
    c.xv[0, 1, 2, 9] = math.inf   # heads 2 and 3
    c.q[2, 3, 1, 4] = math.nan
    c.ok[1, 0, 3, 0] = math.nan   # heads 0 and 1
    c.run()
    for b, heads in ((0, (0, 1, 4, 5)), (1, (4, 5)), (2, (0, 1, 4, 5))):
        for h in heads:
            assert torch.equal(c.out[b, h], clean[b, h]) and torch.equal(c.lse[b, h], lse[b, h]), (b, h)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("what", ["q", "k", "v"])
def test_prompt_bits_beside_bad_values(dtype, what):
    """And of other sequences and kv heads in packed prompts, split ones among them."""
    lens = (100, 1500, 30)
    p = F.params(4, 2, 64, 0, 4096, 128, 4, 0, dtype, sm_scale=0.125)
    q, k, v, out, qs, ks, os, _ = make(lens, 4, 2, 64, dtype, "heads")
    lse = attend(p, lens, q, k, v, out, qs, ks, os)
    again = torch.full_like(out, 7.0)
    log(f"[prompt] {dtype} bits beside a bad {what}")
    {"q": q, "k": k, "v": v}[what][1, 170, 5] = math.nan
    bad = attend(p, lens, q, k, v, again, qs, ks, os)
    heads = slice(1, 2) if what == "q" else slice(2, 4)
    assert torch.isnan(again[heads, 170, 5].float()).all()
    group = slice(0, 2) if what == "q" else heads
    for x, y in ((out, again), (lse, bad)):
        x[group, 100:1600] = y[group, 100:1600] = 0  # (NaN in part, and not equal to itself)
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_units_given_twice(dtype):
    """An entry that stands in a row twice counts twice."""
    c = Case(params(4, 2, 64, dtype, topk=6), 3, 2, 1500, (7, 0, 60))
    c.idx[:, :, 3] = c.idx[:, :, 0]
    c.idx[1, 0, :] = c.idx[1, 0, 2].clone()
    log(f"[prefix] {dtype} entries given twice")
    c.run()
    c.verify()


@pytest.mark.parametrize("dtype,parts,rows", [("bf16", 2, 40), ("bf16", 12, 40), ("f32", 3, 40), ("f32", 20, 2000), ("bf16", 20, 2000)])
def test_merge_of_nan_parts(dtype, parts, rows):
    """A part whose lse is NaN makes its row NaN, lse and all; one of -inf is left out."""
    D, bad, empty = 64, rows // 3, rows // 2
    p = F.params(1, 1, D, 0, 64, 8, 2, 0, dtype)
    g = torch.Generator().manual_seed(parts)
    o = (torch.randn((parts, rows, D), generator=g) * 100).to(torch.float16 if dtype == "bf16" else torch.float32)
    l = torch.randn((parts, rows), generator=g)
    l[1, bad] = math.nan
    l[0, empty] = -math.inf
    pieces = [o, l] + ([torch.zeros((parts, rows), dtype=torch.int32)] if dtype == "bf16" else [])
    ws = torch.cat([x.contiguous().view(torch.uint8).flatten() for x in pieces]).cuda()
    out = torch.empty((1, 1, rows, D), dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
    lse = torch.empty((1, 1, rows), device="cuda")
    log(f"[merge] {dtype} {parts} parts of {rows} rows, a NaN")
    F.infllm_lse_merge(p, 1, rows, parts, ws, out, rows * D, lse)
    want = torch.logsumexp(l.double(), 0)
    w = torch.exp(l.double() - want)
    ref = (w[:, :, None] * o.double()).sum(0)
    ref[bad] = want[bad] = math.nan
    # parts + 8 float32 roundings of sums of weights, exponentials of scores up to 8
    a = (w[:, :, None] * o.double().abs()).sum(0)
    half = torch.finfo(out.dtype).eps / 2
    tol = 2 * (parts + 32) * 2.0 ** -24 * a + half * ref.abs()
    check("out", out[0, 0], ref, tol.nan_to_num())
    check("lse", lse[0, 0], want, torch.full((rows,), (parts + 64) * 2.0 ** -24))
