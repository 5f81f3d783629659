"""Packed prompts (infllm_prompt_attend) against attention in 64 bits (GPU)."""
import math

import pytest
import torch

from paper_2402_04617_amd import infllm as F
from tests.gpu_util import log
from tests.shared_util import attend64, check

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
MIXED = (1, 0, 63, 64, 65, 127, 0, 300, 2, 257)


def make(lens, Hq, Hkv, D, dtype, order, seed=0, scale=1.0, spare=3):
    """q, k, v, out tensors with `spare` rows behind the last sequence (NaN in q, k, v; 7 in out), their
    strides, and views [head][token][D] of them."""
    T = sum(lens) + spare
    g = torch.Generator().manual_seed(seed)
    if order == "heads":
        q, k, v = (torch.randn((h, T, D), generator=g) * s for h, s in ((Hq, scale), (Hkv, 1.0), (Hkv, 1.0)))
        q, k, v = (x.to(DT[dtype]).cuda() for x in (q, k, v))
        views = q, k, v
        qs = ks = (D, T * D)
    elif order == "tokens":
        q, k, v = (torch.randn((T, h, D), generator=g) * s for h, s in ((Hq, scale), (Hkv, 1.0), (Hkv, 1.0)))
        q, k, v = (x.to(DT[dtype]).cuda() for x in (q, k, v))
        views = tuple(x.transpose(0, 1) for x in (q, k, v))
        qs, ks = (Hq * D, D), (Hkv * D, D)
    else:  # one projection's output [token][q heads, k heads, v heads]
        x = torch.randn((T, Hq + 2 * Hkv, D), generator=g)
        x[:, :Hq] *= scale
        x = x.to(DT[dtype]).cuda()
        q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
        views = tuple(y.transpose(0, 1) for y in (q, k, v))
        qs = ks = ((Hq + 2 * Hkv) * D, D)
    for y in views:
        y[:, sum(lens):] = math.nan
    out = torch.full((T, Hq, D) if order != "heads" else (Hq, T, D), 7.0, dtype=DT[dtype], device="cuda")
    os = (D, T * D) if order == "heads" else (Hq * D, D)
    return q, k, v, out, qs, ks, os, views


def attend(p, lens, q, k, v, out, qs, ks, os, stream=None):
    lse = torch.full((p.n_q_heads, max(1, sum(lens))), 7.0, dtype=torch.float32, device="cuda")
    size = F.infllm_prompt_workspace_bytes(p, lens)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda") if size else None
    F.infllm_prompt_attend(p, lens, q, qs, k, v, ks, out, os, lse, ws, stream=stream)
    return lse


def verify(lens, views, out, lse, Hq, Hkv, order, dtype, scale):
    q, k, v = (x.double().cpu() for x in views)
    o = (out if order == "heads" else out.transpose(0, 1)).cpu()
    at = 0
    for n in lens:
        seen = torch.ones((n, n), dtype=torch.bool).tril()
        for h in range(Hq if n else 0):
            kv = h // (Hq // Hkv)
            w = attend64(q[h, at:at + n], k[kv, at:at + n], v[kv, at:at + n], scale, seen, dtype)
            check(f"out, {n} tokens at {at}, head {h}", o[h, at:at + n], w[0], w[2])
            check(f"lse, {n} tokens at {at}, head {h}", lse[h, at:at + n], w[1], w[3])
        at += n
    assert torch.all(o[:, at:] == 7), "rows behind the last sequence were written"


@pytest.mark.parametrize("dtype,Hq,Hkv,D,order,lens", [
    ("bf16", 4, 1, 128, "heads", (1,)),
    ("bf16", 8, 2, 128, "fused", MIXED),
    ("bf16", 8, 2, 64, "tokens", MIXED),
    ("bf16", 3, 3, 128, "heads", (31, 33, 256, 255)),
    ("bf16", 6, 2, 64, "fused", (129, 5)),
    ("bf16", 16, 2, 128, "tokens", (700, 3, 90)),
    ("bf16", 32, 8, 128, "heads", (1100,)),
    ("bf16", 5, 1, 128, "tokens", (0, 513, 0)),
    ("bf16", 2, 1, 64, "heads", (2500,)),
    ("f32", 4, 1, 128, "heads", (1,)),
    ("f32", 4, 2, 64, "fused", MIXED),
    ("f32", 3, 1, 128, "tokens", (33, 100, 7)),
    ("f32", 8, 8, 64, "heads", (64, 65)),
    ("f32", 2, 1, 64, "tokens", (1500,)),
])
def test_prompt_parity(dtype, Hq, Hkv, D, order, lens):
    log(f"[prompt] {dtype} {Hq}/{Hkv} D={D} {order} {lens}")
    scale = D ** -0.5
    p = F.params(Hq, Hkv, D, 0, 4096, 128, 4, 0, dtype, sm_scale=scale)
    q, k, v, out, qs, ks, os, views = make(lens, Hq, Hkv, D, dtype, order)
    lse = attend(p, lens, q, k, v, out, qs, ks, os)
    verify(lens, views, out, lse, Hq, Hkv, order, dtype, scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompt_many_sequences(dtype):
    """More sequences than one launch takes, most of them a few tokens or none."""
    lens = [i % 4 for i in range(600)] + [70] + [i % 3 for i in range(40)]
    log(f"[prompt] {dtype} {len(lens)} sequences")
    p = F.params(4, 2, 64, 0, 4096, 128, 4, 0, dtype, sm_scale=0.125)
    q, k, v, out, qs, ks, os, views = make(lens, 4, 2, 64, dtype, "tokens")
    lse = attend(p, lens, q, k, v, out, qs, ks, os)
    verify(lens, views, out, lse, 4, 2, "tokens", dtype, 0.125)


@pytest.mark.parametrize("dtype,Hq,Hkv,D,lens", [
    ("bf16", 4, 1, 128, (4000,)), ("bf16", 2, 2, 64, (3000, 2999, 64, 1)), ("bf16", 8, 1, 128, (0, 1500, 1400, 7)),
    ("f32", 4, 1, 128, (900, 33)), ("f32", 2, 1, 64, (2000, 1999)),
])
def test_prompt_split_keys(dtype, Hq, Hkv, D, lens):
    """Prompts whose longest row tiles are split along the keys, without an lse as well."""
    log(f"[prompt] {dtype} {Hq}/{Hkv} D={D} {lens} split")
    p = F.params(Hq, Hkv, D, 0, 4096, 128, 4, 0, dtype, sm_scale=D ** -0.5)
    assert F.infllm_prompt_workspace_bytes(p, lens) > 0
    q, k, v, out, qs, ks, os, views = make(lens, Hq, Hkv, D, dtype, "tokens")
    lse = attend(p, lens, q, k, v, out, qs, ks, os)
    verify(lens, views, out, lse, Hq, Hkv, "tokens", dtype, D ** -0.5)
    again = torch.full_like(out, 7.0)
    ws = torch.empty(F.infllm_prompt_workspace_bytes(p, lens), dtype=torch.uint8, device="cuda")
    F.infllm_prompt_attend(p, lens, q, qs, k, v, ks, again, os, None, ws)
    assert torch.equal(again, out)
    with pytest.raises(F.InfllmError):
        F.infllm_prompt_attend(p, lens, q, qs, k, v, ks, again, os, None, ws, workspace_bytes=ws.numel() - 256)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompt_steep_scores(dtype):
    """Scores of some hundreds: one key takes nearly all of a row, and the running maximum moves by jumps."""
    lens = (300, 150)
    log(f"[prompt] {dtype} steep scores")
    p = F.params(4, 2, 64, 0, 4096, 128, 4, 0, dtype, sm_scale=1.0)
    q, k, v, out, qs, ks, os, views = make(lens, 4, 2, 64, dtype, "heads", scale=6.0)
    lse = attend(p, lens, q, k, v, out, qs, ks, os)
    verify(lens, views, out, lse, 4, 2, "heads", dtype, 1.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("what,bad", [("v", math.inf), ("v", math.nan), ("k", math.nan), ("q", math.nan)])
def test_prompt_not_finite_stays(dtype, what, bad):
    """A value that is not finite reaches the rows that see it, and those alone."""
    lens = (100, 200)
    at, seq = 170, (100, 300)  # in the second sequence, inside a tile
    log(f"[prompt] {dtype} {what}={bad}")
    p = F.params(4, 2, 128, 0, 4096, 128, 4, 0, dtype, sm_scale=0.1)
    q, k, v, out, qs, ks, os, views = make(lens, 4, 2, 128, dtype, "heads")
    {"q": q, "k": k, "v": v}[what][1, at, 5] = bad
    lse = attend(p, lens, q, k, v, out, qs, ks, os)
    rows = slice(at, at + 1) if what == "q" else slice(at, seq[1])
    heads = [1] if what == "q" else [2, 3]
    odd = torch.zeros((4, sum(lens)), dtype=torch.bool)
    for h in heads:
        odd[h, rows] = True
    if what == "v":
        assert torch.all(torch.isfinite(lse))
        got = ~torch.isfinite(out[:, :sum(lens)].float()).cpu()
        assert torch.equal(got[..., 5], odd) and not got[..., :5].any() and not got[..., 6:].any()
        if bad == math.inf:
            assert torch.all(out[:, :sum(lens), 5][odd.cuda()] == math.inf)
    else:
        assert torch.equal(torch.isnan(lse).cpu(), odd)
        assert torch.equal(torch.isnan(out[:, :sum(lens)].float()).all(-1).cpu(), odd)
        assert torch.equal(torch.isnan(out[:, :sum(lens)].float()).any(-1).cpu(), odd)
    # the other rows as without it
    {"q": q, "k": k, "v": v}[what][1, at, 5] = 0.5
    clean = torch.full_like(out, 7.0)
    clean_lse = attend(p, lens, q, k, v, clean, qs, ks, os)
    o, c = out[:, :sum(lens)], clean[:, :sum(lens)]
    if what == "v":
        o[..., 5] = c[..., 5]
        assert torch.equal(lse, clean_lse)
    else:
        o[odd.cuda()] = c[odd.cuda()]
        lse[odd.cuda()] = clean_lse[odd.cuda()]
    verify(lens, views, out, lse, 4, 2, "heads", dtype, 0.1)


def test_prompt_repeats_streams_and_graphs():
    """Bitwise the same on another stream and in a replayed graph, whose inputs change between replays."""
    lens = (1, 130, 64, 777)
    p = F.params(8, 2, 128, 0, 4096, 128, 4, 0, "bf16", sm_scale=0.088)
    a = make(lens, 8, 2, 128, "bf16", "tokens", seed=1)
    b = make(lens, 8, 2, 128, "bf16", "tokens", seed=2)
    want = []
    for x in (a, b):
        lse = attend(p, lens, *x[:7])
        want.append((x[3].clone(), lse))
    log("[prompt] another stream")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a[3].fill_(0)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        lse = attend(p, lens, *a[:7])
    torch.cuda.current_stream().wait_stream(side)
    n = sum(lens)
    assert torch.equal(a[3][:n], want[0][0][:n]) and torch.equal(lse, want[0][1])
    log("[prompt] graph")
    ins = [x.clone() for x in a[:3]]
    out = torch.empty_like(a[3])
    lse = torch.empty_like(want[0][1])
    size = F.infllm_prompt_workspace_bytes(p, lens)
    ws = torch.empty(max(16, size), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        F.infllm_prompt_attend(p, lens, ins[0], a[4], ins[1], ins[2], a[5], out, a[6], lse, ws)
    for r in (1, 0, 1, 0):
        for x, y in zip(ins, (a, b)[r][:3]):
            x.copy_(y)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[:n], want[r][0][:n]) and torch.equal(lse, want[r][1])
