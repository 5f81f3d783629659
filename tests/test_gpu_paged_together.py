"""Rotation, appends and attention on paged caches together, as a serving program runs them (GPU)."""
import math

import pytest
import torch

from paper_2402_04617_amd import infllm as F
from tests.paged_util import DT, Cache, attend64, params, rotate64, seen_by
from tests.shared_util import check

pytestmark = pytest.mark.gpu

HQ, HKV = 8, 2


class Layer:
    """A layer's pages and what its program keeps; sequences whose tokens arrive in pieces."""

    def __init__(self, lens, D, page, dtype, form=None, seed=0):
        self.D, self.page, self.dtype, self.lens = D, page, dtype, lens
        self.p = params(HQ, HKV, D, dtype, D ** -0.5)
        g = torch.Generator().manual_seed(seed)
        self.x = [torch.randn((n, HQ + 2 * HKV, D), generator=g).to(DT[dtype]) for n in lens]  # projections of all tokens
        self.wq, self.wk = ((1 + 0.2 * torch.randn(D, generator=g)).to(DT[dtype]) for _ in range(2))
        self.theta = F.infllm_rope_frequencies(D, 10000.0, "parts", 4.0, 1024)
        self.rot = F.rotary(self.theta, False, 1.1, True, self.wq.cuda(), self.wk.cuda(), 1e-5)
        # empty pages, full of NaN
        counts = [-(-n // page) for n in lens]
        n = sum(counts) + 1
        self.k = torch.full((n, HKV, page, D), math.nan, dtype=DT[dtype], device="cuda")
        self.v = self.k.clone()
        self.pages = F.pages(self.k, self.v, page)
        perm = torch.randperm(n, generator=g).to(torch.int32)
        self.table = torch.full((len(lens), max(counts)), -1, dtype=torch.int32)
        at = 0
        for i, c in enumerate(counts):
            self.table[i, :c] = perm[at:at + c]
            at += c
        self.table = self.table.cuda()
        self.form = dict(form or {})
        self.score = F.score(**self.form) if form else None

    def inputs(self, news, pasts):
        return torch.cat([self.x[i][b:b + a] for i, (a, b) in enumerate(zip(news, pasts))])

    def workspace(self, news, pasts):
        return torch.empty(max(256, F.infllm_paged_workspace_bytes(self.p, self.pages, news, pasts, self.score)), dtype=torch.uint8, device="cuda")

    def step(self, qkv, news, pasts, q, out, lse, ws, stream=None):
        D, row = self.D, (HQ + 2 * HKV) * self.D
        F.infllm_paged_append(self.p, self.rot, self.pages, news, pasts, self.table, qkv, (row, D), q, (HQ * D, D), qkv[:, HQ:], qkv[:, HQ + HKV:],
                              (row, D), stream=stream)
        F.infllm_paged_attend(self.p, self.pages, news, pasts, self.table, self.score, q, (HQ * D, D), out, (HQ * D, D), lse, ws, stream=stream)

    def buffers(self, total):
        return (torch.empty((total, HQ, self.D), dtype=DT[self.dtype], device="cuda"), torch.empty((total, HQ, self.D), dtype=DT[self.dtype], device="cuda"),
                torch.empty((HQ, total), dtype=torch.float32, device="cuda"))

    def verify(self, news, pasts, q, out, lse):
        """Queries and keys against their rotation in 64 bits, and the attention of the rows the device has."""
        row = 0
        for i, (new, past) in enumerate(zip(news, pasts)):
            end = past + new
            if new == 0:
                continue
            at = torch.arange(end)
            held = self.table[i].cpu()[at // self.page].long()
            keys, values = self.k.cpu()[held, :, at % self.page], self.v.cpu()[held, :, at % self.page]
            x = self.x[i][:end].double()
            eps, mag = float(torch.tensor(1e-5)), float(torch.tensor(1.1))
            args = (at, self.theta, False, mag, True)
            want, tol = rotate64(x[:, HQ:HQ + HKV], *args, self.wk.double(), eps, self.dtype)
            check(f"keys of sequence {i}", keys, want, tol)
            assert torch.equal(values, self.x[i][:end, HQ + HKV:])
            want, tol = rotate64(x[past:, :HQ], at[past:], *args[1:], self.wq.double(), eps, self.dtype)
            check(f"queries of sequence {i}", q[row:row + new], want, tol)
            seen = seen_by(past, new, self.form.get("window", 0), self.form.get("n_init", 0))
            for h in range(HQ):
                w = attend64(q[row:row + new, h].double().cpu(), keys[:, h // (HQ // HKV)].double(), values[:, h // (HQ // HKV)].double(),
                             self.D ** -0.5, seen, self.dtype, self.form.get("softcap", 0.0))
                check(f"out of sequence {i}, head {h}", out[row:row + new, h], w[0], w[2])
                check(f"lse of sequence {i}, head {h}", lse[h, row:row + new], w[1], w[3])
            row += new


ROUNDS = [((70, 1, 33), (0, 0, 0)), ((64, 0, 1), (70, 1, 33)), ((1, 200, 1), (134, 1, 34)), ((1, 1, 1), (135, 201, 35)), ((5, 8, 0), (136, 202, 36))]


@pytest.mark.parametrize("dtype,D,page,form", [
    ("bf16", 128, 16, None), ("bf16", 64, 20, dict(window=60, n_init=4)), ("f32", 64, 16, dict(softcap=8.0)), ("f32", 128, 5, None)])
def test_prompts_in_chunks_then_steps(dtype, D, page, form):
    a = Layer((141, 210, 36), D, page, dtype, form)
    for news, pasts in ROUNDS:
        q, out, lse = a.buffers(sum(news))
        a.step(a.inputs(news, pasts).cuda(), news, pasts, q, out, lse, a.workspace(news, pasts))
        a.verify(news, pasts, q, out, lse)


def test_the_same_as_packed_prompts():
    """Whole prompts through pages, and rotated in place and attended packed."""
    lens = (130, 1, 77)
    a = Layer(lens, 128, 16, "bf16")
    total, row = sum(lens), (HQ + 2 * HKV) * 128
    q, out, lse = a.buffers(total)
    qkv = a.inputs(lens, (0, 0, 0)).cuda()
    a.step(qkv, lens, (0, 0, 0), q, out, lse, a.workspace(lens, (0, 0, 0)))
    at = torch.cat([torch.arange(n) for n in lens]).cuda()
    F.infllm_rotate(a.p, a.rot, total, at, qkv, (row, 128), qkv, (row, 128), qkv[:, HQ:], (row, 128), qkv[:, HQ:], (row, 128))
    assert torch.equal(qkv[:, :HQ], q), "the append rotates as the rotation does"
    o, l = torch.empty_like(out), torch.empty_like(lse)
    ws = torch.empty(max(256, F.infllm_prompt_workspace_bytes(a.p, lens)), dtype=torch.uint8, device="cuda")
    F.infllm_prompt_attend(a.p, lens, qkv, (row, 128), qkv[:, HQ:], qkv[:, HQ + HKV:], (row, 128), o, (HQ * 128, 128), l, ws)
    # (each within its own bound of 64 bits, so within twice the larger)
    row0 = 0
    for n in lens:
        x = qkv[row0:row0 + n].double().cpu()
        for h in range(HQ):
            kv = h // (HQ // HKV)
            w = attend64(x[:, h], x[:, HQ + kv], x[:, HQ + HKV + kv], 128 ** -0.5, seen_by(0, n), "bf16")
            check("packed", o[row0:row0 + n, h], out[row0:row0 + n, h].double().cpu(), 2 * w[2])
            check("packed lse", l[h, row0:row0 + n], lse[h, row0:row0 + n].double().cpu(), 2 * w[3])
        row0 += n


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_window_is_the_step_without_units(dtype):
    """A decoding step over a memory with units of one token, none looked up: the initial tokens, the last n_local and
    the token itself."""
    D, past, n_init, n_local = 64, 700, 10, 100
    r = Cache([past + 1], HKV, D, 16, dtype)
    p = F.params(HQ, HKV, D, n_init, n_local, 1, 1, 0, dtype=dtype, sm_scale=D ** -0.5)
    g = torch.Generator().manual_seed(9)
    q = torch.randn((1, HQ, D), generator=g).to(DT[dtype]).cuda()
    k, v = (x.transpose(0, 1).contiguous().cuda()[None] for x in (r.keys[0], r.values[0]))
    m = F.Memory(batch=1, capacity=past + 1, k=k.data_ptr(), v=v.data_ptr())
    out, lse = torch.empty_like(q), torch.empty((1, HQ, 1), device="cuda")
    ws = torch.empty(F.infllm_workspace_bytes(p, 1, 1), dtype=torch.uint8, device="cuda")
    F.infllm_chunk_attend(p, m, q, D, 1, past, torch.zeros(4, dtype=torch.int32, device="cuda"), 0, out, D, lse, ws)
    score = F.score(window=n_local + 1, n_init=n_init)
    o, l = torch.empty_like(q), torch.empty((HQ, 1), device="cuda")
    ws = torch.empty(max(256, F.infllm_paged_workspace_bytes(p, r.struct, [1], [past], score)), dtype=torch.uint8, device="cuda")
    F.infllm_paged_attend(p, r.struct, [1], [past], r.table, score, q, (HQ * D, D), o, (HQ * D, D), l, ws)
    for h in range(HQ):
        w = attend64(q[:, h].double().cpu(), r.keys[0][:, h // 4].double(), r.values[0][:, h // 4].double(), D ** -0.5,
                     seen_by(past, 1, n_local + 1, n_init), dtype)
        check("paged", o[:, h], w[0], w[2])
        check("step", out[:, h], w[0], w[2])
        check("lse", l[h], lse[0, h].double().cpu(), 2 * w[3])


@pytest.mark.parametrize("dtype,D,page", [("bf16", 128, 16), ("bf16", 64, 12), ("f32", 64, 16)])
def test_replayed_graphs(dtype, D, page):
    """Two captured steps with workspaces of their own, replayed by turns with new inputs and eager work between."""
    a = Layer((300, 2100, 40), D, page, dtype)
    first = (299, 2099, 0), (0, 0, 0)
    q, out, lse = a.buffers(sum(first[0]))
    a.step(a.inputs(*first).cuda(), *first, q, out, lse, a.workspace(*first))
    calls = [((1, 1, 30), (299, 2099, 0)), ((1, 1, 40), (299, 2099, 0))]
    graphs = []
    for news, pasts in calls:
        qkv = a.inputs(news, pasts).cuda()
        bufs, ws = a.buffers(sum(news)), a.workspace(news, pasts)
        a.step(qkv, news, pasts, *bufs, ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            a.step(qkv, news, pasts, *bufs, ws)
        graphs.append((graph, news, pasts, qkv, bufs, ws))
    gen = torch.Generator().manual_seed(11)
    for turn in range(6):
        graph, news, pasts, qkv, bufs, ws = graphs[turn % 2]
        x = torch.randn(qkv.shape, generator=gen).to(DT[dtype])
        qkv.copy_(x)
        for b in (*bufs, ws):
            b.fill_(85 if b.dtype == torch.uint8 else math.nan)
        graph.replay()
        torch.cuda.synchronize()
        got = [b.clone() for b in bufs]
        kept = a.k.clone()
        other = a.buffers(sum(news))
        a.step(qkv.clone(), news, pasts, *other, a.workspace(news, pasts))
        for b, o in zip(got, other):
            assert torch.equal(b, o), f"replay {turn} differs from the eager call"
        assert torch.equal(torch.nan_to_num(kept.float(), 7), torch.nan_to_num(a.k.float(), 7))


def test_calls_at_once_on_streams():
    """Layers on streams of their own, none the current one, give what they give one after another."""
    layers = [Layer((500, 900), 128, 16, "bf16", seed=i) for i in range(3)]
    news, pasts = (500, 900), (0, 0)
    want, run = [], []
    for a in layers:
        qkv = a.inputs(news, pasts).cuda()
        bufs = a.buffers(sum(news))
        a.step(qkv, news, pasts, *bufs, a.workspace(news, pasts))
        want.append(bufs)
        run.append((a, qkv, a.buffers(sum(news)), a.workspace(news, pasts), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(3):
        for a, qkv, bufs, ws, stream in run:
            a.step(qkv, news, pasts, *bufs, ws, stream=stream)
    torch.cuda.synchronize()
    for (a, _, bufs, _, _), w in zip(run, want):
        for x, y in zip(bufs, w):
            assert torch.equal(x, y)
