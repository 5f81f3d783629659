"""Continuations of a shared document: scoring and attention against 64 bits, and the whole way of a
batch from packed prompts over forks to its steps (GPU)."""
import math

import numpy as np
import pytest
import torch

from oracle import infllm_oracle as O
from paper_2402_04617_amd import infllm as F
from tests.gpu_util import Layer, check_selection, dev, host, log, oparams
from tests.shared_util import U32, attend64, check

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def store(batch, capacity, **tensors):
    m = F.Memory(batch=batch, capacity=capacity)
    for name, t in tensors.items():
        setattr(m, name, t.data_ptr())
    return m


class Case:
    """Document and own stores with NaN wherever the call must not look, and the call's arguments."""

    def __init__(self, p, B, n_q, length, own_lens, seed=0, q_pad=0, given=True, idx="units", scale=1.0):
        g = torch.Generator().manual_seed(seed)
        self.p, self.B, self.n_q, self.length, self.own_lens = p, B, n_q, length, own_lens
        Hq, Hkv, D = p.n_q_heads, p.n_kv_heads, p.head_dim
        dt = DT["bf16" if p.dtype == F.INFLLM_BF16 else "f32"]
        self.dt = dt

        def normal(*shape, s=1.0):
            return (torch.randn(shape, generator=g) * s).to(dt).cuda()

        self.part = O.partition(length, oparams(p))
        cap, room = length + 5, max(own_lens) + n_q + 3
        self.k, self.v = normal(Hkv, cap, D), normal(Hkv, cap, D)
        self.k[:, length:], self.v[:, length:] = math.nan, math.nan
        self.ok, self.ov = normal(B, Hkv, room, D), normal(B, Hkv, room, D)
        self.xk, self.xv = normal(B, Hkv, n_q, D), normal(B, Hkv, n_q, D)
        for b, n in enumerate(own_lens):
            for t, x in ((self.ok, self.xk), (self.ov, self.xv)):
                t[b, :, n:] = math.nan
                if not given:
                    t[b, :, n:n + n_q] = x[b]
        self.given = given
        self.q_rows = n_q + q_pad
        self.q = normal(B, Hq, self.q_rows, D, s=scale)
        self.q[:, :, n_q:] = math.nan
        nu, k_m = self.part.n_units, p.topk
        self.idx = torch.full((B, Hkv, max(k_m, 1)), -1, dtype=torch.int32)
        for b in range(B):
            for h in range(Hkv):
                c = torch.randperm(max(nu, 1), generator=g)[:min(k_m, nu)].sort().values
                if idx == "some":  # padding, and entries out of range, between valid ones
                    c = c[: len(c) // 2 + (b + h) % 2]
                    row = torch.tensor([-1, nu, 2 ** 31 - 1, -2 ** 31], dtype=torch.int64)[: k_m - len(c)]
                    self.idx[b, h, : len(row)] = row
                    self.idx[b, h, len(row):len(row) + len(c)] = c
                elif idx == "units":
                    self.idx[b, h, : len(c)] = c
        # units that nobody looks up hold NaN
        for h in range(Hkv):
            used = set(int(u) for u in self.idx[:, h].flatten() if 0 <= u < nu)
            for u in range(nu):
                if u not in used:
                    a = p.n_init + u * p.block_size
                    self.k[h, a:a + p.block_size], self.v[h, a:a + p.block_size] = math.nan, math.nan
        self.idx = self.idx.cuda()
        self.out = torch.full((B, Hq, self.q_rows, D), 7.0, dtype=dt, device="cuda")
        self.lse = torch.full((B, Hq, n_q), 7.0, dtype=torch.float32, device="cuda")
        self.doc, self.own = store(1, cap, k=self.k, v=self.v), store(B, room, k=self.ok, v=self.ov)
        self.ws = torch.empty(max(16, F.infllm_prefix_workspace_bytes(p, B, n_q, length, room)), dtype=torch.uint8, device="cuda")

    def run(self, stream=None):
        D = self.p.head_dim
        xk, xv = (self.xk, self.xv) if self.given else (None, None)
        F.infllm_prefix_attend(self.p, self.doc, self.length, self.own, self.own_lens, self.q, self.q_rows * D, xk, xv, self.n_q * D,
                               self.n_q, self.idx if self.p.topk else None, self.p.topk, self.out, self.q_rows * D, self.lse, self.ws,
                               stream=stream)

    def want(self, b, h):
        """Keys, values and visibility of continuation b, query head h."""
        p, g = self.p, h // (self.p.n_q_heads // self.p.n_kv_heads)
        at = list(range(self.part.n_init))
        for u in self.idx[b, g].tolist()[: min(p.topk, self.part.n_units)]:
            if 0 <= u < self.part.n_units:
                at += range(p.n_init + u * p.block_size, p.n_init + (u + 1) * p.block_size)
        at += range(self.part.local_begin, self.length)
        n = self.own_lens[b]
        k, v = (torch.cat([d[g][at], o[b, g, :n], x[b, g]]).double().cpu()
                for d, o, x in ((self.k, self.ok, self.xk), (self.v, self.ov, self.xv)))
        seen = torch.ones((self.n_q, len(k)), dtype=torch.bool).tril(len(k) - self.n_q)
        return k, v, seen

    def verify(self):
        dtype = "bf16" if self.dt == torch.bfloat16 else "f32"
        for b in range(self.B):
            for h in range(self.p.n_q_heads):
                k, v, seen = self.want(b, h)
                w = attend64(self.q[b, h, :self.n_q].double().cpu(), k, v, float(self.p.sm_scale), seen, dtype)
                check(f"out of continuation {b}, head {h}", self.out[b, h, :self.n_q], w[0], w[2])
                check(f"lse of continuation {b}, head {h}", self.lse[b, h], w[1], w[3])
        assert torch.all(self.out[:, :, self.n_q:] == 7), "rows behind the queries were written"
        for b, n in enumerate(self.own_lens):
            for t, x in ((self.ok, self.xk), (self.ov, self.xv)):
                assert torch.equal(t[b, :, n:n + self.n_q], x[b])
                assert torch.isnan(t[b, :, n + self.n_q:].float()).all()


def params(Hq, Hkv, D, dtype, local=256, init=16, block=64, topk=3):
    return F.params(Hq, Hkv, D, init, local, block, 2, topk, dtype, sm_scale=D ** -0.5)


@pytest.mark.parametrize("dtype,Hq,Hkv,D,kw,B,n_q,length,own,more", [
    ("bf16", 8, 2, 128, {}, 4, 1, 2000, (0, 1, 63, 200), {}),
    ("bf16", 8, 2, 128, {}, 4, 1, 2000, (0, 1, 63, 200), dict(idx="some", q_pad=2)),
    ("bf16", 8, 2, 64, dict(block=37, init=5, local=100), 3, 5, 1111, (64, 0, 130), dict(idx="some")),
    ("bf16", 6, 2, 128, dict(topk=0, local=5000), 9, 1, 3001, tuple(range(9)), {}),
    ("bf16", 5, 1, 64, dict(topk=0, local=5000), 64, 1, 777, tuple(3 * i for i in range(64)), {}),
    ("bf16", 32, 8, 128, dict(local=1024, init=128, block=128, topk=8), 16, 4, 8000, tuple(40 * i for i in range(16)), {}),
    ("bf16", 4, 4, 128, {}, 1, 1, 1, (0,), {}),
    ("bf16", 4, 2, 128, {}, 2, 3, 0, (0, 70), {}),                       # no document at all
    ("bf16", 4, 2, 64, {}, 2, 2, 0, (0, 0), {}),                         # and nothing of their own: X alone
    ("bf16", 4, 2, 128, {}, 3, 8, 900, (0, 0, 0), {}),                   # the most tokens that the merge meets
    ("bf16", 4, 2, 128, {}, 3, 9, 900, (0, 5, 64), dict(q_pad=1)),       # one more
    ("bf16", 4, 2, 128, dict(topk=0), 2, 1, 2000, (5, 6), {}),            # I and L alone
    ("bf16", 4, 2, 128, {}, 3, 200, 1500, (0, 300, 17), dict(q_pad=1)),   # chunks
    ("bf16", 4, 2, 128, {}, 2, 2, 2000, (10, 20), dict(idx="none", given=False)),
    ("f32", 4, 2, 64, {}, 4, 1, 2000, (0, 1, 63, 200), {}),
    ("f32", 8, 2, 128, dict(block=37, init=5, local=100), 3, 5, 1111, (64, 0, 130), dict(idx="some", q_pad=1)),
    ("f32", 3, 1, 64, dict(topk=0, local=5000), 20, 2, 901, tuple(range(20)), dict(given=False)),
    ("f32", 4, 2, 64, {}, 2, 90, 0, (0, 70), {}),
    ("f32", 4, 2, 128, {}, 2, 8, 500, (0, 0), {}),
    ("f32", 2, 1, 64, {}, 1, 1, 0, (0,), {}),
])
def test_prefix_parity(dtype, Hq, Hkv, D, kw, B, n_q, length, own, more):
    log(f"[prefix] {dtype} {Hq}/{Hkv} D={D} {kw} B={B} n_q={n_q} length={length} {more}")
    c = Case(params(Hq, Hkv, D, dtype, **kw), B, n_q, length, own, **more)
    c.run()
    c.verify()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prefix_steep_scores(dtype):
    log(f"[prefix] {dtype} steep scores")
    p = F.params(4, 2, 64, 16, 256, 64, 2, 3, dtype, sm_scale=1.0)
    c = Case(p, 3, 2, 1500, (0, 100, 5), scale=6.0)
    c.run()
    c.verify()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prefix_not_finite_stays(dtype):
    """An infinite value of a current token reaches the queries from it on; a NaN key of one continuation
    reaches that continuation; a NaN query its own row."""
    p = params(4, 2, 128, dtype)
    c = Case(p, 3, 4, 1500, (7, 100, 60), given=True)
    c.run()
    clean, clean_lse = c.out.clone(), c.lse.clone()
    c.verify()
    log(f"[prefix] {dtype} not finite")
    c.xv[0, 1, 2, 9] = math.inf
    c.ok[1, 0, 3, 0] = math.nan
    c.q[2, 3, 1, 4] = math.nan
    c.run()
    o, odd = c.out, torch.zeros((3, 4, 4, 128), dtype=torch.bool, device="cuda")
    odd[0, 2:, 2:, 9] = True
    odd[1, :2] = True
    odd[2, 3, 1] = True
    assert torch.equal(~torch.isfinite(o.float()), odd)
    assert torch.all(o[0, 2:, 2:, 9] == math.inf)
    assert torch.isnan(o[1, :2].float()).all() and torch.isnan(o[2, 3, 1].float()).all()
    lost = torch.isnan(c.lse)
    assert lost[1, :2].all() and lost[2, 3, 1] and int(lost.sum()) == 2 * 4 + 1
    # everything else as before, within the roundings of either
    c.xv[0, 1, 2, 9] = 0.25
    c.ok[1, 0, 3, 0] = 0.25
    c.q[2, 3, 1, 4] = 0.25
    again = c.out.clone()
    again_lse = c.lse.clone()
    c.run()
    again[odd] = c.out[odd]
    again_lse[lost] = c.lse[lost]
    c.out, c.lse = again, again_lse
    c.verify()
    del clean, clean_lse


@pytest.mark.parametrize("dtype,Hq,Hkv,D,B,n_q,units,max_units", [
    ("bf16", 8, 2, 128, 1, 1, 1, 1), ("bf16", 32, 8, 128, 16, 1, 217, 224), ("bf16", 6, 2, 64, 9, 3, 64, 70),
    ("bf16", 4, 1, 128, 33, 70, 1000, 1000), ("f32", 4, 2, 64, 7, 1, 65, 80), ("f32", 8, 8, 128, 3, 40, 2001, 2001),
])
def test_prefix_score_parity(dtype, Hq, Hkv, D, B, n_q, units, max_units):
    log(f"[prefix score] {dtype} {Hq}/{Hkv} D={D} B={B} n_q={n_q} units={units}")
    g = torch.Generator().manual_seed(units)
    q = torch.randn((B, Hq, n_q + 1, D), generator=g).to(DT[dtype]).cuda()
    ksum = torch.randn((1, Hkv, D // 4, max_units, 4), generator=g).cuda()
    q[:, :, n_q:] = math.nan
    ksum[:, :, :, units:] = math.nan
    p = params(Hq, Hkv, D, dtype)
    scores = torch.full((B * Hkv * units + 9,), 7.0, device="cuda")
    m = F.Memory(batch=1, capacity=1, max_units=max_units)
    m.unit_ksum = ksum.data_ptr()
    ws = torch.empty(F.infllm_prefix_workspace_bytes(p, B, n_q, 0, 0), dtype=torch.uint8, device="cuda")
    F.infllm_prefix_score(p, m, B, q, (n_q + 1) * D, n_q, units, scores, ws)
    got = scores[:B * Hkv * units].view(B, Hkv, units).double().cpu()
    G = Hq // Hkv
    qs = q[:, :, :n_q].double().cpu().view(B, Hkv, G * n_q, D)
    ks = ksum[0, :, :, :units].double().cpu().permute(0, 1, 3, 2).reshape(Hkv, D, units)
    want = qs.sum(2).transpose(0, 1) @ ks
    # sums of G n_q queries, then D products, each addition one rounding of at most the absolute sum
    tol = (G * n_q + D + 4) * U32 * (qs.abs().sum(2).transpose(0, 1) @ ks.abs())
    check("scores", got.transpose(0, 1), want, tol)
    assert torch.all(scores[B * Hkv * units:] == 7)


def test_prefix_repeats_streams_and_graphs():
    """Bitwise the same on another stream and in a replayed graph with other inputs; two graphs that share a
    workspace, replayed one after the other, do not disturb each other."""
    p = params(8, 2, 128, "bf16")
    cases = [Case(p, 4, 1, 2000, (3, 70, 128, 0), seed=s) for s in (1, 2)]
    want = []
    for c in cases:
        c.run()
        want.append((c.out.clone(), c.lse.clone()))
    log("[prefix] another stream")
    c = cases[0]
    side = torch.cuda.Stream()
    c.out.zero_()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.run()
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(c.out, want[0][0]) and torch.equal(c.lse, want[0][1])
    log("[prefix] graphs")
    cases[1].ws = cases[0].ws
    graphs = []
    for c in cases:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            c.run()
    keep = [(c.q.clone(), c.xk.clone(), c.xv.clone()) for c in cases]
    for turn in range(3):
        for c, graph, w in zip(cases, graphs, want):
            c.out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(c.out, w[0]) and torch.equal(c.lse, w[1]), turn
    for x, y in zip((cases[0].q, cases[0].xk, cases[0].xv), keep[1]):
        x.copy_(y)
    graphs[0].replay()
    cases[0].verify()


def test_batch_from_prompts_to_steps():
    """A document is encoded chunk by chunk, forked to two slots, and continued there by whole steps; the same
    continuations as branches of the shared document give the same scores, lookups and outputs.  Before that
    its question goes through the packed prompts, which agree with a step that has nothing before it."""
    Hq, Hkv, D = 8, 2, 128
    p = F.params(Hq, Hkv, D, 16, 256, 64, 2, 3, "bf16", sm_scale=D ** -0.5)
    rng = np.random.default_rng(5)
    S, chunk, n_q = 2000, 250, 3
    q, k, v = ((rng.standard_normal((1, h, S, D))).astype(np.float32) for h in (Hq, Hkv, Hkv))
    qd, kd, vd = (dev(x, "bf16") for x in (q, k, v))

    log("[batch] packed prompts and steps")
    lens = (130, 1, 222)
    T = sum(lens)
    po, pl = torch.empty((Hq, T, D), dtype=torch.bfloat16, device="cuda"), torch.empty((Hq, T), device="cuda")
    size = F.infllm_prompt_workspace_bytes(p, lens)
    F.infllm_prompt_attend(p, lens, qd, (D, S * D), kd, vd, (D, S * D), po, (D, T * D), pl,
                           torch.empty(max(16, size), dtype=torch.uint8, device="cuda"))
    at = 0
    for n in lens:
        L = Layer(p, 1, n, n)
        sl = tuple(x[:, :, at:at + n].contiguous() for x in (qd, kd, vd))
        L.step(*sl, 0, n)
        # both round their weights and outputs once: twice a half step of bf16 each, of outputs below 5
        assert (po[:, at:at + n].float() - L.out[0].float()).abs().max() <= 4 * 5 * 2.0 ** -8
        assert (pl[:, at:at + n] - L.lse[0]).abs().max() <= 1e-4
        at += n

    log("[batch] encode, fork, step")
    doc = Layer(p, 1, S, chunk)
    for past in range(0, S, chunk):
        doc.step(qd, kd, vd, past, chunk)
    nu = O.partition(S, oparams(p)).n_units
    F.infllm_build_units(p, doc.mem.struct, doc.units_built, nu - doc.units_built, S)
    slots = Layer(p, 2, S + 40, chunk, ring=doc.ring)
    F.infllm_copy_sequences(p, slots.mem.struct, doc.mem.struct, [1, 0], [0, 0], [S, S], [nu, nu])
    own_cap = 10
    own = tuple(torch.full((2, Hkv, own_cap, D), math.nan, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    m_own = store(2, own_cap, k=own[0], v=own[1])
    assert O.partition(S + 2 * n_q, oparams(p)).n_units == nu  # (nothing is evicted while the branches grow)
    ws = torch.empty(F.infllm_prefix_workspace_bytes(p, 2, n_q, S, own_cap), dtype=torch.uint8, device="cuda")
    for turn in range(2):
        x = [torch.randn((2, h, n_q, D), generator=torch.Generator().manual_seed(turn)).to(torch.bfloat16).cuda() for h in (Hq, Hkv, Hkv)]
        past = S + turn * n_q
        F.infllm_step(p, slots.mem.struct, x[0], n_q * D, x[1], x[2], n_q * D, n_q, past, nu, slots.scores, slots.idx, slots.out,
                      slots.chunk * D, slots.lse, slots.ws)
        scores = torch.empty((2, Hkv, nu), device="cuda")
        idx = torch.empty((2, Hkv, 3), dtype=torch.int32, device="cuda")
        out, lse = torch.empty((2, Hq, n_q, D), dtype=torch.bfloat16, device="cuda"), torch.empty((2, Hq, n_q), device="cuda")
        F.infllm_prefix_score(p, doc.mem.struct, 2, x[0], n_q * D, n_q, nu, scores, ws)
        F.infllm_select_topk(2 * Hkv, scores, nu, 3, idx)
        F.infllm_prefix_attend(p, doc.mem.struct, S, m_own, [turn * n_q] * 2, x[0], n_q * D, x[1], x[2], n_q * D, n_q, idx, 3, out,
                               n_q * D, lse, ws)
        step_scores = slots.scores[: 2 * Hkv * nu].view(2, Hkv, nu)
        assert (scores - step_scores).abs().max() <= 1e-5 * step_scores.abs().max()
        for r in range(2 * Hkv):
            check_selection(host(idx).reshape(-1, 3)[r], host(slots.idx).reshape(-1, 3)[r], host(step_scores).reshape(-1, nu)[r].astype(np.float64), 3)
        assert torch.equal(idx, slots.idx)
        assert (out.float() - slots.out[:, :, :n_q].float()).abs().max() <= 4 * 5 * 2.0 ** -8
        assert (lse.flatten() - slots.lse.flatten()[: lse.numel()]).abs().max() <= 1e-4
