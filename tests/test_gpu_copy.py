"""Copies of sequences between memories: bitwise, nothing else touched, and continued like their source (GPU)."""
import pytest
import torch

from paper_2402_04617_amd import infllm as F
from tests.gpu_util import Layer, log

pytestmark = pytest.mark.gpu

PARTS = ("k", "v", "k_rot", "repr_idx", "unit_ksum", "qprefix", "rpart")


def memory(p, batch, capacity, units, ring, seed):
    """A memory of random contents."""
    m = F.alloc_memory(p, batch, capacity, units, ring)
    g = torch.Generator().manual_seed(seed)
    for name in PARTS:
        t = getattr(m, name)
        if t is not None:
            t.copy_(torch.randint(-999, 999, t.shape, generator=g).to(t.dtype))
    return m


def copied(p, dst, src, pairs):
    """What the destination has to hold afterwards, part by part (plain slices, on the CPU)."""
    want = {n: getattr(dst, n).cpu().clone() for n in PARTS if getattr(dst, n) is not None}
    have = {n: getattr(src, n).cpu().clone() for n in want}
    for a, b, n, u in pairs:
        for name in ("k", "v", "k_rot"):
            if name in want:
                want[name][b, :, :n] = have[name][a, :, :n]
        want["unit_ksum"][b, :, :, :u] = have["unit_ksum"][a, :, :, :u]
        if not p.mean_repr:
            want["repr_idx"][b, :, :u] = have["repr_idx"][a, :, :u]
            rs, rd = src.struct.ring, dst.struct.ring
            for t in range(n - min(n, rs, rd), n):
                want["qprefix"][b, :, t % rd] = have["qprefix"][a, :, t % rs]
                want["rpart"][b, :, :, t % rd] = have["rpart"][a, :, :, t % rs]
    return want


@pytest.mark.parametrize("dtype,D,kw,src,dst,pairs", [
    # (batch, capacity, units, ring) of either side; (from, to, length, units)
    ("bf16", 128, {}, (1, 900, 10, 300), (4, 900, 10, 300), [(0, 0, 900, 8), (0, 1, 900, 8), (0, 2, 900, 8), (0, 3, 900, 8)]),
    ("bf16", 64, {}, (3, 700, 6, 200), (4, 1000, 9, 333), [(2, 0, 700, 5), (0, 3, 1, 0), (2, 1, 650, 4), (1, 2, 0, 0)]),
    ("bf16", 128, {}, (2, 700, 6, 333), (2, 650, 5, 200), [(0, 1, 201, 0), (1, 0, 650, 3)]),
    ("bf16", 128, dict(rope=True), (2, 300, 3, 250), (3, 310, 3, 250), [(1, 2, 300, 0), (1, 0, 299, 0)]),
    ("bf16", 64, dict(repr_mode="mean"), (1, 3000, 40, 1), (2, 3000, 44, 1), [(0, 1, 2999, 38)]),
    ("f32", 64, {}, (2, 400, 4, 150), (2, 400, 4, 150), [(1, 0, 400, 3), (0, 1, 17, 0)]),
    ("f32", 128, {}, (1, 129, 1, 500), (1, 257, 2, 130), [(0, 0, 129, 0)]),
])
def test_copy_bitwise(dtype, D, kw, src, dst, pairs):
    log(f"[copy] {dtype} D={D} {kw} {src} -> {dst}: {pairs}")
    p = F.params(6, 3, D, 7, 60, 70, 3, 4, dtype, rope_inv_freq=F.rope_frequencies(D) if kw.get("rope") else None,
                 repr_mode=kw.get("repr_mode", "tokens"))
    a, b = memory(p, *src, seed=1), memory(p, *dst, seed=2)
    want = copied(p, b, a, pairs)
    F.infllm_copy_sequences(p, b.struct, a.struct, *([x[i] for x in pairs] for i in (1, 0, 2, 3)))
    for name, w in want.items():
        assert torch.equal(getattr(b, name).cpu(), w), name


def test_copy_in_place():
    """A batch closed up in its own memory."""
    p = F.params(4, 2, 128, 16, 100, 32, 2, 4, "bf16")
    m = memory(p, 64, 300, 5, 220, seed=3)
    pairs = [(63 - i, i, 300 - 7 * i, 4 if i == 0 else 0) for i in range(32)]
    want = copied(p, m, m, pairs)
    log("[copy] 32 moves in place")
    F.infllm_copy_sequences(p, m.struct, m.struct, *([x[i] for x in pairs] for i in (1, 0, 2, 3)))
    for name, w in want.items():
        assert torch.equal(getattr(m, name).cpu(), w), name


def test_copy_continues_and_replays():
    """A fork taken in the middle of a stream goes on exactly like its source, also when the copy is a
    replayed graph's and the source has moved on in between."""
    p = F.params(4, 2, 64, 16, 128, 32, 2, 4, "bf16", sm_scale=0.125)
    S, chunk = 1200, 100
    g = torch.Generator().manual_seed(0)
    q, k, v = (torch.randn((1, h, S, 64), generator=g).to(torch.bfloat16).cuda() for h in (4, 2, 2))
    a = Layer(p, 1, S, chunk)
    forks = Layer(p, 3, S + 64, chunk, ring=a.ring + 33)
    cut = 600
    for past in range(0, cut, chunk):
        a.step(q, k, v, past, chunk)
    built = a.units_built
    graph = torch.cuda.CUDAGraph()
    log("[copy] fork, eager and captured")
    args = (p, forks.mem.struct, a.mem.struct, [2, 0], [0, 0], [cut, cut], [built, built])
    F.infllm_copy_sequences(*args)
    with torch.cuda.graph(graph):
        F.infllm_copy_sequences(*args)
    for turn in range(2):
        if turn:
            for t in (forks.mem.k, forks.mem.v, forks.mem.unit_ksum, forks.mem.qprefix, forks.mem.rpart):
                t.zero_()
            graph.replay()
        ref = Layer(p, 1, S, chunk)
        for past in range(0, cut, chunk):
            ref.step(q, k, v, past, chunk)
        forks.units_built = built
        for past in range(cut, cut + 300, chunk):
            ref.step(q, k, v, past, chunk)
            forks.step(*(x.expand(3, -1, -1, -1).contiguous() for x in (q, k, v)), past, chunk)
            n = ref.units_built
            for s in (0, 2):
                assert torch.equal(forks.out[s], ref.out[0]) and torch.equal(forks.lse[s], ref.lse[0]), (turn, past, s)
                assert torch.equal(forks.idx[s], ref.idx[0])
                assert torch.equal(forks.mem.unit_ksum[s, :, :, :n], ref.mem.unit_ksum[0, :, :, :n])
