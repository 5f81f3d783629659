"""Rows whose scores are all far below zero (about -150: their exponentials underflow unless they are taken against
the row's own maximum), with lookup entries to skip before the first key that the row sees (GPU)."""
import pytest
import torch

from oracle import infllm_oracle as O
from paper_2402_04617_amd import infllm as F
from tests.gpu_util import Layer, log, oparams
from tests.shared_util import attend64, check

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def low(g, dtype, sign, *shape):
    """Rows near +1 or -1: a query and a key score about -D, spread by D^0.5 / 14."""
    return (sign + 0.05 * torch.randn(shape, generator=g)).to(DT[dtype]).cuda()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,init,block", [(128, 0, 64), (64, 5, 37), (128, 16, 128)])
def test_prefix_low_scores_after_skipped_entries(dtype, D, init, block):
    log(f"[low] prefix {dtype} D={D} init={init} block={block}")
    Hq, Hkv, B, n_q, k_m, length, own = 4, 2, 32, 1, 40, 9000, 7
    p = F.params(Hq, Hkv, D, init, 100, block, 2, k_m, dtype, sm_scale=150.0 / D)
    part = O.partition(length, oparams(p))
    g = torch.Generator().manual_seed(D + block)
    dk, dv = low(g, dtype, 1, Hkv, length, D), torch.randn((Hkv, length, D), generator=g).to(DT[dtype]).cuda()
    ok, ov = low(g, dtype, 1, B, Hkv, own + n_q, D), torch.randn((B, Hkv, own + n_q, D), generator=g).to(DT[dtype]).cuda()
    q = low(g, dtype, -1, B, Hq, n_q, D)
    # runs of entries to skip and of valid ones, shifted from row to row, so that parts begin with either
    skip = [(j + 3 * r) % 7 < 4 for r in range(B * Hkv) for j in range(k_m)]
    idx = torch.randint(part.n_units, (B, Hkv, k_m), generator=g, dtype=torch.int32)
    idx = torch.where(torch.tensor(skip).view(B, Hkv, k_m), torch.tensor([-1, part.n_units]).int()[torch.arange(k_m) % 2], idx)
    idx[:, :, :4] = -1
    doc, mem = F.Memory(batch=1, capacity=length), F.Memory(batch=B, capacity=own + n_q)
    for m, a, c in ((doc, dk, dv), (mem, ok, ov)):
        m.k, m.v = a.data_ptr(), c.data_ptr()
    out, lse = torch.empty_like(q), torch.empty((B, Hq, n_q), device="cuda")
    ws = torch.empty(F.infllm_prefix_workspace_bytes(p, B, n_q, length, own + n_q), dtype=torch.uint8, device="cuda")
    F.infllm_prefix_attend(p, doc, length, mem, [own] * B, q, n_q * D, None, None, 0, n_q, idx.cuda(), k_m, out, n_q * D, lse, ws)
    for b in range(B):
        for h in range(Hq):
            kv = h // (Hq // Hkv)
            at = list(range(part.n_init))
            for u in idx[b, kv, :min(k_m, part.n_units)].tolist():
                if 0 <= u < part.n_units:
                    at += range(init + u * block, init + (u + 1) * block)
            at += range(part.local_begin, length)
            k, v = (torch.cat([d[kv, at], o[b, kv]]).double().cpu() for d, o in ((dk, ok), (dv, ov)))
            w = attend64(q[b, h].double().cpu(), k, v, float(p.sm_scale), torch.ones((n_q, len(k)), dtype=torch.bool), dtype)
            check(f"out of continuation {b}, head {h}", out[b, h], w[0], w[2])
            check(f"lse of continuation {b}, head {h}", lse[b, h], w[1], w[3])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_q,D,block,parts", [(3, 128, 64, False), (40, 64, 64, False), (70, 128, 37, True), (1, 128, 64, False),
                                               (1, 64, 64, True)])
def test_chunk_low_scores_after_skipped_entries(dtype, n_q, D, block, parts):
    log(f"[low] chunk {dtype} n_q={n_q} D={D} block={block} parts={parts}")
    Hq, Hkv, past, k_m = 4, 2, 1500, 9
    p = F.params(Hq, Hkv, D, 0, 100, block, 2, k_m, dtype, sm_scale=150.0 / D)
    part = O.partition(past, oparams(p))
    assert part.n_units >= k_m
    L = Layer(p, 1, past + n_q, chunk=n_q, ring=n_q + 101)
    g = torch.Generator().manual_seed(n_q + D)
    L.mem.k.copy_(low(g, dtype, 1, 1, Hkv, past + n_q, D))
    L.mem.v.copy_(torch.randn((1, Hkv, past + n_q, D), generator=g))
    q = low(g, dtype, -1, 1, Hq, n_q, D)
    nu = part.n_units
    idx = torch.tensor([[[-1, -1, -1, 2, 7, -1, nu, 5, -1], [nu, -1, 1, -1, -1, -1, -1, nu - 1, 3]]], dtype=torch.int32)
    out, lse = torch.empty_like(q), torch.empty((1, Hq, n_q), device="cuda")
    F.infllm_chunk_attend(p, L.mem.struct, q, n_q * D, n_q, past, idx.cuda(), k_m, out, n_q * D, lse, L.ws if parts else None)
    for h in range(Hq):
        kv = h // (Hq // Hkv)
        at = [u * block + j for u in idx[0, kv].tolist() if 0 <= u < nu for j in range(block)]
        at += range(part.local_begin, past + n_q)
        k, v = (t[0, kv, at].double().cpu() for t in (L.mem.k, L.mem.v))
        seen = torch.ones((n_q, len(at)), dtype=torch.bool).tril(len(at) - n_q)
        w = attend64(q[0, h].double().cpu(), k, v, float(p.sm_scale), seen, dtype)
        check(f"out of head {h}", out[0, h], w[0], w[2])
        check(f"lse of head {h}", lse[0, h], w[1], w[3])
