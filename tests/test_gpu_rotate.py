"""Norms and rotation (infllm_rotate) and the append to pages (infllm_paged_append) against 64 bits (GPU)."""
import math

import pytest
import torch

from paper_2402_04617_amd import infllm as F
from tests.paged_util import DT, Cache, params, rotate64
from tests.shared_util import check

pytestmark = pytest.mark.gpu


def fused(T, Hq, Hkv, D, dtype, seed=0, spare=2):
    """One projection's output [token][q, k, v heads], NaN behind the last token."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((T + spare, Hq + 2 * Hkv, D), generator=g).to(DT[dtype])
    x[T:] = math.nan
    return x


def weights(D, dtype, seed=5):
    g = torch.Generator().manual_seed(seed)
    return [(1 + 0.3 * torch.randn(D, generator=g)).to(DT[dtype]) for _ in range(2)]


def theta_of(rot, base=10000.0):
    return [base ** (-2.0 * i / rot) for i in range(rot // 2)]


@pytest.mark.parametrize("dtype,Hq,Hkv,D,rot,interleaved,norm,T", [
    ("bf16", 32, 8, 128, 128, False, True, 1),
    ("bf16", 32, 8, 128, 128, True, False, 5),
    ("bf16", 5, 1, 128, 64, False, True, 33),
    ("bf16", 4, 2, 64, 64, False, False, 300),
    ("bf16", 4, 2, 64, 20, False, True, 7),      # partners that lie across pieces
    ("bf16", 3, 3, 64, 20, True, True, 7),
    ("bf16", 2, 1, 128, 0, False, True, 9),      # norms alone
    ("bf16", 7, 1, 128, 2, False, False, 3),
    ("bf16", 8, 2, 128, 128, False, True, 2500),  # a wave per token
    ("f32", 8, 2, 64, 64, False, True, 40),
    ("f32", 8, 2, 128, 128, True, True, 11),
    ("f32", 3, 1, 128, 12, False, False, 130),
    ("f32", 1, 1, 64, 64, False, False, 1),
])
def test_rotate(dtype, Hq, Hkv, D, rot, interleaved, norm, T):
    x = fused(T, Hq, Hkv, D, dtype)
    wq, wk = weights(D, dtype)
    theta = theta_of(rot) if rot else []
    g = torch.Generator().manual_seed(1)
    at = torch.randint(0, 1 << 20, (T,), generator=g)
    at[0] = (1 << 31) + 12345
    if T > 2:
        at[1], at[2] = 0, -77
    magnitude = 1.25
    r = F.rotary(theta, interleaved, magnitude, norm, wq.cuda(), wk.cuda(), 1e-5)
    xd = x.cuda()
    q_out = torch.full((Hq, T + 1, D), 7.0, dtype=DT[dtype], device="cuda")
    k_out = torch.full((T + 1, Hkv, D + 8), 7.0, dtype=DT[dtype], device="cuda")
    st = ((Hq + 2 * Hkv) * D, D)
    p = params(Hq, Hkv, D, dtype)
    F.infllm_rotate(p, r, T, at.cuda(), xd, st, q_out, (D, (T + 1) * D), xd[:, Hq:], st, k_out, (Hkv * (D + 8), D + 8))
    for name, rows, w, got in (("q", x[:T, :Hq], wq, q_out.transpose(0, 1)), ("k", x[:T, Hq:Hq + Hkv], wk, k_out[..., :D])):
        want, tol = rotate64(rows.double(), at, theta, interleaved, magnitude, norm, w.double(), 1e-5, dtype)
        check(name, got[:T], want, tol)
        assert torch.all(got[T:] == 7), "a row behind the last token was written"
    assert torch.all(k_out[..., D:] == 7), "the gap between rows was written"
    # in place, and one of the two alone, give the same bits
    F.infllm_rotate(p, r, T, at.cuda(), None, None, None, None, xd[:, Hq:], st, xd[:, Hq:], st)
    assert torch.equal(xd[:T, Hq:Hq + Hkv], k_out[:T, :, :D])
    assert torch.equal(xd[:T, :Hq].cpu(), x[:T, :Hq]) and torch.equal(xd[:T, Hq + Hkv:].cpu(), x[:T, Hq + Hkv:])
    F.infllm_rotate(p, r, T, at.cuda(), xd, st, xd, st, None, None, None, None)
    assert torch.equal(xd[:T, :Hq], q_out.transpose(0, 1)[:T])


def test_positions_from_a_first_one():
    p = params(4, 2, 128, "bf16")
    x = fused(6, 4, 2, 128, "bf16").cuda()
    r = F.rotary(theta_of(128))
    got = [torch.empty((6, 4, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    at = torch.arange(6, device="cuda") + 1000001
    for o, kw in zip(got, (dict(positions=at), dict(positions=None, first_position=1000001))):
        F.infllm_rotate(p, r, 6, q=x, q_strides=(8 * 128, 128), q_out=o, q_out_strides=(512, 128), k=None, k_strides=None,
                        k_out=None, k_out_strides=None, **kw)
    assert torch.equal(*got)


@pytest.mark.parametrize("interleaved,rot", [(False, 128), (True, 128), (False, 64), (True, 64), (False, 20)])
def test_values_that_are_not_finite_stay_in_their_rows(interleaved, rot):
    """An infinity or NaN reaches its own pair (with norms its own row), and no other row."""
    T, H, D = 3, 4, 128
    g = torch.Generator().manual_seed(3)
    x = torch.randn((T, H, D), generator=g)
    clean = x.clone()
    x[1, 2, 5], x[1, 3, D - 1] = math.inf, math.nan
    p = params(H, 1, D, "f32")
    r = F.rotary(theta_of(rot), interleaved)
    at = torch.arange(T, device="cuda") * 17 + 1
    out = []
    for y in (x, clean):
        o = torch.empty((T, H, D), device="cuda")
        F.infllm_rotate(p, r, T, at, y.cuda(), (H * D, D), o, (H * D, D), None, None, None, None)
        out.append(o.cpu())
    odd = ~torch.isfinite(out[0])
    mate = lambda d: d if d >= rot else (d ^ 1 if interleaved else (d + rot // 2) % rot)  # noqa: E731
    want = torch.zeros_like(odd)
    for h, d in ((2, 5), (3, D - 1)):
        want[1, h, d] = want[1, h, mate(d)] = True
    assert torch.equal(odd, want)
    assert torch.equal(out[0][~odd], out[1][~odd])


def test_zero_rows_and_large_ones():
    """A row of zeros stays zero with eps 0 refused by nothing: 0 / sqrt(eps); rows near the type's ends keep their shape."""
    H, D = 4, 64
    x = torch.zeros((1, H, D), dtype=torch.bfloat16)
    x[0, 1], x[0, 2], x[0, 3] = 1e18, -1e-18, 2.0
    p = params(H, 1, D, "bf16")
    r = F.rotary([], norm=True, eps=1e-6)
    o = torch.empty((1, H, D), dtype=torch.bfloat16, device="cuda")
    F.infllm_rotate(p, r, 1, None, x.cuda(), (H * D, D), o, (H * D, D), None, None, None, None)
    want, tol = rotate64(x.double(), torch.zeros(1, dtype=torch.int64), [], False, 1.0, True, None, float(torch.tensor(1e-6)), "bf16")
    check("normed", o, want, tol)


MIXED = ((1, 0, 5, 1, 64, 33, 0, 17), (100, 3, 0, 63, 1, 4095, 0, 15))


@pytest.mark.parametrize("dtype,Hq,Hkv,D,page,order,rot,interleaved,norm", [
    ("bf16", 8, 2, 128, 16, "heads", 128, False, True),
    ("bf16", 8, 2, 128, 64, "tokens", 64, True, False),
    ("bf16", 5, 1, 64, 24, "apart", 64, False, True),
    ("bf16", 3, 3, 64, 1, "tokens", 20, False, False),
    ("bf16", 16, 2, 128, 50, "apart", 0, False, False),
    ("f32", 4, 4, 64, 7, "heads", 64, False, True),
    ("f32", 4, 1, 128, 256, "tokens", 128, True, False),
])
def test_append(dtype, Hq, Hkv, D, page, order, rot, interleaved, norm):
    news, pasts = MIXED
    total = sum(news)
    c = Cache([a + b for a, b in zip(news, pasts)], Hkv, D, page, dtype, order, fill=3.0)
    before_k, before_v = c.slots(c.k).clone(), c.slots(c.v).clone()
    x = fused(total, Hq, Hkv, D, dtype, seed=2)
    wq, wk = weights(D, dtype)
    theta = theta_of(rot) if rot else []
    r = F.rotary(theta, interleaved, 0.8, norm, wq.cuda(), wk.cuda(), 1e-5)
    p = params(Hq, Hkv, D, dtype)
    xd = x.cuda()
    st = ((Hq + 2 * Hkv) * D, D)
    q_out = torch.full((total + 1, Hq, D), 7.0, dtype=DT[dtype], device="cuda")
    F.infllm_paged_append(p, r, c.struct, news, pasts, c.table, xd, st, q_out, (Hq * D, D), xd[:, Hq:], xd[:, Hq + Hkv:], st)
    at = torch.tensor([b + j for a, b in zip(news, pasts) for j in range(a)])
    args = (at, theta, interleaved, 0.8, norm)
    wide = torch.float32 if dtype == "f32" else torch.bfloat16
    eps = float(torch.tensor(1e-5, dtype=torch.float32))
    q, tq = rotate64(x[:total, :Hq].double(), *args, wq.double(), eps, dtype)
    k, tk = rotate64(x[:total, Hq:Hq + Hkv].double(), *args, wk.double(), eps, dtype)
    check("q", q_out[:total], q, tq)
    assert torch.all(q_out[total:] == 7)
    want_k, want_v, tol = before_k.double(), before_v.clone(), torch.zeros(before_k.shape, dtype=torch.float64)
    row = 0
    for i, (new, past) in enumerate(zip(news, pasts)):
        for j in range(new):
            x_, slot = int(c.host_table[i, (past + j) // page]), (past + j) % page
            want_k[x_, slot], tol[x_, slot], want_v[x_, slot] = k[row], tk[row], x[row, Hq + Hkv:].to(wide)
            row += 1
    check("k", c.slots(c.k), want_k, tol)
    assert torch.equal(c.slots(c.v), want_v), "values, or slots that no new token takes"
    if order == "apart":
        assert torch.all(c.kv[..., D:] == 3), "the gap between rows was written"
    # the keys alone, without rotation: the projection's own bits
    plain = Cache([a + b for a, b in zip(news, pasts)], Hkv, D, page, dtype, order, fill=3.0)
    F.infllm_paged_append(p, None, plain.struct, news, pasts, plain.table, None, None, None, None, xd[:, Hq:], xd[:, Hq + Hkv:], st)
    row = 0
    got = plain.slots(plain.k)
    for i, (new, past) in enumerate(zip(news, pasts)):
        for j in range(new):
            assert torch.equal(got[int(plain.host_table[i, (past + j) // page]), (past + j) % page], x[row, Hq:Hq + Hkv])
            row += 1


def test_append_does_not_follow_bad_pages():
    Hq, Hkv, D, page = 4, 2, 128, 16
    news, pasts = (40, 3), (8, 14)
    c = Cache([48, 17], Hkv, D, page, "bf16", fill=3.0)
    x = fused(43, Hq, Hkv, D, "bf16").cuda()
    st = ((Hq + 2 * Hkv) * D, D)
    p = params(Hq, Hkv, D, "bf16")
    F.infllm_paged_append(p, None, c.struct, news, pasts, c.table, None, None, None, None, x[:, Hq:], x[:, Hq + Hkv:], st)
    whole = c.k.clone()
    for bad in (-1, c.k.shape[0], -(1 << 31), (1 << 31) - 1):
        d = Cache([48, 17], Hkv, D, page, "bf16", fill=3.0)
        lost = d.k[d.host_table[0, 1].item()].clone()
        d.table[0, 1] = bad
        q_out = torch.zeros((43, Hq, D), dtype=torch.bfloat16, device="cuda")
        F.infllm_paged_append(p, None, d.struct, news, pasts, d.table, x, st, q_out, (Hq * D, D), x[:, Hq:], x[:, Hq + Hkv:], st)
        want = whole.clone()
        want[d.host_table[0, 1].item()] = lost
        assert torch.equal(d.k, want)
        assert torch.equal(q_out, x[:43, :Hq])


def test_append_of_many_sequences():
    """More sequences than a launch takes."""
    Hq, Hkv, D, page = 2, 1, 64, 16
    news = [(i * 7) % 4 for i in range(600)]
    pasts = [(i * 13) % 50 for i in range(600)]
    total = sum(news)
    c = Cache([a + b for a, b in zip(news, pasts)], Hkv, D, page, "bf16", fill=3.0)
    x = fused(total, Hq, Hkv, D, "bf16")
    p = params(Hq, Hkv, D, "bf16")
    theta = theta_of(D)
    r = F.rotary(theta)
    st = ((Hq + 2 * Hkv) * D, D)
    xd = x.cuda()
    q_out = torch.empty((total, Hq, D), dtype=torch.bfloat16, device="cuda")
    F.infllm_paged_append(p, r, c.struct, news, pasts, c.table, xd, st, q_out, (Hq * D, D), xd[:, Hq:], xd[:, Hq + Hkv:], st)
    at = torch.tensor([b + j for a, b in zip(news, pasts) for j in range(a)])
    q, tq = rotate64(x[:total, :Hq].double(), at, theta, False, 1.0, False, None, 0.0, "bf16")
    k, tk = rotate64(x[:total, Hq:Hq + Hkv].double(), at, theta, False, 1.0, False, None, 0.0, "bf16")
    check("q", q_out, q, tq)
    seq = torch.tensor([i for i, a in enumerate(news) for _ in range(a)])
    got = c.slots(c.k)[c.host_table[seq, at // page].long(), at % page]
    check("k", got, k, tk)
    assert torch.equal(c.slots(c.v)[c.host_table[seq, at // page].long(), at % page], x[:total, Hq + Hkv:])


def test_append_past_32_bit_offsets():
    """A page whose rows lie past 4 GiB and past 2^31 elements."""
    Hq, Hkv, D, page = 1, 1, 128, 64
    n = (5 << 30) // (page * D * 2)
    k = torch.empty((n, Hkv, page, D), dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    st = F.pages(k, v, page)
    table = torch.tensor([[0, n - 1]], dtype=torch.int32, device="cuda")
    k[n - 1].zero_()
    v[n - 1].zero_()
    k[0].zero_()
    x = fused(3, Hq, Hkv, D, "bf16").cuda()
    F.infllm_paged_append(params(Hq, Hkv, D, "bf16"), None, st, (3,), (page + 5,), table, None, None, None, None, x[:, 1:], x[:, 2:], (3 * D, D))
    assert torch.equal(k[n - 1, 0, 5:8], x[:3, 1]) and torch.equal(v[n - 1, 0, 5:8], x[:3, 2])
    assert torch.all(k[n - 1, 0, :5] == 0) and torch.all(k[n - 1, 0, 8:] == 0) and torch.all(k[0] == 0)
