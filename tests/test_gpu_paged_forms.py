"""Capped and biased scores over paged caches at the ends of their ranges, against 64 bits (GPU).

The bounds here are those of the formulas in float32 and of what the header says of bf16, not of any kernel's way to
form them."""
import math

import pytest
import torch

from paper_2402_04617_amd import infllm as F
from tests.paged_util import seen_by
from tests.shared_util import HALF, STEP, U32, check
from tests.test_gpu_paged_attend import Run

pytestmark = pytest.mark.gpu

MOST_FOLDED = 64.0  # bf16: up to this cap a score is off by 2^-20 of the cap at most


def form64(q, k, v, scale, seen, distance, dtype, cap, slope):
    """q [n][D], k, v [m][D], seen, distance [n][m] (float64; positions of the queries less those of the keys): the
    attention, its log-sum-exp, and how far the kernels' results may be off.

    A score x: D products summed in float32 and the scale, D + 2 roundings of at most the sum of the absolute products
    (twice that for the base-2 domain's own factor).  The cap passes an error on at most as it is; its own is relative to
    the score: x / c, the function and the product, 16 roundings where |x| < c / 8, and where the tangent is 1 - 2 r,
    whose error is some 8 roundings of c and |z| >= c tanh(1 / 8), 64.  bf16 caps up to MOST_FOLDED add 16 roundings of the cap.
    The bias: its slope, the product and the sum, 8 roundings of the bias itself: of the key at the query's own
    position, whose bias is 0, none.  From there on as in paged_util.attend64.
    """
    x = (q @ k.T) * scale
    raw = (q.abs() @ k.abs().T) * scale
    e = U32 * (2 * q.shape[1] * raw + 8 * (raw + 1))
    z = x
    if cap:
        z = cap * torch.tanh(x / cap)
        e = e + U32 * torch.where(x.abs() < cap / 8, 16 * z.abs(), 64 * z.abs())
        if dtype == "bf16" and cap <= MOST_FOLDED:
            e = e + 16 * U32 * cap
    bias = -slope * distance
    z, e = z + bias, e + 8 * U32 * bias.abs()
    z = torch.where(seen, z, torch.full_like(z, -math.inf))
    lse = torch.logsumexp(z, dim=-1)
    p = torch.where(seen.any(-1)[:, None], torch.exp(z - lse[:, None]), torch.zeros_like(z))
    pe = p * e
    a, e_norm, e_sum = p @ v.abs(), pe.sum(-1), (k.shape[0] + 16) * U32
    out = p @ v
    tol = 2 * (pe @ v.abs()) + 2 * (e_norm + 2 * e_sum)[:, None] * a + STEP[dtype] * out.abs()
    if dtype == "bf16":
        tol = tol + STEP["bf16"] * a + HALF * a.amax(-1, keepdim=True)
    return out, lse, tol, 2 * e_norm + e_sum + 4 * U32 * lse.abs()


def verify(r, out, lse, cap=0.0, slopes=None, heads=None):
    at = 0
    out, lse = out.cpu(), lse.cpu()
    for i, (new, past) in enumerate(zip(r.news, r.pasts)):
        seen = seen_by(past, new, r.form.get("window", 0), r.form.get("n_init", 0))
        distance = (torch.arange(past, past + new)[:, None] - torch.arange(past + new)[None]).double()
        for h in heads or range(r.Hq):
            kv = h // (r.Hq // r.Hkv)
            w = form64(r.q[at:at + new, h].double(), r.c.keys[i][:, kv].double(), r.c.values[i][:, kv].double(), r.scale, seen, distance, r.dtype,
                       cap, 0.0 if slopes is None else float(slopes[h]))
            check(f"lse, sequence {i} ({past} + {new}), head {h}", lse[h, at:at + new], w[1], w[3])
            check(f"out, sequence {i} ({past} + {new}), head {h}", out[at:at + new, h], w[0], w[2])
        at += new


def with_form(dtype, D, news, pasts, page=16, Hq=4, Hkv=1, cap=0.0, slopes=None, q_scale=1.0, **window):
    r = Run(news, pasts, Hq, Hkv, D, page, dtype, form=dict(window, softcap=cap), q_scale=q_scale)
    if slopes is not None:
        r.score = F.score(slopes=torch.tensor(slopes, dtype=torch.float32, device="cuda"), softcap=cap, **window)
    return r


CAPS = [1.0, 30.0, 50.0, MOST_FOLDED, MOST_FOLDED * (1 + 2.0 ** -20), 100.0, 1e3, 1e4, 1e6, 1e8, 1.5e38, 3e38]
SOME = ((1, 40, 3, 1), (900, 300, 0, 6000))  # few rows and row tiles, whole and in parts


@pytest.mark.parametrize("dtype,D,page", [("bf16", 128, 16), ("bf16", 64, 50), ("f32", 64, 16), ("f32", 128, 24)])
@pytest.mark.parametrize("cap", CAPS)
def test_caps(cap, dtype, D, page):
    """Ordinary scores under every cap: a large one changes nothing."""
    r = with_form(dtype, D, *SOME, page=page, cap=cap)
    verify(r, *r.call(), cap=cap)


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 64)])
@pytest.mark.parametrize("cap", [20.0, MOST_FOLDED, 65.0, 300.0])
def test_scores_of_the_caps_order(cap, dtype, D):
    """Scores from far below the cap to far above it."""
    for q_scale in (cap / 10, cap):
        r = with_form(dtype, D, *SOME, cap=cap, q_scale=q_scale, window=500, n_init=20)
        verify(r, *r.call(), cap=cap)


@pytest.mark.parametrize("cap", [50.0, 1e4])
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 64)])
def test_values_that_are_not_finite_under_a_cap(dtype, D, cap):
    """A value that only later rows see leaves the earlier ones as they were; an infinite key's score is the cap."""
    for news, past in (((90, 1), 70), ((3, 1), 700), ((2, 1), 6000)):
        clean, odd = (with_form(dtype, D, news, (past, 40), cap=cap) for _ in range(2))
        t = past + 1
        odd.c.v[int(odd.c.host_table[0, t // 16]), 0, t % 16, 3] = math.inf
        out, lse = odd.call()
        want, want_lse = clean.call()
        assert torch.equal(lse, want_lse)
        assert torch.isfinite(out[0]).all() and (out[0].double() - want[0].double()).abs().max() <= (2e-2 if dtype == "bf16" else 1e-5)
        assert torch.all(out[1, :, 3] == math.inf) and torch.isfinite(out[1, :, :3]).all()
        assert torch.equal(out[sum(news) - 1], want[sum(news) - 1])
        # keys of one infinite dimension: all their scores are the cap, or its negative
        for s in range(past + news[0]):
            odd.c.k[int(odd.c.host_table[0, s // 16]), 0, s % 16, 5] = math.inf
        _, lse = odd.call()
        q = odd.q[:news[0], :, 5].double().T
        count = torch.arange(past + 1, past + news[0] + 1).double().log()
        top = torch.where(q > 0, torch.full_like(q, cap), torch.full_like(q, -cap)) + count
        check("lse", lse[:, :news[0]], top, (16 * cap + past + news[0] + 16) * U32 + 4 * U32 * top.abs())


STEEP = [[1e5, 1e3, 7.0, 0.3], [3.3e6, 0.0, -0.05, 1.0], [1e30, 1e-30, -1e-3, 12345.678], [3.4e38, 1e37, 2e35, 6e36]]


@pytest.mark.parametrize("dtype,D,page", [("bf16", 128, 16), ("bf16", 64, 50), ("f32", 64, 16)])
@pytest.mark.parametrize("slopes", STEEP, ids=str)
@pytest.mark.parametrize("kw", [dict(), dict(cap=5.0), dict(cap=1e3), dict(window=90, n_init=33), dict(window=2000, n_init=3)], ids=str)
def test_steep_biases(kw, slopes, dtype, D, page):
    """The key at the query's own position keeps its score, however steep the bias is."""
    for news, pasts in (((1, 200, 3, 1), (900, 30, 0, 6000)), ((130,), (1900,)), ((64, 65, 127), (64, 63, 1))):
        r = with_form(dtype, D, news, pasts, page=page, slopes=slopes, **kw)
        verify(r, *r.call(), cap=kw.get("cap", 0.0), slopes=slopes)


def test_steep_biases_of_one_head_each():
    """Row tiles of 128 queries: rows and their nearest keys in different tiles."""
    for slopes, pasts in (([1e5, 2e3], (3000, 65)), ([77.0, 1e4], (5001, 127))):
        r = with_form("bf16", 128, (300, 128), pasts, Hq=2, Hkv=2, slopes=slopes)
        verify(r, *r.call(), slopes=slopes)


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 64)])
@pytest.mark.parametrize("slopes", [[1e3, 50.0, 0.5, -0.02], [1e5, 1e9, 1e25, -10.0]], ids=str)
def test_steep_biases_whose_nearest_keys_are_far(slopes, dtype, D):
    """The last pages are not followed: the nearest key that a query sees is hundreds of positions before it."""
    for news, pasts in (((1, 2), (900, 5000)), ((60, 1), (1500, 300))):
        r = with_form(dtype, D, news, pasts, slopes=slopes)
        bad = {}
        for i, (new, past) in enumerate(zip(news, pasts)):
            pages = -(-(new + past) // 16)
            bad[i] = range(pages - 16, pages)
            r.c.table[i, pages - 16:pages] = -1
        out, lse = r.call()
        r.slopes = torch.tensor(slopes, dtype=torch.float32)
        at = 0
        for i, (new, past) in enumerate(zip(news, pasts)):
            seen = seen_by(past, new)
            for x in bad[i]:
                seen[:, x * 16:(x + 1) * 16] = False
            distance = (torch.arange(past, past + new)[:, None] - torch.arange(past + new)[None]).double()
            for h in range(4):
                w = form64(r.q[at:at + new, h].double(), r.c.keys[i][:, 0].double(), r.c.values[i][:, 0].double(), r.scale, seen, distance, dtype, 0.0, float(r.slopes[h]))
                check(f"lse, sequence {i}, head {h}", lse[h, at:at + new], w[1], w[3])
                check(f"out, sequence {i}, head {h}", out[at:at + new, h], w[0], w[2])
            at += new
