"""Attention over paged caches (infllm_paged_attend) against attention in 64 bits (GPU)."""
import math

import pytest
import torch

from paper_2402_04617_amd import infllm as F
from tests.gpu_util import log
from tests.paged_util import DT, Cache, attend64, params, seen_by
from tests.shared_util import check

pytestmark = pytest.mark.gpu


class Run:
    """One call's inputs: pages, queries (NaN behind the last token), outputs (7 behind it)."""

    def __init__(self, news, pasts, Hq, Hkv, D, page, dtype, order="heads", form=None, q_order="tokens", seed=0, q_scale=1.0, fill=math.nan):
        self.news, self.pasts, self.Hq, self.Hkv, self.D, self.dtype, self.q_order = tuple(news), tuple(pasts), Hq, Hkv, D, dtype, q_order
        self.c = Cache([a + b for a, b in zip(news, pasts)], Hkv, D, page, dtype, order, seed=seed + 1, fill=fill)
        self.scale = D ** -0.5
        self.p = params(Hq, Hkv, D, dtype, self.scale)
        self.total = sum(news)
        g = torch.Generator().manual_seed(seed)
        self.q = (torch.randn((self.total + 3, Hq, D), generator=g) * q_scale).to(DT[dtype])
        self.q[self.total:] = math.nan
        self.form = dict(form or {})
        self.slopes = None
        if self.form.pop("slopes", False):
            self.slopes = torch.tensor([2.0 ** (-8.0 * (h + 1) / Hq) for h in range(Hq)], dtype=torch.float32)
        self.score = F.score(slopes=None if self.slopes is None else self.slopes.cuda(), **self.form) if form else None
        if q_order == "tokens":
            self.qd, self.st = self.q.cuda(), (Hq * D, D)
        else:
            self.qd, self.st = self.q.transpose(0, 1).contiguous().cuda(), (D, (self.total + 3) * D)

    def ws_bytes(self):
        return F.infllm_paged_workspace_bytes(self.p, self.c.struct, self.news, self.pasts, self.score)

    def call(self, stream=None, spare_ws=0):
        size = self.ws_bytes()
        ws = torch.empty(size + spare_ws, dtype=torch.uint8, device="cuda").fill_(255) if size + spare_ws else None
        out = torch.full_like(self.qd, 7.0)
        lse = torch.full((self.Hq, self.total), 7.0, dtype=torch.float32, device="cuda")
        F.infllm_paged_attend(self.p, self.c.struct, self.news, self.pasts, self.c.table, self.score, self.qd, self.st, out, self.st, lse,
                              ws, stream=stream)
        return (out if self.q_order == "tokens" else out.transpose(0, 1)), lse

    def visible(self, i, bad=()):
        """[new][key] of sequence i; `bad` places of its table are not followed."""
        seen = seen_by(self.pasts[i], self.news[i], self.form.get("window", 0), self.form.get("n_init", 0))
        for x in bad:
            seen[:, x * self.c.page:(x + 1) * self.c.page] = False
        return seen

    def verify(self, out, lse, bad=None, heads=None):
        at = 0
        out, lse = out.cpu(), lse.cpu()
        for i, (new, past) in enumerate(zip(self.news, self.pasts)):
            if new == 0:
                continue
            seen = self.visible(i, (bad or {}).get(i, ()))
            distance = torch.arange(past, past + new)[:, None] - torch.arange(past + new)[None]
            for h in heads or range(self.Hq):
                kv = h // (self.Hq // self.Hkv)
                slope = 0.0 if self.slopes is None else float(self.slopes[h])
                w = attend64(self.q[at:at + new, h].double(), self.c.keys[i][:, kv].double(), self.c.values[i][:, kv].double(), self.scale,
                             seen, self.dtype, self.form.get("softcap", 0.0), None if self.slopes is None else -slope * distance.double(), slope)
                check(f"out, sequence {i} ({past} + {new}), head {h}", out[at:at + new, h], w[0], w[2])
                check(f"lse, sequence {i} ({past} + {new}), head {h}", lse[h, at:at + new], w[1], w[3])
            at += new
        assert torch.all(out[self.total:] == 7), "rows behind the last token were written"


MIXED = ((1, 0, 63, 1, 64, 5, 0, 130, 1), (0, 70, 1, 64, 63, 500, 0, 77, 1023))
STEPS = ((1,) * 7, (0, 1, 63, 64, 700, 2047, 129))

CASES = [
    ("bf16", 4, 1, 128, 16, "heads", (1,), (0,)),
    ("bf16", 8, 2, 128, 16, "heads", *MIXED),
    ("bf16", 8, 2, 64, 64, "tokens", *MIXED),
    ("bf16", 3, 3, 128, 24, "apart", *MIXED),
    ("bf16", 5, 1, 64, 1, "tokens", *MIXED),
    ("bf16", 12, 4, 128, 50, "heads", *MIXED),
    ("bf16", 16, 2, 128, 256, "apart", *STEPS),
    ("bf16", 32, 8, 128, 16, "heads", *STEPS),
    ("bf16", 7, 7, 64, 8, "heads", *STEPS),
    ("bf16", 4, 1, 128, 64, "heads", (700,), (333,)),
    ("bf16", 2, 1, 64, 128, "tokens", (300, 300), (0, 4000)),
    ("bf16", 8, 2, 128, 16, "heads", (8,) * 4, (0, 57, 900, 2011)),   # 32 rows of a kv head
    ("bf16", 9, 1, 64, 50, "tokens", (3, 2, 1, 4), (61, 640, 0, 1500)),
    ("bf16", 4, 1, 128, 1, "heads", (7, 4, 1), (1, 333, 4000)),
    ("bf16", 17, 1, 128, 32, "heads", (1, 1, 2), (5, 1029, 700)),
    ("bf16", 33, 1, 64, 8, "apart", (1, 1), (63, 470)),
    ("f32", 4, 1, 128, 16, "heads", (1,), (0,)),
    ("f32", 4, 2, 64, 24, "tokens", *MIXED),
    ("f32", 8, 2, 128, 64, "apart", *STEPS),
    ("f32", 3, 1, 128, 1, "heads", *MIXED),
    ("f32", 2, 2, 64, 50, "heads", (200,), (611,)),
]


@pytest.mark.parametrize("dtype,Hq,Hkv,D,page,order,news,pasts", CASES)
def test_attend(dtype, Hq, Hkv, D, page, order, news, pasts):
    r = Run(news, pasts, Hq, Hkv, D, page, dtype, order, q_order="tokens" if page % 16 == 0 else "heads")
    log(f"[paged] {dtype} {Hq}/{Hkv} x {D}, pages of {page}, {news} after {pasts}, workspace {r.ws_bytes()}")
    out, lse = r.call()
    r.verify(out, lse)
    again = r.call(spare_ws=4096)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1]), "not the same bits"


FORMS = [
    dict(softcap=5.0),
    dict(slopes=True),
    dict(window=1),
    dict(window=100),
    dict(window=64, n_init=64),
    dict(window=300, n_init=5),
    dict(window=40, n_init=1 << 30),
    dict(window=2000, n_init=3),
    dict(softcap=2.0, slopes=True, window=130, n_init=70),
    dict(n_init=7),                              # without a window: everything
]


@pytest.mark.parametrize("form", FORMS, ids=lambda f: " ".join(f"{k}={v}" for k, v in f.items()))
@pytest.mark.parametrize("dtype,Hq,Hkv,D,page,order", [
    ("bf16", 8, 2, 128, 16, "heads"), ("bf16", 3, 1, 64, 50, "tokens"), ("f32", 4, 2, 64, 24, "heads"), ("f32", 4, 4, 128, 64, "tokens")])
def test_score_forms(form, dtype, Hq, Hkv, D, page, order):
    news, pasts = (1, 70, 1, 0, 129, 1), (900, 333, 0, 9, 1100, 64)
    r = Run(news, pasts, Hq, Hkv, D, page, dtype, order, form=form, q_scale=2.0)
    r.verify(*r.call())


@pytest.mark.parametrize("form", FORMS, ids=lambda f: " ".join(f"{k}={v}" for k, v in f.items()))
def test_score_forms_of_few_rows(form):
    """Rows that share the keys between the waves: 4 to 32 of a kv head."""
    r = Run((1, 8, 5, 1), (1300, 700, 131, 0), 8, 2, 128, 16, "bf16", form=form, q_scale=2.0)
    r.verify(*r.call())


def test_a_struct_of_zeros_changes_nothing():
    a = Run(*MIXED, 8, 2, 128, 16, "bf16")
    b = Run(*MIXED, 8, 2, 128, 16, "bf16", form=dict(window=0))
    assert b.score is not None
    for x, y in zip(a.call(), b.call()):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype,D,page,form", [
    ("bf16", 128, 16, None), ("bf16", 64, 50, dict(window=90, n_init=20)), ("bf16", 128, 64, dict(softcap=3.0)), ("f32", 64, 16, None),
    ("f32", 128, 7, dict(slopes=True))])
def test_bad_pages_are_not_seen(dtype, D, page, form):
    """Entries out of range, in the middle, first and last; a sequence whose pages are all bad gives zeros and -inf."""
    news, pasts = (1, 60, 3, 1, 2), (500, 200, 0, 130, 129)
    r = Run(news, pasts, 4, 2, D, page, dtype, form=form)
    n = r.c.k.shape[0]
    pages = [-(-(a + b) // page) for a, b in zip(news, pasts)]
    bad = {0: (0, pages[0] // 2), 1: (pages[1] - 1, 1), 2: tuple(range(pages[2])), 4: tuple(range(pages[4]))}
    for i, places in bad.items():
        for j, x in enumerate(places):
            r.c.table[i, x] = (-1, n, (1 << 31) - 1, -(1 << 31))[j % 4]
    out, lse = r.call()
    assert torch.all(lse[:, 61:64] == -math.inf) and torch.all(out[61:64] == 0)
    r.verify(out, lse, bad)


@pytest.mark.parametrize("dtype,D,form", [("bf16", 128, None), ("bf16", 64, dict(window=70, n_init=3)), ("f32", 64, None), ("f32", 128, dict(softcap=4.0))])
def test_values_that_are_not_finite_stay_with_the_rows_that_see_them(dtype, D, form):
    news, pasts = (40, 1, 100), (60, 300, 150)
    clean = Run(news, pasts, 4, 2, D, 16, dtype, form=form)
    odd = Run(news, pasts, 4, 2, D, 16, dtype, form=form)
    at = [(0, 80, "values", math.inf), (0, 91, "keys", math.nan), (2, 200, "values", math.nan), (2, 249, "keys", math.inf), (2, 30, "values", -math.inf)]
    for i, t, what, x in at:
        page, slot = int(odd.c.host_table[i, t // 16]), t % 16
        getattr(odd.c, what)[i][t, 1, 3] = x
        (odd.c.k if what == "keys" else odd.c.v)[page, 1, slot, 3] = x
    out, lse = odd.call()
    want, want_lse = clean.call()
    row = 0
    for i, (new, past) in enumerate(zip(news, pasts)):
        seen = clean.visible(i)
        touched = torch.zeros(new, dtype=torch.bool)
        for j, t, what, x in at:
            if j == i:
                touched |= seen[:, t]
        for h in range(4):
            hit = touched if h >= 2 else torch.zeros(new, dtype=torch.bool)
            o, w = out[row:row + new, h].cpu(), want[row:row + new, h].cpu()
            assert torch.isfinite(o[~hit]).all(), f"sequence {i}, head {h}"
            # (a row formed apart from its tile's is rounded elsewhere)
            assert ((o[~hit].double() - w[~hit].double()).abs() <= (2e-2 if dtype == "bf16" else 1e-5)).all()
            assert torch.equal(lse[h, row:row + new].cpu()[~hit], want_lse[h, row:row + new].cpu()[~hit])
        row += new
    # a value that is seen reaches its own dimension alone
    row = 40 + 1
    seen = clean.visible(2)
    for j in range(100):
        o = out[row + j, 2:].cpu()
        if form is None and seen[j, 30] and not seen[j, 200]:
            assert torch.all(o[:, 3] == -math.inf) and torch.isfinite(o[:, :3]).all() and torch.isfinite(o[:, 4:]).all()
    # a NaN score is its row's: key 91 of the first sequence
    for j in range(40):
        if clean.visible(0)[j, 91]:
            assert torch.isnan(out[j, 2:]).all() and torch.isnan(lse[2:, j]).all()


@pytest.mark.parametrize("form", [None, dict(window=70, n_init=3), dict(softcap=4.0, slopes=True)], ids=str)
@pytest.mark.parametrize("page", [16, 50])
def test_values_that_are_not_finite_with_few_rows(form, page):
    """Two current tokens of four heads: an infinite value and a NaN key that only the second sees, and values that the
    window hides from both; split and whole."""
    for past in (100, 6000):
        clean, odd = (Run((2, 1), (past, 40), 4, 1, 128, page, "bf16", form=form) for _ in range(2))
        at = [(past + 1, "values", math.inf), (past - 80, "values", math.nan)] if form and "window" in form else [(past + 1, "values", math.inf)]
        for t, what, x in at:
            odd.c.v[int(odd.c.host_table[0, t // page]), 0, t % page, 3] = x
        out, lse = odd.call()
        want, want_lse = clean.call()
        assert torch.equal(lse, want_lse)
        assert torch.isfinite(out[0]).all() and (out[0].double() - want[0].double()).abs().max() <= 2e-2
        assert torch.all(out[1, :, 3] == math.inf) and torch.isfinite(out[1, :, :3]).all() and torch.isfinite(out[1, :, 4:]).all()
        assert torch.equal(out[2], want[2])
        odd.c.k[int(odd.c.host_table[0, (past + 1) // page]), 0, (past + 1) % page, 5] = math.nan
        out, lse = odd.call()
        assert torch.isfinite(out[0]).all() and torch.isnan(out[1]).all() and torch.isnan(lse[:, 1]).all()
        assert torch.equal(out[2], want[2]) and torch.equal(lse[:, 0], want_lse[:, 0])


def test_low_and_high_scores():
    """Rows whose scores lie far below or above 0, and rise or fall along the keys."""
    for sign in (1, -1):
        for slope in (0.0, 1.0):
            r = Run((90, 1), (200, 411), 2, 1, 64, 16, "bf16", seed=4)
            ramp = torch.linspace(0, 1, 412)[:, None, None] * slope + (1 - slope)
            for i in range(2):
                k = (sign * 30 * ramp[:len(r.c.keys[i])] * torch.ones_like(r.c.keys[i].float())).to(torch.bfloat16)
                r.c.keys[i] = k
                for t in range(len(k)):
                    r.c.k[int(r.c.host_table[i, t // 16]), :, t % 16] = k[t].cuda()
            r.q[:r.total] = r.q[:r.total].abs()
            r.qd = r.q.cuda()
            r.verify(*r.call())


def test_more_sequences_than_a_launch_takes():
    news = [(i * 5) % 3 for i in range(300)]
    pasts = [(i * 37) % 200 for i in range(300)]
    r = Run(news, pasts, 2, 1, 64, 16, "bf16")
    r.verify(*r.call())


@pytest.mark.parametrize("before,between,behind", [(0, 0, 9), (0, 0, 400), (193, 0, 0), (5, 300, 200), (192, 192, 192)])
def test_batches_padded_with_empty_sequences(before, between, behind):
    """192 sequences and more of which the first, some between and the last have no new token."""
    some = [(1, 5), (3, 40), (1, 700), (2, 0)]
    seqs = [(0, 0)] * before + some * 24 + [(0, 3)] * between + some * 24 + [(0, 0)] * behind
    r = Run([a for a, _ in seqs], [b for _, b in seqs], 2, 1, 64, 16, "bf16")
    out, lse = r.call()
    r.verify(out, lse, heads=[1])
    assert torch.isfinite(lse).all() and not (lse[0] == 7).any()


@pytest.mark.parametrize("dtype,Hq,new,past,step", [("bf16", 32, 300, 6000, 150), ("f32", 8, 150, 1500, 60)])
def test_more_partial_rows_than_workgroups_at_once(dtype, Hq, new, past, step):
    """A chunk and single tokens in more parts than the chip has places for the merge's workgroups."""
    singles = 24
    r = Run((1,) * 11 + (new,) + (1,) * (singles - 11), tuple(range(50, 50 + 11 * step, step)) + (past,) + tuple(range(50 + 11 * step, 50 + singles * step, step)),
            Hq, 8, 128, 16, dtype)
    rows = r.ws_bytes() // (128 * 2 + 8 if dtype == "bf16" else 128 * 4 + 4)
    log(f"[paged] {dtype}: {rows} partial rows")
    out, lse = r.call()
    r.verify(out, lse, heads=[0, 13 % Hq, Hq - 1])
    again = r.call()
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


def test_shared_pages():
    """Sequences that share a prompt's pages see the same keys as with copies of their own."""
    r = Run((1, 1, 5), (160, 160, 156), 4, 2, 128, 16, "bf16")
    for i in (1, 2):
        for x in range(9):
            r.c.table[i, x] = r.c.host_table[0, x]
        r.c.keys[i][:144], r.c.values[i][:144] = r.c.keys[0][:144], r.c.values[0][:144]
    r.verify(*r.call())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pages_past_32_bit_offsets(dtype):
    """Pages whose rows lie past 2^32 bytes and 2^31 elements."""
    r = Run((1, 3), (70, 130), 4, 1, 128, 64, dtype)
    size = 64 * 128 * (2 if dtype == "bf16" else 4)
    n = (9 << 30) // size
    k = torch.empty((n, 1, 64, 128), dtype=DT[dtype], device="cuda")
    v = torch.empty_like(k)
    place = torch.linspace(0, n - 1, r.c.k.shape[0]).long()
    k[place.cuda()], v[place.cuda()] = r.c.k, r.c.v
    table = r.c.host_table.clone()
    for i in range(2):
        used = -(-(r.news[i] + r.pasts[i]) // 64)
        table[i, :used] = place[table[i, :used].long()].to(torch.int32)
    r.c.struct, r.c.table = F.pages(k, v, 64), table.cuda()
    r.verify(*r.call())


def test_a_table_wider_than_its_rows():
    """Tables with a row stride of their own (a view of a larger one)."""
    r = Run((3, 1), (40, 99), 4, 2, 128, 16, "bf16")
    wide = torch.full((2, 20), 1 << 30, dtype=torch.int32, device="cuda")
    wide[:, :r.c.table.shape[1]] = r.c.table
    r.c.table = wide[:, :r.c.table.shape[1]]
    r.verify(*r.call())


def test_workspace_refusal():
    r = Run((1,), (30000,), 4, 1, 128, 16, "bf16")
    size = r.ws_bytes()
    out = torch.zeros_like(r.qd)
    if size == 0:
        pytest.skip("the keys are not split")
    for ws in (None, torch.empty(size // 2, dtype=torch.uint8, device="cuda")):
        with pytest.raises(F.InfllmError) as e:
            F.infllm_paged_attend(r.p, r.c.struct, r.news, r.pasts, r.c.table, None, r.qd, r.st, out, r.st, None, ws)
        assert e.value.code == 5
    assert torch.all(out == 0)
