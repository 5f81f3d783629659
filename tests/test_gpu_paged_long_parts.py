"""Paged attention whose parts are longer than what is looked up of them at once (GPU).

Key places are looked up ahead: of row tiles 1,024 entries in LDS (128 key tiles of 64 with pages of a multiple of 8 tokens,
16 with others; float32: 256 and 32 tiles of 32), of few rows 32 or 4 tiles in registers.  Batches that fill the chip keep
a sequence's keys in one part, and so come to the entries behind.  All sequences here share one document's pages."""
import math

import pytest
import torch

from paper_2402_04617_amd import infllm as F
from tests.paged_util import DT, attend64, params, seen_by
from tests.shared_util import check
from tests.test_gpu_paged_attend import FORMS as SCORE_FORMS, Run

pytestmark = pytest.mark.gpu

HKV, D, LONGEST = 8, 64, 17_500


class Shared:
    """n sequences of `new` tokens each, at and before the end of one document in pages."""

    def __init__(self, dtype, G, page, n, new, form, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.dtype, self.G, self.page, self.new = dtype, G, page, new
        self.Hq = G * HKV
        self.keys, self.values = (torch.randn((LONGEST, HKV, D), generator=g).to(DT[dtype]) for _ in range(2))
        count = -(-LONGEST // page)
        k = torch.full((count + 2, page, HKV, D), math.nan, dtype=DT[dtype])
        v = k.clone()
        place = torch.randperm(count + 2, generator=g)[:count]
        for cache, rows in ((k, self.keys), (v, self.values)):
            at = torch.arange(LONGEST)
            cache[place[at // page], at % page] = rows
        self.k, self.v = k.cuda(), v.cuda()
        self.pages = F.pages(self.k, self.v, page, page * HKV * D, HKV * D, D)
        self.table = place.to(torch.int32)[None].repeat(n, 1)
        self.pasts = [LONGEST - new - 13 * i for i in range(n)]
        self.form = dict(form)
        self.slopes = None
        if self.form.pop("slopes", False):
            self.slopes = torch.tensor([2.0 ** (-8.0 * (h + 1) / self.Hq) for h in range(self.Hq)], dtype=torch.float32)
        self.score = F.score(slopes=None if self.slopes is None else self.slopes.cuda(), **self.form)
        self.q = torch.randn((n * new, self.Hq, D), generator=g).to(DT[dtype])
        self.p = params(self.Hq, HKV, D, dtype, D ** -0.5)
        self.news = [new] * n
        self.bad = {}

    def lose(self, i, pages):
        """Entries of sequence i's table that are not followed."""
        self.bad[i] = pages
        for j, x in enumerate(pages):
            self.table[i, x] = (-1, 1 << 30)[j % 2]

    def part_tiles(self):
        """Fewest key tiles of a sequence's parts but the last, from the workspace: partial rows of every part."""
        size = F.infllm_paged_workspace_bytes(self.p, self.pages, self.news, self.pasts, self.score)
        rows = min(128 if self.dtype == "bf16" else 32 << (self.new * self.G > 32), -(-self.new * self.G // 8) * 8)
        items = size // (D * 2 + 8 if self.dtype == "bf16" else D * 4 + 4) // (HKV * rows)
        most = max(1, -(-items // len(self.news)))          # (sequences of nearly one length)
        keys = min(min(self.pasts), self.form.get("window", LONGEST) or LONGEST)
        return keys // (64 if self.dtype == "bf16" else 32) // most

    def call(self):
        q = self.q.cuda()
        out = torch.full_like(q, 7.0)
        lse = torch.full((self.Hq, len(q)), 7.0, dtype=torch.float32, device="cuda")
        ws = torch.empty(max(256, F.infllm_paged_workspace_bytes(self.p, self.pages, self.news, self.pasts, self.score)), dtype=torch.uint8, device="cuda")
        F.infllm_paged_attend(self.p, self.pages, self.news, self.pasts, self.table.cuda(), self.score, q, (self.Hq * D, D), out, (self.Hq * D, D), lse, ws)
        return out, lse

    def verify(self, out, lse, seqs):
        out, lse = out.cpu(), lse.cpu()
        assert torch.isfinite(out).all() and torch.isfinite(lse).all()
        for i in seqs:
            past, row = self.pasts[i], i * self.new
            end = past + self.new
            seen = seen_by(past, self.new, self.form.get("window", 0), self.form.get("n_init", 0))
            for x in self.bad.get(i, ()):
                seen[:, x * self.page:(x + 1) * self.page] = False
            distance = (torch.arange(past, end)[:, None] - torch.arange(end)[None]).double()
            for h in (0, self.Hq // 2, self.Hq - 1):
                slope = 0.0 if self.slopes is None else float(self.slopes[h])
                w = attend64(self.q[row:row + self.new, h].double(), self.keys[:end, h // self.G].double(), self.values[:end, h // self.G].double(),
                             D ** -0.5, seen, self.dtype, self.form.get("softcap", 0.0), None if self.slopes is None else -slope * distance, slope)
                check(f"out, sequence {i}, head {h}", out[row:row + self.new, h], w[0], w[2])
                check(f"lse, sequence {i}, head {h}", lse[h, row:row + self.new], w[1], w[3])


FORMS = [dict(), dict(slopes=True), dict(window=12_000, n_init=200), dict(softcap=30.0, slopes=True, window=14_000, n_init=70), dict(softcap=100.0)]


@pytest.mark.parametrize("form", FORMS, ids=lambda f: " ".join(f"{k}={v}" for k, v in f.items()) or "plain")
@pytest.mark.parametrize("dtype,G,page,new,ahead", [
    ("bf16", 1, 16, 40, 128), ("bf16", 4, 50, 33, 16),      # row tiles
    ("bf16", 4, 16, 1, 32), ("bf16", 5, 50, 3, 4),          # few rows
    ("f32", 1, 16, 33, 256), ("f32", 2, 50, 20, 32), ("f32", 1, 50, 1, 32)])
def test_parts_longer_than_what_is_looked_up(dtype, G, page, new, ahead, form):
    n = 126
    a = Shared(dtype, G, page, n, new, form)
    pages = a.table.shape[1]
    # in the first look-up, behind it alone, in the last tiles of the past, and on both sides of the 128th tile
    a.lose(3, [2, 3, pages // 3])
    a.lose(5, [2 * pages // 3])
    a.lose(7, [(a.pasts[7] - 1) // page - 1])
    a.lose(9, [8192 // page - 1, 8192 // page, pages // 2])
    assert a.part_tiles() > ahead + 8
    out, lse = a.call()
    a.verify(out, lse, (0, 3, 5, 7, 9, n - 1))
    again = a.call()
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("form", SCORE_FORMS, ids=lambda f: " ".join(f"{k}={v}" for k, v in f.items()))
@pytest.mark.parametrize("page", [16, 50])
def test_score_forms_of_shared_keys(form, page):
    """4 to 16 rows of a kv head, all of which share the keys of a tile between the waves."""
    r = Run((1, 4, 3, 1, 2), (1300, 700, 131, 0, 5000), 8, 2, 128, page, "bf16", form=form, q_scale=2.0)
    r.verify(*r.call())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq", [130, 300])
def test_groups_larger_than_a_row_tile(dtype, Hq):
    """One kv head for 130 and 300 query heads: row tiles that end within a token's heads."""
    r = Run((1, 3, 0, 2), (900, 70, 5, 0), Hq, 1, 64, 16, dtype, form=dict(window=300, n_init=9))
    r.verify(*r.call(), heads=[0, 1, 63, 64, 127, 128, Hq - 2, Hq - 1])
