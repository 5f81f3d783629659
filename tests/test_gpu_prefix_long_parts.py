"""Prefix attention where a workgroup's part of the keys is longer than its table of positions (GPU): 16 tiles of 64
keys where the initial tokens or the units are not a multiple of 8, 128 tiles else.  Many rows leave each region one
to three parts; the lengths put the part's end on either side of each move of the table."""
import random

import pytest
import torch

from paper_2402_04617_amd import infllm as F
from tests.gpu_util import log
from tests.shared_util import attend64, check
from tests.test_gpu_prefix import Case, params

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def freed():
    yield
    torch.cuda.empty_cache()


def verify_some(c, n):
    """n pairs of continuation and head against 64 bits; no NaN anywhere (every key that nobody sees is one)."""
    assert not torch.isnan(c.out[:, :, :c.n_q].float()).any() and not torch.isnan(c.lse).any()
    dtype = "bf16" if c.dt == torch.bfloat16 else "f32"
    r = random.Random(c.length)
    for b, h in [(0, 0), (c.B - 1, c.p.n_q_heads - 1)] + [(r.randrange(c.B), r.randrange(c.p.n_q_heads)) for _ in range(n)]:
        k, v, seen = c.want(b, h)
        w = attend64(c.q[b, h, :c.n_q].double().cpu(), k, v, float(c.p.sm_scale), seen, dtype)
        check(f"out of continuation {b}, head {h}", c.out[b, h, :c.n_q], w[0], w[2])
        check(f"lse of continuation {b}, head {h}", c.lse[b, h], w[1], w[3])


@pytest.mark.parametrize("init,block,lengths", [
    (5, 37, (900, 1790, 1919, 1985, 2050, 2177, 4100, 6200)),  # 2 and 3 parts of 7 to 33 tiles
    (16, 64, (24300, 24580, 24800, 49300)),                     # 3 parts of 127 to 257 tiles
])
def test_document_parts_past_the_table(init, block, lengths):
    p = params(64, 8, 64, "bf16", local=100000, init=init, block=block, topk=0)
    for length in lengths:
        log(f"[prefix] whole document of {length}, init={init}")
        c = Case(p, 64, 8, length, (0,) * 64, seed=length)
        c.run()
        verify_some(c, 6)


@pytest.mark.parametrize("Hq,D,k_m,idx", [(8, 64, 100, "some"), (8, 128, 57, "units"), (16, 64, 28, "some"), (8, 64, 90, "units")])
def test_units_past_the_table(Hq, D, k_m, idx):
    """Units of 37 tokens: 17 to 58 tiles of a continuation in one part, some of the entries to skip."""
    log(f"[prefix] {k_m} units of 37, {Hq} heads of {D}, {idx}")
    c = Case(params(Hq, 8, D, "bf16", local=100, init=5, block=37, topk=k_m), 64, 1, 9000, (0,) * 64, seed=k_m, idx=idx)
    c.run()
    verify_some(c, 12)


@pytest.mark.parametrize("own", [16300, 16900, 17700])
def test_own_tokens_past_the_table(own):
    """Four continuations of some 17,000 tokens of their own: two parts of 128 and more tiles, X at the second's end."""
    log(f"[prefix] {own} own tokens")
    c = Case(params(64, 8, 64, "bf16"), 4, 256, 1000, (own, own - 64, own - 500, own), seed=own)
    c.run()
    verify_some(c, 2)
