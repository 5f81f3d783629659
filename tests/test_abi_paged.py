"""Refusals of the calls on paged caches, and rotary frequencies (CPU).

Every call carries an argument error that the library must find before its first HIP call; the
fake device pointers are never dereferenced.
"""
import ctypes
import math

import pytest

from paper_2402_04617_amd import infllm as F
from tests.test_abi_host import FAKE, P, L  # noqa: F401  (L: the loaded library, a fixture)
from tests.test_abi_shared import NULL, RANGE, SHAPE, UNSUPPORTED, WORKSPACE, caller, i32, i64  # noqa: F401

D, HQ, HKV = 128, 32, 8


def rot(dim=128, **kw):
    table = (ctypes.c_double * 64)(*[0.5] * 64)
    r = F.Rotary(dim, 0, ctypes.cast(table, ctypes.POINTER(ctypes.c_double)), 1.0, 1, 1e-6, FAKE, FAKE)
    r._held = table
    for name, x in kw.items():
        setattr(r, name, x)
    return ctypes.byref(r)


def pages(**kw):
    g = F.Pages(100, 16, FAKE, FAKE, 16 * HKV * D, D, 16 * D)
    for name, x in kw.items():
        setattr(g, name, x)
    return ctypes.byref(g)


def freqs(*values):
    table = (ctypes.c_double * 64)(*(list(values) + [0.5] * (64 - len(values))))
    return ctypes.cast(table, ctypes.POINTER(ctypes.c_double))


def bad_rotaries():
    yield NULL, None
    for dim in (-2, 130, 3):
        yield SHAPE, rot(dim)
    yield NULL, rot(inv_freq=ctypes.POINTER(ctypes.c_double)())
    for x in (math.nan, math.inf, -0.5):
        yield SHAPE, rot(inv_freq=freqs(0.1, x))
    for x in (math.nan, math.inf):
        yield SHAPE, rot(magnitude=x)
        yield SHAPE, rot(norm_eps=x)
    yield SHAPE, rot(norm_eps=-1e-6)
    yield SHAPE, rot(q_weight=FAKE + 4)
    yield SHAPE, rot(k_weight=FAKE + 8)


def test_rotate_refusals(L):  # noqa: F811
    p = P()
    names = ["p", "rot", "n", "at", "first", "q", "qt", "qh", "qo", "qot", "qoh", "k", "kt", "kh", "ko", "kot", "koh", "stream"]
    row = (HQ + 2 * HKV) * D
    ok = (ctypes.byref(p), rot(), 5, FAKE, 0, FAKE, row, D, FAKE, HQ * D, D, FAKE, row, D, FAKE, HKV * D, D, None)
    call = caller(L.infllm_rotate, names, ok)
    for status, r in bad_rotaries():
        assert call(rot=r) == status
    assert call(p=None) == NULL
    assert call(n=-1) == SHAPE
    assert call(n=0) == 0 and call(q=None, qo=None, k=None, ko=None) == 0   # nothing to do
    for name in ("q", "qo", "k", "ko"):
        assert call(**{name: None}) == NULL, name
        assert call(**{name: FAKE + 8}) == SHAPE, name
    assert call(at=FAKE + 4) == SHAPE
    for name in ("qt", "qh", "qot", "qoh", "kt", "kh", "kot", "koh"):
        assert call(**{name: -8}) == SHAPE, name
        assert call(**{name: 8 * row + 4}) == SHAPE, name
    assert call(qot=D) == SHAPE and call(koh=0) == SHAPE                    # output rows that overlap
    assert call(qot=D, qoh=4 * D) == SHAPE
    assert call(qt=1 << 61) == UNSUPPORTED and call(kot=1 << 61) == UNSUPPORTED
    assert call(n=1 << 30) == UNSUPPORTED and call(n=(1 << 26) - 8192) == UNSUPPORTED
    pr = P(rope_inv_freq=F.rope_frequencies(128))
    assert call(p=ctypes.byref(pr)) == UNSUPPORTED


def bad_pages():
    yield NULL, None
    yield NULL, pages(k=None)
    yield NULL, pages(v=None)
    yield SHAPE, pages(n_pages=0)
    yield SHAPE, pages(page_size=0)
    yield SHAPE, pages(k=FAKE + 8)
    yield SHAPE, pages(v=FAKE + 8)
    for name in ("page_stride", "token_stride", "head_stride"):
        yield SHAPE, pages(**{name: -8})
        yield SHAPE, pages(**{name: 1 << 24 | 4})
        yield SHAPE, pages(**{name: 0})
    yield SHAPE, pages(page_stride=16 * HKV * D - 8)    # the next page's rows begin within the last head
    yield SHAPE, pages(head_stride=15 * D)
    yield SHAPE, pages(token_stride=2 * D)
    yield UNSUPPORTED, pages(page_stride=1 << 58)


SEQS = dict(n=3, lens=i32(1, 0, 40), pasts=i64(15, 5, 24), width=4)


def seq_refusals(call):
    assert call(n=-1) == SHAPE
    assert call(lens=None) == NULL and call(pasts=None) == NULL
    assert call(width=-1) == SHAPE
    assert call(lens=i32(1, -1, 40)) == SHAPE and call(pasts=i64(15, -1, 24)) == SHAPE
    assert call(lens=i32(1, 0, 41)) == RANGE and call(width=3) == RANGE and call(pasts=i64(64, 5, 24)) == RANGE
    assert call(pasts=i64(1 << 31, 5, 24), width=1 << 40) == UNSUPPORTED
    assert call(pasts=i64((1 << 63) - 1, 5, 24)) == UNSUPPORTED
    assert call(width=1 << 60) == UNSUPPORTED
    assert call(lens=i32((1 << 31) - 300, 0, (1 << 31) - 300), pasts=i64(0, 0, 0), width=1 << 40) == UNSUPPORTED
    assert call(table=None) == NULL and call(table=FAKE + 2) == SHAPE
    # nothing to do
    assert call(n=0, lens=None, pasts=None, table=None) == 0
    assert call(lens=i32(0, 0, 0), pasts=i64(1 << 62, 0, 0), table=None) == 0


def test_append_refusals(L):  # noqa: F811
    p = P()
    row = (HQ + 2 * HKV) * D
    names = ["p", "rot", "pages", "n", "lens", "pasts", "table", "width", "q", "qt", "qh", "qo", "qot", "qoh", "k", "v", "kt", "kh", "stream"]
    ok = (ctypes.byref(p), rot(), pages(), SEQS["n"], SEQS["lens"], SEQS["pasts"], FAKE, SEQS["width"], FAKE, row, D, FAKE, HQ * D, D,
          FAKE, FAKE, row, D, None)
    call = caller(L.infllm_paged_append, names, ok)
    for status, r in bad_rotaries():
        if r is not None:
            assert call(rot=r) == status
    for status, g in bad_pages():
        assert call(pages=g) == status
    seq_refusals(call)
    assert call(p=None) == NULL
    for name in ("q", "qo", "k", "v"):
        assert call(**{name: None}) == NULL, name
        assert call(**{name: FAKE + 8}) == SHAPE, name
    for name in ("qt", "qh", "qot", "qoh", "kt", "kh"):
        assert call(**{name: -8}) == SHAPE, name
        assert call(**{name: 8 * row + 4}) == SHAPE, name
    assert call(qot=D) == SHAPE
    assert call(qt=1 << 61) == UNSUPPORTED and call(kt=1 << 61) == UNSUPPORTED and call(qot=1 << 61) == UNSUPPORTED
    pr = P(rope_inv_freq=F.rope_frequencies(128))
    assert call(p=ctypes.byref(pr)) == UNSUPPORTED


def test_attend_refusals(L):  # noqa: F811
    p = P()
    names = ["p", "pages", "n", "lens", "pasts", "table", "width", "score", "q", "qt", "qh", "out", "ot", "oh", "lse", "ws", "wb", "stream"]
    ok = (ctypes.byref(p), pages(), SEQS["n"], SEQS["lens"], SEQS["pasts"], FAKE, SEQS["width"], None, FAKE, HQ * D, D, FAKE, HQ * D, D,
          None, None, 0, None)
    call = caller(L.infllm_paged_attend, names, ok)
    for status, g in bad_pages():
        assert call(pages=g) == status
    seq_refusals(call)
    for kw in (dict(softcap=-1.0), dict(softcap=1e-39), dict(softcap=math.nan), dict(softcap=math.inf), dict(window=-1), dict(n_init=-1), dict(slopes=FAKE + 2)):
        f = F.ScoreForm(**kw)
        assert call(score=ctypes.byref(f)) == SHAPE, kw
        assert L.infllm_paged_workspace_bytes(ctypes.byref(p), pages(), 3, SEQS["lens"], SEQS["pasts"], ctypes.byref(f)) == 0
    assert call(p=None) == NULL
    for name in ("q", "out"):
        assert call(**{name: None}) == NULL, name
        assert call(**{name: FAKE + 8}) == SHAPE, name
    for name in ("qt", "qh", "ot", "oh"):
        assert call(**{name: -8}) == SHAPE, name
        assert call(**{name: 8 * D * HQ + 4}) == SHAPE, name
    assert call(ot=D) == SHAPE and call(oh=0) == SHAPE
    assert call(ot=D, oh=40 * D) == SHAPE                                   # 41 tokens
    assert call(qt=1 << 61) == UNSUPPORTED and call(ot=1 << 61) == UNSUPPORTED
    assert call(lse=FAKE + 2) == SHAPE
    # rows of k past 64 GiB
    assert call(pages=pages(page_stride=(1 << 35) // 99 // 8 * 8 + 64)) == UNSUPPORTED
    # tokens 256 MiB apart
    assert call(pages=pages(token_stride=1 << 27, page_stride=1 << 31, n_pages=2)) == UNSUPPORTED
    # total * G past 2^31
    assert call(lens=i32(1 << 29, 0, 1), pasts=i64(0, 0, 0), width=1 << 30) == UNSUPPORTED
    pr = P(rope_inv_freq=F.rope_frequencies(128))
    assert call(p=ctypes.byref(pr)) == UNSUPPORTED
    uneven = (pages(), 2, i32(1, 1), i64(30000, 100), None)
    assert L.infllm_paged_workspace_bytes(ctypes.byref(p), *uneven) > 0
    assert L.infllm_paged_workspace_bytes(ctypes.byref(pr), *uneven) == 0


def test_page_tables_that_the_wrappers_refuse(L):  # noqa: F811
    import torch
    p, g = P(), F.Pages(100, 16, FAKE, FAKE, 16 * HKV * D, D, 16 * D)
    wide = torch.zeros((3, 8), dtype=torch.int32)
    for table, lens, pasts in ((wide[:1], (1, 1), (0, 0)), (wide.long(), (1,), (0,)), (wide.T, (1,), (0,)), (wide.T, (1, 1), (0, 0)),
                               (wide[:, 4:], (1, 0, 40), (63, 1 << 40, 25)), (wide[:, 7:], (1, 1), (0, 16))):
        with pytest.raises(ValueError):
            F.infllm_paged_append(p, None, g, lens, pasts, table, None, None, None, None, FAKE, FAKE, (HKV * D, D))
        with pytest.raises(ValueError):
            F.infllm_paged_attend(p, g, lens, pasts, table, None, FAKE, (HQ * D, D), FAKE, (HQ * D, D))
    for table in (wide[1:2, 4:], wide[:, 4:][:2]):         # a single row, and rows of a wider table: too many tokens for their pages
        with pytest.raises((ValueError, F.InfllmError)):
            F.infllm_paged_attend(p, g, (1,) * len(table), (64,) * len(table), table, None, FAKE, (HQ * D, D), FAKE, (HQ * D, D),
                                  stream=FAKE)
    with pytest.raises(ValueError):
        F.infllm_paged_append(p, None, g, (1, 1), (0,), wide, None, None, None, None, FAKE, FAKE, (HKV * D, D))


def test_workspace_of_uneven_batches(L):  # noqa: F811
    # one token beside sequences whose keys are tens of thousands of tiles, of every type and head layout
    seqs = [(1, 0), (1, 1), (3, 60000), (700, 0), (1, 100000), (5000, 1 << 20), (1, 10 ** 7), (40, (1 << 31) - 300)]
    forms = [None, F.ScoreForm(window=4096, n_init=128), F.ScoreForm(window=1), F.ScoreForm(n_init=(1 << 31) - 1, window=(1 << 31) - 1)]
    for dtype, size in (("bf16", 2), ("f32", 4)):
        for d, hq, hkv in ((128, 32, 8), (64, 8, 8), (128, 5, 1)):
            p = P(n_q_heads=hq, n_kv_heads=hkv, head_dim=d, dtype=dtype)
            for some in (seqs[:2], seqs[:5], seqs, seqs[::-1], [(1, 0)] * 191 + [(1, 10 ** 7)], [(1, 0), (1, 1 << 30)] * 96):
                for form in forms:
                    n = F.infllm_paged_workspace_bytes(p, F.Pages(100, 16, FAKE, FAKE, 16 * hkv * d, d, 16 * d),
                                                       [x for x, _ in some], [y for _, y in some], form)
                    parts = 256 * hkv * sum(-(-x * hq // hkv // 32) for x, _ in some)  # of row tiles of 32 rows and more
                    assert 0 <= n <= parts * 128 * (d * size + 8) + 255


def test_frequencies():
    turns = lambda t, n: n * t / (2 * math.pi)  # noqa: E731
    plain = F.infllm_rope_frequencies(64, 10000.0)
    assert plain == pytest.approx([10000.0 ** (-i / 32) for i in range(32)], rel=1e-15)
    assert F.infllm_rope_frequencies(64, 10000.0, "linear", 4.0) == pytest.approx([x / 4 for x in plain], rel=1e-15)
    base = F.infllm_rope_frequencies(64, 10000.0, "base", 8.0)
    # the fastest pair as it was, the slowest slowed by the factor
    assert base[0] == 1.0 and base[-1] == pytest.approx(plain[-1] / 8, rel=1e-13)
    parts = F.infllm_rope_frequencies(64, 10000.0, "parts", 8.0, 4096, 1.0, 32.0)
    kept = [i for i, t in enumerate(plain) if turns(t, 4096) >= 32]
    slowed = [i for i, t in enumerate(plain) if turns(t, 4096) <= 1]
    assert kept and slowed and len(kept) + len(slowed) < 32
    for i, t in enumerate(plain):
        if i in kept:
            assert parts[i] == pytest.approx(t, rel=1e-15)
        elif i in slowed:
            assert parts[i] == pytest.approx(t / 8, rel=1e-15)
        else:
            g = (turns(t, 4096) - 1) / 31
            assert parts[i] == pytest.approx(g * t + (1 - g) * t / 8, rel=1e-13)
    assert F.infllm_rope_frequencies(0) == []
    assert F.infllm_rope_frequencies(128) == pytest.approx(F.rope_frequencies(128), rel=1e-14)


@pytest.mark.parametrize("kw", [
    dict(rotary_dim=-2), dict(rotary_dim=3), dict(base=0.0), dict(base=math.nan), dict(scaling="linear", factor=0.0),
    dict(scaling="base", factor=math.inf), dict(scaling="base", rotary_dim=2, factor=2.0),
    dict(scaling="parts", factor=2.0, original_len=0), dict(scaling="parts", factor=2.0, original_len=10, slow=3.0, fast=3.0),
    dict(scaling="parts", factor=2.0, original_len=10, slow=math.nan)])
def test_frequency_refusals(kw):
    with pytest.raises(F.InfllmError):
        F.infllm_rope_frequencies(**dict(dict(rotary_dim=64), **kw))


def test_frequency_status(L):  # noqa: F811
    one = ctypes.c_double * 4
    d = ctypes.c_double
    assert L.infllm_rope_frequencies(8, d(1e4), 4, d(1), 0, d(1), d(2), ctypes.addressof(one())) == SHAPE
    assert L.infllm_rope_frequencies(8, d(1e4), 0, d(1), 0, d(1), d(2), None) == NULL


def test_binding_numbers():
    """Lengths that do not fit their type, or do not match, are refused by the binding."""
    p, g = P(), F.Pages(100, 16, FAKE, FAKE, 16 * HKV * D, D, 16 * D)
    with pytest.raises(OverflowError):
        F.infllm_paged_workspace_bytes(p, g, [1 << 31], [0])
    with pytest.raises(OverflowError):
        F.infllm_paged_workspace_bytes(p, g, [1], [1 << 63])
    with pytest.raises(ValueError):
        F.infllm_paged_workspace_bytes(p, g, [1, 1], [0])
