"""Refusals of the entry points for packed prompts, shared documents and copies (CPU).

Every call carries an argument error that the library must find before its first HIP call; the
fake device pointers are never dereferenced.
"""
import ctypes

import pytest

from paper_2402_04617_amd import infllm as F
from tests.test_abi_host import FAKE, P, L, mem  # noqa: F401  (L: the loaded library, a fixture)

BIG = 1 << 40
NULL, SHAPE, RANGE, UNSUPPORTED, WORKSPACE = 1, 2, 3, 4, 5


def i32(*x):
    return (ctypes.c_int32 * len(x))(*x)


def i64(*x):
    return (ctypes.c_int64 * len(x))(*x)


def caller(fn, names, ok):
    def call(**kw):
        a = dict(zip(names, ok))
        assert set(kw) <= set(names)
        a.update(kw)
        return fn(*a.values())
    return call


def test_prompt_refusals(L):  # noqa: F811
    p = P()
    D, Hq, Hkv = 128, 32, 8
    lens = i32(5, 0, 300)
    names = ["p", "n", "lens", "q", "qt", "qh", "k", "v", "kt", "kh", "out", "ot", "oh", "lse", "ws", "wb", "stream"]
    ok = (ctypes.byref(p), 3, lens, FAKE, Hq * D, D, FAKE, FAKE, Hkv * D, D, FAKE, Hq * D, D, None, None, 0, None)
    call = caller(L.infllm_prompt_attend, names, ok)
    for name in ("p", "lens", "q", "k", "v", "out"):
        assert call(**{name: None}) == NULL, name
    assert call(n=-1) == SHAPE
    assert call(lens=i32(5, -1, 300)) == SHAPE
    assert call(n=0, lens=None, q=None) == 0             # nothing to do
    assert call(lens=i32(0, 0, 0), q=None) == 0
    for name in ("q", "k", "v", "out"):
        assert call(**{name: FAKE + 8}) == SHAPE, name     # not 16-byte aligned
    for name in ("qt", "qh", "kt", "kh", "ot", "oh"):
        assert call(**{name: -8}) == SHAPE, name
        assert call(**{name: 8 * D + 4}) == SHAPE, name    # rows not on 16 bytes
    assert call(ot=D, oh=D) == SHAPE                      # output rows that overlap
    assert call(ot=0) == SHAPE
    assert call(ot=Hq * D - 8) == SHAPE
    assert call(ot=D, oh=304 * D) == SHAPE                # one row short
    assert call(kt=1 << 24) == UNSUPPORTED                # 300 keys of 32 MiB each: past 4 GiB
    assert call(lens=i32(1 << 30, 1 << 30, 1 << 30)) == UNSUPPORTED
    assert call(lens=i32(1 << 29, 5, 5)) == UNSUPPORTED   # total * G past 2^31
    pr = P(rope_inv_freq=F.rope_frequencies(128))
    assert call(p=ctypes.byref(pr)) == UNSUPPORTED
    bad = P(head_dim=96)
    assert call(p=ctypes.byref(bad)) == UNSUPPORTED


def test_prefix_score_refusals(L):  # noqa: F811
    p, m = P(), mem()
    names = ["p", "m", "batch", "q", "qs", "n_q", "units", "scores", "ws", "wb", "stream"]
    call = caller(L.infllm_prefix_score, names, (ctypes.byref(p), ctypes.byref(m), 4, FAKE, 128, 1, 100, FAKE, FAKE, 1 << 20, None))
    for name in ("p", "m", "q", "scores", "ws"):
        assert call(**{name: None}) == NULL, name
    assert call(m=ctypes.byref(mem(unit_ksum=None))) == NULL
    assert call(m=ctypes.byref(mem(unit_ksum=FAKE + 4))) == SHAPE
    assert call(m=ctypes.byref(mem(batch=2))) == SHAPE
    assert call(batch=0) == SHAPE
    assert call(n_q=-1) == SHAPE
    assert call(units=-1) == SHAPE
    assert call(units=2049) == RANGE
    assert call(qs=120) == SHAPE
    assert call(q=FAKE + 2) == SHAPE
    assert call(wb=16) == WORKSPACE
    assert call(ws=FAKE + 4) == SHAPE
    assert call(batch=1 << 20) == UNSUPPORTED
    assert call(units=0, q=None, scores=None, ws=None) == 0
    pr = P(rope_inv_freq=F.rope_frequencies(128))
    assert call(p=ctypes.byref(pr)) == UNSUPPORTED


def test_prefix_attend_refusals(L):  # noqa: F811
    p, m = P(), mem()
    own = mem(batch=3, capacity=1000, max_units=0, repr_idx=None, unit_ksum=None, qprefix=None, rpart=None, ring=0)
    lens = i64(5, 0, 900)
    names = ["p", "m", "len", "own", "lens", "q", "qs", "k", "v", "kvs", "n_q", "idx", "n_idx", "out", "os", "lse", "ws", "wb", "stream"]
    ok = (ctypes.byref(p), ctypes.byref(m), 20000, ctypes.byref(own), lens, FAKE, 256, FAKE, FAKE, 256, 2, FAKE, 32, FAKE, 256, None,
          FAKE, BIG, None)
    call = caller(L.infllm_prefix_attend, names, ok)
    for name in ("p", "m", "own", "lens", "q", "k", "v", "idx", "out"):
        assert call(**{name: None}) == NULL, name
    assert call(m=ctypes.byref(mem(k=None))) == NULL
    assert call(own=ctypes.byref(mem(batch=3, capacity=1000, v=None))) == NULL
    assert call(m=ctypes.byref(mem(batch=2))) == SHAPE
    assert call(own=ctypes.byref(mem(batch=0, capacity=1000))) == SHAPE
    assert call(own=ctypes.byref(mem(batch=65, capacity=1000)), lens=i64(*[0] * 65)) == UNSUPPORTED
    assert call(len=-1) == SHAPE
    assert call(len=(1 << 17) + 1) == RANGE
    assert call(lens=i64(5, -1, 900)) == SHAPE
    assert call(lens=i64(5, 0, 999)) == RANGE             # 999 + 2 tokens in 1,000
    assert call(n_q=-1) == SHAPE
    assert call(n_idx=-1) == SHAPE
    for name in ("qs", "kvs", "os"):
        assert call(**{name: 255}) == SHAPE, name
    for name in ("q", "k", "v", "out"):
        assert call(**{name: FAKE + 2}) == SHAPE, name
    assert call(ws=None) == WORKSPACE
    assert call(wb=2 * 3 * 32 * 2 * 264) == WORKSPACE     # two parts' rows: three regions need three
    assert call(ws=FAKE + 4) == SHAPE
    assert call(n_q=0) == 0
    wide = mem(batch=3, capacity=1 << 24)                 # 3 * 32 * 2^23 rows in all
    assert call(own=ctypes.byref(wide), n_q=1 << 23, qs=128 << 23, kvs=128 << 23, os=128 << 23) == UNSUPPORTED
    far = mem(capacity=1 << 25)
    assert call(m=ctypes.byref(far)) == UNSUPPORTED       # 2^25 rows of 256 bytes: past 4 GiB
    pr = P(rope_inv_freq=F.rope_frequencies(128))
    assert call(p=ctypes.byref(pr)) == UNSUPPORTED


def test_prefix_workspace(L):  # noqa: F811
    p = P()
    f = lambda *a: L.infllm_prefix_workspace_bytes(ctypes.byref(p), *a)  # noqa: E731
    assert f(0, 1, 100, 100) == 0 and f(1, -1, 100, 100) == 0 and f(1, 1, -1, 100) == 0 and f(1, 1, 100, -1) == 0
    assert L.infllm_prefix_workspace_bytes(None, 1, 1, 100, 100) == 0
    row = 2 * 128 + 8
    for batch, n_q, length, cap in ((1, 1, 0, 1), (4, 1, 31999, 300), (64, 8, 1 << 20, 4096), (3, 200, 5, 1000)):
        size = f(batch, n_q, length, cap)
        assert size % 256 == 0 and size >= batch * n_q * 32 * row
        # the query sums of scoring: a part for every 128 rows of a group, 16 at most
        assert size >= batch * 8 * min(16, -(-4 * n_q // 128)) * 128 * 4


def test_copy_refusals(L):  # noqa: F811
    p = P()
    src, dst = mem(batch=2), mem(batch=4, k=2 * FAKE, v=2 * FAKE)
    names = ["p", "dst", "src", "n", "to", "from", "lens", "units", "stream"]
    call = caller(L.infllm_copy_sequences, names, (ctypes.byref(p), ctypes.byref(dst), ctypes.byref(src), 2, i32(0, 3), i32(1, 1),
                                                   i64(5000, 100), i32(6, 0), None))
    for name in ("p", "dst", "src", "to", "from", "lens", "units"):
        assert call(**{name: None}) == NULL, name
    for field in ("k", "v", "qprefix", "rpart", "unit_ksum", "repr_idx"):
        assert call(src=ctypes.byref(mem(batch=2, **{field: None}))) == NULL, field
    assert call(src=ctypes.byref(mem(batch=2, qprefix=FAKE + 8))) == SHAPE
    assert call(src=ctypes.byref(mem(batch=2, ring=0))) == SHAPE
    assert call(n=-1) == SHAPE
    assert call(n=0, to=None) == 0
    many = 65
    assert call(n=many, to=i32(*range(many)), **{"from": i32(*[0] * many)}, lens=i64(*[1] * many), units=i32(*[0] * many)) == UNSUPPORTED
    assert call(to=i32(0, 4)) == RANGE
    assert call(to=i32(-1, 3)) == RANGE
    assert call(**{"from": i32(1, 2)}) == RANGE
    assert call(lens=i64(-1, 100)) == SHAPE
    assert call(lens=i64((1 << 17) + 1, 100)) == RANGE
    assert call(units=i32(-1, 0)) == SHAPE
    assert call(units=i32(7, 0)) == SHAPE                  # 5,000 tokens hold 6 evicted units
    assert call(dst=ctypes.byref(mem(batch=4, k=2 * FAKE, max_units=5))) == RANGE
    assert call(to=i32(3, 3)) == SHAPE                     # two copies to one slot
    same = mem(batch=4)
    assert call(dst=ctypes.byref(same), src=ctypes.byref(same), **{"from": i32(1, 0)}, to=i32(2, 1)) == SHAPE  # slot 1 is read too
    assert call(dst=ctypes.byref(same), src=ctypes.byref(same), **{"from": i32(1, 0)}, to=i32(1, 2)) == SHAPE
    pr = P(rope_inv_freq=F.rope_frequencies(128))
    assert call(p=ctypes.byref(pr)) == NULL                # the remap's rotated keys


def test_numbers_past_64_bits(L):  # noqa: F811
    """Arguments whose products do not fit 64 bits are refused like the ones that do."""
    D, Hq, Hkv, huge = 128, 32, 8, 1 << 62
    p, one = P(), P(n_q_heads=1, n_kv_heads=1)
    prompt = lambda q, lens, ot, oh: L.infllm_prompt_attend(  # noqa: E731
        ctypes.byref(q), len(lens), lens, FAKE, Hq * D, D, FAKE, FAKE, Hkv * D, D, FAKE, ot, oh, None, None, 0, None)
    assert prompt(p, i32(1 << 20), huge, huge) == SHAPE       # rows of neither stride step over the other's
    assert prompt(p, i32(1 << 20), huge >> 10, huge) == SHAPE
    assert prompt(p, i32(1), huge, 0) == SHAPE                # one token, heads on top of each other
    assert prompt(one, i32(300), 0, huge) == SHAPE            # one head, tokens on top of each other
    size = lambda *lens: L.infllm_prompt_workspace_bytes(ctypes.byref(one), len(lens), i32(*lens))  # noqa: E731
    assert size(*[(1 << 31) - 1] * 3) == 0                    # what the attention refuses has no workspace
    assert size(4000) > 0                                     # (one head of 4,000 rows leaves most units idle: split)
    own = mem(batch=1, capacity=(1 << 63) - 1)
    attend = lambda m, o, n, lens: L.infllm_prefix_attend(  # noqa: E731
        ctypes.byref(p), ctypes.byref(m), 5, ctypes.byref(o), lens, FAKE, 256, FAKE, FAKE, 256, n, FAKE, 0, FAKE, 256, None, FAKE, BIG, None)
    assert attend(mem(), own, 2, i64((1 << 63) - 1)) == RANGE
    assert attend(mem(), own, 2, i64(0)) == UNSUPPORTED       # (bf16: slices past 4 GiB)
    assert attend(mem(capacity=1 << 56), mem(batch=1, capacity=100), 2, i64(0)) == UNSUPPORTED


@pytest.mark.parametrize("lens", [(3,), (1, 2, 3, 4)])
def test_binding_checks_lengths(L, lens):  # noqa: F811
    own = mem(batch=2, capacity=100)
    with pytest.raises(ValueError):
        F.infllm_prefix_attend(P(), mem(), 10, own, lens, FAKE, 128, None, None, 0, 1, None, 0, FAKE, 128, stream=0)
    with pytest.raises(ValueError):
        F.infllm_copy_sequences(P(), mem(), mem(), [0, 1], [0], [1, 1], [0, 0], stream=0)
