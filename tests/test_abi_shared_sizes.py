"""Sizes and strides of the shared-document calls whose products wrap in 64 bits (CPU): refused before the first HIP
call, like the ones that merely pass 31 bits, and without a workspace."""
import ctypes

from paper_2402_04617_amd import infllm as F
from tests.test_abi_host import FAKE, P, L, mem  # noqa: F401  (L: the loaded library, a fixture)
from tests.test_abi_shared import BIG, RANGE, UNSUPPORTED, i32, i64

B31, B62 = (1 << 31) - 1, 1 << 62


def test_prefix_rows(L):  # noqa: F811
    """2^30 heads by 2^30 tokens by 64 continuations: 2^66 rows, 0 in 64 bits."""
    p = P(n_q_heads=1 << 30, n_kv_heads=1, dtype=F.INFLLM_F32)
    n = 1 << 30
    own = mem(batch=64, capacity=1 << 31)
    st = L.infllm_prefix_attend(ctypes.byref(p), ctypes.byref(mem()), 5, ctypes.byref(own), i64(*[0] * 64), FAKE, 128 << 30, None, None, 0,
                                n, FAKE, 0, FAKE, 128 << 30, None, FAKE, BIG, None)
    assert st == UNSUPPORTED
    assert L.infllm_prefix_score(ctypes.byref(p), ctypes.byref(mem()), 64, FAKE, 128 << 30, n, 5, FAKE, FAKE, BIG, None) == UNSUPPORTED
    for batch, n_q in ((64, n), (B31, B31), (1 << 20, 1 << 14)):
        assert L.infllm_prefix_workspace_bytes(ctypes.byref(p), batch, n_q, 100, 100) == 0
    assert L.infllm_prefix_workspace_bytes(ctypes.byref(P()), B31, B31, 100, 100) == 0


def test_prefix_strides_and_stores(L):  # noqa: F811
    p = P(dtype=F.INFLLM_F32)
    own = mem(batch=3, capacity=1000)

    def call(m=mem(), own=own, qs=256, kvs=256, os=256, lens=i64(5, 0, 900)):
        return L.infllm_prefix_attend(ctypes.byref(p), ctypes.byref(m), 5, ctypes.byref(own), lens, FAKE, qs, FAKE, FAKE, kvs, 2, FAKE, 0,
                                      FAKE, os, None, FAKE, BIG, None)
    for name in ("qs", "kvs", "os"):
        for stride in (B62, B62 >> 6):
            assert call(**{name: stride}) == UNSUPPORTED, (name, stride)
    for capacity in (B62, 1 << 55, (1 << 63) - 1):
        assert call(m=mem(capacity=capacity)) == UNSUPPORTED
        assert call(own=mem(batch=3, capacity=capacity)) == UNSUPPORTED
    assert call(lens=i64(5, 0, 999)) == RANGE
    assert L.infllm_prefix_score(ctypes.byref(p), ctypes.byref(mem()), 4, FAKE, B62, 1, 5, FAKE, FAKE, BIG, None) == UNSUPPORTED


def test_prompt_strides(L):  # noqa: F811
    p = P(dtype=F.INFLLM_F32)

    def call(lens=(5, 300), qt=4096, qh=128, kt=1024, kh=128, ot=4096, oh=128):
        return L.infllm_prompt_attend(ctypes.byref(p), len(lens), i32(*lens), FAKE, qt, qh, FAKE, FAKE, kt, kh, FAKE, ot, oh, None, None, 0, None)
    for name in ("qt", "qh", "kt", "kh", "ot"):
        for stride in (B62, B62 >> 4):
            assert call(**{name: stride}) == UNSUPPORTED, (name, stride)
    assert call(ot=128, oh=B62 >> 4) == UNSUPPORTED


def test_copy_sizes(L):  # noqa: F811
    def call(p, **kw):
        src, dst = mem(batch=2, **kw), mem(batch=4, k=2 * FAKE, v=2 * FAKE, **kw)
        return L.infllm_copy_sequences(ctypes.byref(p), ctypes.byref(dst), ctypes.byref(src), 1, i32(3), i32(1), i64(5), i32(0), None)
    assert call(P(n_q_heads=1 << 30, n_kv_heads=1 << 30), ring=1 << 29) == UNSUPPORTED    # 2^65 pieces of a ring
    assert call(P(), capacity=1 << 55) == UNSUPPORTED                                      # slots past 2^62 bytes
    assert call(P(), capacity=(1 << 63) - 1) == UNSUPPORTED
