"""What the Python wrappers of the calls on paged caches refuse: tensors that the device would read at other places or as
other numbers (CPU; the fake device pointers are never dereferenced)."""
import pytest
import torch

from paper_2402_04617_amd import infllm as F
from tests.test_abi_host import FAKE, P, L  # noqa: F401  (L: the loaded library, a fixture)

D, HQ, HKV = 128, 32, 8


def rotate(n, positions, rot=None, p=None):
    rot = F.rotary([0.5] * (D // 2)) if rot is None else rot
    F.infllm_rotate(P() if p is None else p, rot, n, positions, FAKE, (HQ * D, D), FAKE, (HQ * D, D), None, None, None, None, stream=FAKE)


def past_the_wrapper(call):
    """The library itself is reached: here, without a device, it says so."""
    try:
        call()
    except F.InfllmError as e:
        assert e.code == 7


@pytest.mark.parametrize("positions", [
    torch.zeros(5, dtype=torch.int32), torch.zeros(5, dtype=torch.float64), torch.zeros(4, dtype=torch.int64),
    torch.zeros(10, dtype=torch.int64)[::2], torch.zeros((5, 2), dtype=torch.int64)[:, 0]])
def test_positions(L, positions):  # noqa: F811
    with pytest.raises(ValueError, match="positions"):
        rotate(5, positions)


def test_positions_that_do(L):  # noqa: F811
    if torch.cuda.is_available():
        pytest.skip("fake pointers")
    for positions in (torch.zeros(5, dtype=torch.int64), torch.zeros(9, dtype=torch.int64)[2:], torch.zeros((1, 5), dtype=torch.int64), FAKE, None):
        past_the_wrapper(lambda: rotate(5, positions))


def append(rot):
    g = F.Pages(100, 16, FAKE, FAKE, 16 * HKV * D, D, 16 * D)
    F.infllm_paged_append(P(), rot, g, (1,), (0,), FAKE, None, None, None, None, FAKE, FAKE, (HKV * D, D), table_stride=4, stream=FAKE)


@pytest.mark.parametrize("which", ["q_weight", "k_weight"])
@pytest.mark.parametrize("weight", [
    torch.ones(D), torch.ones(D, dtype=torch.float16), torch.ones(D // 2, dtype=torch.bfloat16), torch.ones((HQ, D), dtype=torch.bfloat16)])
def test_weights(L, which, weight):  # noqa: F811
    """Of a bf16 layer: float32 weights (as checkpoints often hold them), other types, other lengths."""
    rot = F.rotary([0.5] * (D // 2), norm=True, **{which: weight})
    with pytest.raises(ValueError, match=which):
        rotate(5, None, rot)
    with pytest.raises(ValueError, match=which):
        append(rot)
    with pytest.raises(ValueError, match=which):
        F.rotary([], norm=True, **{which: torch.ones(2 * D, dtype=torch.bfloat16)[::2]})


def test_weights_that_do(L):  # noqa: F811
    if torch.cuda.is_available():
        pytest.skip("fake pointers")
    one = torch.ones(D + 8, dtype=torch.bfloat16)
    for w in (one[8:], one[:D].view(1, D), FAKE, None):
        past_the_wrapper(lambda: rotate(5, None, F.rotary([0.5] * (D // 2), norm=True, q_weight=w, k_weight=w)))
        past_the_wrapper(lambda: append(F.rotary([], norm=True, q_weight=w, k_weight=w)))
    past_the_wrapper(lambda: rotate(5, None, F.rotary([], norm=True, q_weight=torch.ones(D)), P(dtype="f32")))
    past_the_wrapper(lambda: rotate(5, None, F.rotary([], q_weight=torch.ones(D))))      # without norms they are not read
    past_the_wrapper(lambda: append(None))


def attend(score=None, pages=None, table=FAKE, table_stride=4, p=None, lens=(1,), pasts=(0,)):
    g = F.Pages(100, 16, FAKE, FAKE, 16 * HKV * D, D, 16 * D) if pages is None else pages
    F.infllm_paged_attend(P() if p is None else p, g, lens, pasts, table, score, FAKE, (HQ * D, D), FAKE, (HQ * D, D), table_stride=table_stride,
                          stream=FAKE)


def test_slopes(L):  # noqa: F811
    for slopes in (torch.ones(HQ, dtype=torch.bfloat16), torch.ones(HQ, dtype=torch.float64), torch.ones(2 * HQ)[::2], torch.ones(0)):
        with pytest.raises(ValueError, match="slopes"):
            F.score(slopes=slopes)
    for n in (1, HKV, HQ - 1, HQ + 1):
        with pytest.raises(ValueError, match="slopes"):
            attend(F.score(slopes=torch.ones(n)))


def test_slopes_that_do(L):  # noqa: F811
    if torch.cuda.is_available():
        pytest.skip("fake pointers")
    for slopes in (torch.ones(HQ), torch.ones((HKV, HQ // HKV)), torch.ones(2 * HQ)[HQ:], FAKE, None):
        past_the_wrapper(lambda: attend(F.score(softcap=3.0, slopes=slopes)))
    past_the_wrapper(lambda: attend(F.ScoreForm(window=5, slopes=FAKE)))
    past_the_wrapper(lambda: attend(None))


def test_page_tables(L):  # noqa: F811
    for dtype in (torch.float32, torch.int64, torch.int16):
        for stride in (None, 4):
            with pytest.raises(ValueError, match="page_table"):
                attend(table=torch.zeros((2, 4), dtype=dtype), table_stride=stride)
            with pytest.raises(ValueError, match="page_table"):
                g = F.Pages(100, 16, FAKE, FAKE, 16 * HKV * D, D, 16 * D)
                F.infllm_paged_append(P(), None, g, (1, 1), (0, 0), torch.zeros((2, 4), dtype=dtype), None, None, None, None, FAKE, FAKE,
                                      (HKV * D, D), table_stride=stride, stream=FAKE)


def test_page_tables_that_do(L):  # noqa: F811
    if torch.cuda.is_available():
        pytest.skip("fake pointers")
    table = torch.zeros((2, 4), dtype=torch.int32)
    for stride in (None, 4):
        past_the_wrapper(lambda: attend(table=table, table_stride=stride, lens=(1, 1), pasts=(0, 63)))


def test_pages(L):  # noqa: F811
    k = torch.zeros((6, HKV, 16, D), dtype=torch.bfloat16)
    for v in (k.float(), k[:5], torch.zeros((6, 16, HKV, D), dtype=torch.bfloat16), torch.zeros((6, 16, HKV, D), dtype=torch.bfloat16).transpose(1, 2),
              torch.zeros((6, HKV, 16, D + 8), dtype=torch.bfloat16)[..., :D]):
        with pytest.raises(ValueError, match="k and v"):
            F.pages(k, v, 16)
    t = torch.zeros((6, HKV, D, 16), dtype=torch.bfloat16).transpose(2, 3)
    with pytest.raises(ValueError, match="row"):
        F.pages(t, t, 16)
    # another type than the layer's, and rows behind the tensors' end
    f = k.float()
    for g in (F.pages(f, f, 16), F.pages(k, k, 17), F.pages(k[:, :4], k[:, 4:], 16, token_stride=2 * D), F.pages(k[:, 4:], k[:, 4:], 16),
              F.pages(k[1:], k[1:], 16, page_stride=17 * HKV * D), F.pages(k.view(-1)[:1], k.view(-1)[:1], 1 << 20, HKV * D, HKV * D, D)):
        with pytest.raises(ValueError, match="[kv]: "):
            attend(pages=g)
        with pytest.raises(ValueError, match="[kv]: "):
            F.infllm_paged_append(P(), None, g, (1,), (0,), FAKE, None, None, None, None, FAKE, FAKE, (HKV * D, D), table_stride=4, stream=FAKE)


def test_pages_that_do(L):  # noqa: F811
    if torch.cuda.is_available():
        pytest.skip("fake pointers")
    one = torch.zeros((1, HKV, 16, D), dtype=torch.bfloat16)
    both = torch.zeros((6, 2, 16, HKV, D + 8), dtype=torch.bfloat16)
    k = torch.zeros((6, HKV, 16, D), dtype=torch.bfloat16)
    for g in (F.pages(k, k.clone(), 16), F.pages(k, k, 8), F.pages(one, both.view(-1)[:16 * HKV * D].view(1, HKV, 16, D), 16),
              F.pages(both[:, 0], both[:, 1], 16, both.stride(0), HKV * (D + 8), D + 8),
              F.pages(both[:, 0, ..., :D], both[:, 1, ..., :D], 16, both.stride(0), HKV * (D + 8), D + 8),
              F.pages(k.transpose(1, 2), k.transpose(1, 2), 16, k.stride(0), D, 16 * D)):
        for _ in range(2):
            past_the_wrapper(lambda: attend(pages=g))
    f = k.float()
    past_the_wrapper(lambda: attend(pages=F.pages(f, f, 16), p=P(dtype="f32")))
    past_the_wrapper(lambda: attend(pages=F.pages(k, k, 16), p=P(n_q_heads=4, n_kv_heads=4)))


@pytest.mark.parametrize("kw", [
    dict(base=1e300, scaling="base", factor=1e9), dict(base=1e-300, scaling="base", factor=1e-30), dict(scaling="linear", factor=1e-310, base=1e-3),
    dict(scaling="parts", factor=1e-310, original_len=4096, base=1e-10), dict(scaling="linear", factor=5e-324)])
def test_frequencies_past_float64(L, kw):  # noqa: F811
    """A base or a frequency that overflows, or a base of 0, is refused, and not returned as 0 or infinity."""
    with pytest.raises(F.InfllmError):
        F.infllm_rope_frequencies(64, **kw)


def test_frequencies_at_the_ends(L):  # noqa: F811
    for kw in (dict(base=1e300), dict(base=1e-300), dict(base=1e300, scaling="linear", factor=1e-5), dict(base=1e-250, scaling="base", factor=1e-20)):
        x = F.infllm_rope_frequencies(64, **kw)
        assert len(x) == 32 and all(0.0 < y < float("inf") for y in x), kw
