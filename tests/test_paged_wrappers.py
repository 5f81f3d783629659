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
