"""Host numbers of the batch calls in the binding (CPU): any integers, refused where they do not fit, never wrapped."""
import numpy as np
import pytest

from paper_2402_04617_amd import infllm as F
from tests.test_abi_host import FAKE, P, L, mem  # noqa: F401  (L: the loaded library, a fixture)


@pytest.mark.parametrize("n", [1 << 31, (1 << 32) + 5, -(1 << 31) - 1])
def test_lengths_past_32_bits(L, n):  # noqa: F811
    with pytest.raises(OverflowError):
        F.infllm_prompt_workspace_bytes(P(), [3, n])
    with pytest.raises(OverflowError):
        F.infllm_prompt_attend(P(), [3, n], FAKE, (4096, 128), FAKE, FAKE, (1024, 128), FAKE, (4096, 128), stream=0)
    for at in (0, 1, 3):  # destination, source, units
        pairs = [[0], [1], [4], [0]]
        pairs[at] = [n]
        with pytest.raises(OverflowError):
            F.infllm_copy_sequences(P(), mem(batch=2), mem(batch=2), *pairs, stream=0)


@pytest.mark.parametrize("n", [1 << 63, (1 << 64) + 7])
def test_lengths_past_64_bits(L, n):  # noqa: F811
    with pytest.raises(OverflowError):
        F.infllm_copy_sequences(P(), mem(batch=2), mem(batch=2), [0], [1], [n], [0], stream=0)
    with pytest.raises(OverflowError):
        F.infllm_prefix_attend(P(), mem(), 10, mem(batch=1, capacity=100), [n], FAKE, 128, None, None, 0, 1, None, 0, FAKE, 128, stream=0)


def test_integers_of_any_kind(L):  # noqa: F811
    p = P(n_q_heads=4, n_kv_heads=1)
    want = F.infllm_prompt_workspace_bytes(p, [4000, 0, 17])
    assert want > 0
    for lens in ((4000, 0, 17), np.array([4000, 0, 17]), np.array([4000, 0, 17], np.int16), [np.int32(4000), np.uint8(0), 17]):
        assert F.infllm_prompt_workspace_bytes(p, lens) == want
    assert F.infllm_prompt_workspace_bytes(p, []) == 0
    with pytest.raises(TypeError):
        F.infllm_prompt_workspace_bytes(p, [4000.5])
