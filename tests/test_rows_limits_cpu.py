"""Sizes of linear attention's buffers for the longest rows, without a GPU."""
import pytest

from paper_2301_09266_amd import finc


@pytest.mark.parametrize("L", [1 << 30, (1 << 31) - 513, (1 << 31) - 512, (1 << 31) - 511, (1 << 31) - 1])
def test_states_of_the_longest_rows(L):
    parts = -(-L // finc.ATTENTION_PART)
    up = lambda n: -(-n // 256) * 256   # noqa: E731
    for H, D in ((1, 1), (2, 8)):
        want = up(H * (parts + 1) * D * D * 4) + up(H * parts * 4)
        assert finc.lib().finc_linear_attention_states_bytes(1, L, H, D, D) == want
        assert finc.lib().finc_linear_attention_workspace_bytes(1, L, H, H, D, D) >= want
