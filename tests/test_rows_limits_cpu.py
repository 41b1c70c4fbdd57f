"""Sizes at their limits, of linear attention's longest rows and of embeddings, without a GPU."""
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


@pytest.mark.parametrize("M,V,D,fits", [
    (1, 1, (1 << 31) - 512, True), (1, 1, (1 << 31) - 511, False), (1, 1, (1 << 31) - 1, False),
    (0, 1, (1 << 31) - 4, False), (8, 1, 1 << 30, True), (16, 1, 1 << 30, False),
    ((1 << 30) - 1, 4, 8, True), (1 << 30, 4, 8, False), (4, 1 << 30, 8, False)])
def test_embedding_sizes(M, V, D, fits):
    """Rows whose columns do not count within 31 bits, to the end of the last slice of 512."""
    n = finc.lib().finc_embed_workspace_bytes(M, V, D)
    assert (n > 0) == fits
    if not fits:
        at = [1 << 52, 2 << 52, 3 << 52, 4 << 52]
        assert finc.lib().finc_embed_backward(0, at[0], 1, at[1], D, at[2], M, V, D, 1.0, at[3],
                                              None) == finc.EINVAL
        assert finc.lib().finc_embed_forward(0, 0, at[0], 1, at[1], D, at[2], D, M, V, D, 1.0,
                                             None) == finc.EINVAL
