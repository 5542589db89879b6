"""What the learning calls ask of a workspace (no GPU needed)."""
import pytest

from paper_1503_08294_amd import gsn


@pytest.mark.parametrize("tokens", [1, 2, 16, 17, 64])
@pytest.mark.parametrize("dim", [1_001, 4_096, 100_000])
def test_a_few_tokens_take_no_copy_of_the_weights(tokens, dim):
    """They read w as it is, whatever its alignment: the tokens in 8 bits and their scales are kept,
    each up to 256 bytes, and 256 to align the whole."""
    for out in (64, 1 << 20):
        p = gsn.gsn_linear_params(gsn.GSN_BF16, dim, out, tokens)
        size = gsn.gsn_linear_quantised_workspace_bytes(p)
        assert 0 < size <= tokens * (dim + 15) + 4 * tokens + 3 * 256


def test_many_tokens_take_one():
    p = gsn.gsn_linear_params(gsn.GSN_BF16, 1_001, 1 << 12, 65)
    assert gsn.gsn_linear_quantised_workspace_bytes(p) >= 1_008 << 12
