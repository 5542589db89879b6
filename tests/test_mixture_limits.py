"""Sizes past what the kernels count in 32 bits are refused on the host (no GPU needed)."""
import pytest

from paper_1503_08294_amd import gsn

FAKE = 1 << 20  # never dereferenced: every call below fails validation first


@pytest.mark.parametrize("dim", [(1 << 27) + 1, 1 << 28, (1 << 31) - 257, (1 << 31) - 1])
def test_layer_norm_rows(dim):
    """A row's last step would pass 2^31, or the join of the columns' sums 2^32 threads."""
    assert gsn._lib.gsn_layer_norm(gsn.GSN_BF16, gsn.GSN_F32, 1, dim, FAKE, dim, None, None, 1e-5,
                                   FAKE, dim, None, None) == gsn.GSN_E_INVAL
    assert gsn._lib.gsn_layer_norm_backward(
        gsn.GSN_BF16, gsn.GSN_F32, 1, dim, FAKE, dim, FAKE, dim, None, FAKE, FAKE, dim, FAKE,
        FAKE, FAKE, 1 << 40, None) == gsn.GSN_E_INVAL
    assert gsn.gsn_layer_norm_workspace_bytes(1, dim) == 0
    assert gsn.gsn_layer_norm_workspace_bytes(1, 1 << 27) > 0
