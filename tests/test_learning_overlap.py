"""Outputs that begin where an input does that is still read when they are written are refused (no GPU
needed: every call below fails validation)."""
from paper_1503_08294_amd import gsn

X, W, Q, S, Y, T, R, D = (i << 20 for i in range(1, 9))  # never dereferenced
LOTS = 1 << 60


def test_rows_in_8_bits():
    for q, s in ((X, S), (Q, X), (Q, Q)):
        assert gsn._lib.gsn_quantise(gsn.GSN_F32, 4, 64, X, 64, q, 64, s, None) == gsn.GSN_E_INVAL


def test_layers_in_8_bits():
    p = gsn.gsn_linear_params(gsn.GSN_BF16, 64, 64, 8)
    for y in (X, W, S):
        assert gsn._lib.gsn_linear_quantised(p, X, 64, W, 64, S, y, 64, R, LOTS,
                                             None) == gsn.GSN_E_INVAL


def test_cross_entropy():
    p = gsn.gsn_entropy_params(gsn.GSN_BF16, 64, 100, 8)
    for loss, stats in ((T, None), (X, None), (W, S), (S, S), (Y, X), (Y, W), (Y, T)):
        assert gsn._lib.gsn_cross_entropy(p, X, 64, W, 64, T, None, loss, stats, R, LOTS,
                                          None) == gsn.GSN_E_INVAL
    # dw: a piece of the classes after the other, each from all of x, the targets and the statistics
    for dx, dw in ((Y, Y), (None, X), (Y, X), (None, T), (None, S), (None, D), (D, None), (T, None)):
        assert gsn._lib.gsn_cross_entropy_backward(p, D, X, 64, W, 64, T, None, S, dx, dw, R, LOTS,
                                                   None) == gsn.GSN_E_INVAL
