"""The range of what the experts' products round between them: that of the elements' type."""
import pytest
import torch

from test_gpu_mixture import F16, TYPES, expert_inputs, expert_tolerance, experts_in_float64, near

pytestmark = pytest.mark.gpu

# few pairs; tiles of 64, 128 and 256
SIZES = [(20, 8, 2, 72, 40), (300, 3, 2, 136, 72), (3000, 4, 2, 515, 701), (3000, 4, 2, 520, 1032)]


@pytest.fixture(scope="module")
def mix():
    from paper_1503_08294_amd import mixture
    return mixture


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,experts,k,dim,hidden", SIZES)
def test_large_activations(mix, dtype, tokens, experts, k, dim, hidden):
    """One token whose activations pass 65,520: not finite in float16 and right otherwise; the
    other tokens have what they had."""
    x, ids, weights, w1, w2, _ = (t.cuda() for t in expert_inputs(dtype, tokens, experts, k, dim,
                                                                 hidden, 65))
    good = mix.experts(x, ids, weights, w1, w2)
    x[7] *= 1024  # gates and ups of about 1,000: products up to some 10^6
    for got in (mix.experts(x, ids, weights, w1, w2),
                mix.experts_forward(x, ids, weights, w1, w2)[0]):
        rest = torch.arange(tokens, device="cuda") != 7
        rel = expert_tolerance(dtype, dim, hidden, tokens * k)
        near(got[rest], good[rest].double().cpu(), 2 * rel, "the others")
        if dtype == F16:
            assert not torch.isfinite(got[7]).any()
        else:
            want = experts_in_float64(x, ids, weights, w1, w2, x)[0].detach()
            near(got[7:8], want[7:8].cpu(), rel, "out")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,experts,k,dim,hidden", SIZES)
def test_small_gradients(mix, dtype, tokens, experts, k, dim, hidden):
    """Gradients of gate and up of less than 2^-25: float16 has none of them, and dout scaled by
    a power of two brings them back."""
    x, ids, weights, w1, w2, dout = expert_inputs(dtype, tokens, experts, k, dim, hidden, 66)
    # d = 2^-28 everywhere; |up| and |silu| stay below 3 (halves of normal values), the slope of
    # silu and the weights below 1.11: 2^-28 * 3 * 1.11^2 < 2^-26
    x = x / 2
    w2[:], dout[:] = 0.0, 2.0 ** -14
    w2[:, 3] = 2.0 ** -14
    a = [t.cuda() for t in (x, ids, weights, w1, w2, dout)]
    want = [v.detach().cpu() for v in experts_in_float64(*a)]
    rel = expert_tolerance(dtype, dim, hidden, tokens * k)
    _, saved = mix.experts_forward(*a[:5])
    got = mix.experts_backward(a[5], *a[:5], saved)
    scaled = mix.experts_backward(a[5] * 2.0 ** 26, *a[:5], saved)
    for i, name in ((0, "dx"), (2, "dw1")):
        if dtype == F16:
            assert not got[i].any(), name
        else:
            near(got[i], want[i + 1], rel, name)
        near(scaled[i], want[i + 1] * 2.0 ** 26, rel, name + " of the scaled loss")
