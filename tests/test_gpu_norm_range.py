"""The norm where a step between its input and its codes leaves the 32-bit range although the result does not."""
import pytest
import torch

from test_gpu_norm_product import bf, check_norm, gen, tlq  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [1, 3, 700])
@pytest.mark.parametrize("c", [128, 3584, 16400, 29568, 32768])
def test_norm_of_scales_beyond_the_reciprocals_range(tlq, n, c):  # noqa: F811
    """w and s of 2^127 in the same channels: their quotient is 1, and one over s is below the smallest normal number."""
    g = gen(n + c)
    x, w, s = bf(torch.randn(n, c, generator=g)), bf(1 + 0.2 * torch.randn(c, generator=g)), bf(torch.rand(c, generator=g) + 0.5)
    w[::7] = s[::7] = 2.0 ** 127
    w[3::7], s[3::7] = -1.5 * 2.0 ** 126, -1.25 * 2.0 ** 126
    w[5::7] = s[5::7] = 2.0 ** -126
    out = tlq.tlq_norm_quantize(x, w, s=s, want_values=True)
    check_norm(tlq, out, x, None, w, s)
