"""The norm where a step between its input and its codes leaves the 32-bit range although the result does not."""
import math

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


@pytest.mark.parametrize("n", [1, 5, 700])
@pytest.mark.parametrize("c", [128, 1536, 3584, 8192, 16400, 29568])
@pytest.mark.parametrize("size", [16.0, 1000.0, 1e15, 1e38])
def test_norm_whose_input_times_its_weight_leaves_the_range(tlq, n, c, size):  # noqa: F811
    """|h w / s| is infinite where the norm times w / s is not.  (Of evenly spread values, a ninth of them almost 0, the mean of the squares is
    8/27 of the largest, and half of that at least over 128 of them: no value is above 2.6 of the root.)"""
    g = gen(c)
    x = bf((torch.rand(n, c, generator=g) * 2 - 1) * size)
    x[:, ::9] *= 2.0 ** -60                              # some that round to 0
    for w, s in ((2.0 ** 126, None), (None, 2.0 ** -126), (2.0 ** 64, 2.0 ** -61)):
        w = None if w is None else bf(torch.full((c,), w))
        s = None if s is None else bf(torch.full((c,), s))
        for bits in (2, 8):
            out = tlq.tlq_norm_quantize(x, w, tlq.config(tlq.W8A8_SYM, a_bits=bits), s=s, want_values=True, want_y=True)
            check_norm(tlq, out, x, None, w, s, bits=bits)
            assert torch.all(out["codes"].abs().amax(1) == 2 ** (bits - 1) - 1)


def test_norm_that_leaves_the_range_itself_is_no_number(tlq):  # noqa: F811
    x = bf(torch.rand(300, 1536, generator=gen(1)) + 1)
    x[::2] = bf(torch.rand(150, 1536, generator=gen(2)) + 1) * 0.0
    x[::2, 7] = 1e5                                      # all of the row's energy in one channel: sqrt(1536) 2^126
    out = tlq.tlq_norm_quantize(x, bf(torch.full((1536,), 2.0 ** 126)), want_values=True)
    assert torch.isnan(out["steps"][::2]).all() and torch.all(out["codes"][::2] == 0) and torch.isnan(out["values"][::2].float()).all()
    assert torch.isfinite(out["steps"][1::2]).all() and torch.all(out["codes"][1::2].abs().amax(1) == 127)
    bad = x[1::2].clone()
    bad[4, 5], bad[9, 0] = math.nan, math.inf
    out = tlq.tlq_norm_quantize(bad, bf(torch.full((1536,), 2.0 ** 126)), want_values=True)
    assert torch.isnan(out["steps"][[4, 9]]).all() and torch.isfinite(out["steps"][[3, 5, 8, 10]]).all()
