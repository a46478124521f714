"""The norm's eps is a normal number: squares of 32 bits that are beside a smaller one, but below the normal numbers themselves, would be lost."""
import ctypes
import math

import pytest
import torch

import __graft_entry__ as entry


def test_norm_refuses_an_eps_below_the_normal_numbers():
    entry.build()
    from paper_2602_07899_b200 import tlq
    buf = (ctypes.c_uint8 * (1 << 16))()
    a = (ctypes.addressof(buf) + 255) // 256 * 256
    cfg = tlq.config(tlq.W8A8_SYM)

    def call(eps, codes=a + 4096, steps=a + 8192, y=None):
        return tlq.lib.tlq_norm_quantize(a, 4, 64, 64, None, 0, None, eps, None, ctypes.byref(cfg), None, 0, codes, steps, None, y, None)

    for eps in (2.0 ** -149, 1e-40, 2.0 ** -126 * (1 - 2.0 ** -20), 0.0, -1e-6, math.nan, math.inf):
        assert call(eps) == tlq.ERR_INVALID_ARG, eps
        assert call(eps, None, None, a + 4096) == tlq.ERR_INVALID_ARG, eps
    if not torch.cuda.is_available():
        for eps in (2.0 ** -126, 1e-12, 1e-5, 1e30):
            assert call(eps) == tlq.ERR_CUDA, eps


@pytest.mark.gpu
@pytest.mark.parametrize("c", [128, 3584, 29568])
def test_norm_of_small_numbers_with_the_smallest_eps(c):
    """Squares that are lost are below 2^-149, so the mean is off by 2^-23 of such an eps, and the root by half of that."""
    from paper_2602_07899_b200 import tlq
    eps = 2.0 ** -126
    g = torch.Generator().manual_seed(c)
    for n, size in ((3, 2.0 ** -63), (700, 2.0 ** -66), (3, 2.0 ** -72), (3, 3.0)):
        x = (torch.randn(n, c, generator=g) * size).bfloat16().cuda()
        y = tlq.tlq_norm_quantize(x, None, eps=eps, want_y=True, want_codes=False)["y"].double()
        want = x.double() / ((x.double() ** 2).mean(1, keepdim=True) + eps).sqrt()
        assert torch.all((y - want).abs() <= (2.0 ** -8 * (1 + 2.0 ** -7) + 2.0 ** -19) * want.abs())
