"""Which buffers lie over one another: ranges of columns of one allocation do not, whatever their pitch spans.  All on the host."""
import ctypes

import pytest
import torch

import __graft_entry__ as entry


@pytest.fixture(scope="module")
def tlq():
    entry.build()
    from paper_2602_07899_b200 import tlq as mod
    return mod


@pytest.fixture(scope="module")
def addr():
    buf = (ctypes.c_uint8 * (1 << 20))()
    addr.keep = buf
    return (ctypes.addressof(buf) + 255) // 256 * 256


def taken(tlq, call, **args):
    """Refused for nothing but that there is no device (and not called where there is one)."""
    if not torch.cuda.is_available():
        assert call(**args) == tlq.ERR_CUDA, args


def test_norm_of_columns_of_one_buffer(tlq, addr):
    a, good, far = addr, tlq.config(tlq.W8A8_SYM), addr + (1 << 19)

    def call(x=a, n=4, c=64, ldx=64, r=None, ldr=0, h=None, ldh=0, codes=far, steps=far + 8192, values=None):
        return tlq.lib.tlq_norm_quantize(x, n, c, ldx, r, ldr, None, 1e-6, None, ctypes.byref(good), h, ldh, codes, steps, values, None, None)

    # rows of 3 x 64 channels: 128 bytes each, 384 apart
    for fine in (dict(ldx=192, h=a + 128, ldh=192), dict(x=a + 128, ldx=192, h=a, ldh=192), dict(x=a + 256, ldx=192, h=a + 128, ldh=192),
                 dict(ldx=192, r=a + 128, ldr=192, h=a + 256, ldh=192), dict(ldx=192, r=a + 128, ldr=192, h=a, ldh=192),
                 dict(ldx=192, r=a + 128, ldr=192, h=a + 128, ldh=192), dict(ldx=192, h=a + 384 + 128, ldh=192), dict(x=a + 384 * 2, ldx=192, h=a + 128, ldh=192),
                 dict(n=1, ldx=192, h=a, ldh=64), dict(n=1, h=a, ldh=1024), dict(n=1, r=a + 128, ldr=64, ldx=192, h=a + 128, ldh=192)):
        taken(tlq, call, **fine)
    for bad in (dict(ldx=192, h=a + 112, ldh=192), dict(ldx=192, h=a + 16, ldh=192), dict(ldx=192, h=a + 384, ldh=192), dict(ldx=192, h=a + 272, ldh=192),
                dict(x=a + 128, ldx=192, h=a + 16, ldh=192), dict(ldx=192, h=a + 128, ldh=200), dict(ldx=192, r=a + 128, ldr=192, h=a + 64, ldh=192),
                dict(ldx=192, codes=a + 128), dict(ldx=64, h=a + 512 - 16, ldh=64), dict(n=1, ldx=192, h=a + 16, ldh=64)):
        assert call(**bad) == tlq.ERR_INVALID_ARG, bad
    # (nothing of such a size is in one place: no number of bytes may run over)
    assert call(n=0x7FFFFF00, ldx=1 << 40, r=a, ldr=1 << 40, h=a + 16, ldh=1 << 40) == tlq.ERR_INVALID_ARG
    assert call(n=0x7FFFFF00, ldx=1 << 40, h=a + 128, ldh=1 << 39, codes=None, steps=None) == tlq.ERR_INVALID_ARG


def test_product_with_a_residual_of_one_row(tlq, addr):
    a, far = addr, addr + (1 << 19)

    def call(n=4, co=8, res=None, ldr=0, y=a):
        return tlq.lib.tlq_linear_i8_act(far, far, n, 64, far, far, co, None, 1, 0, res, ldr, far, 1 << 30, y, None)

    for fine in (dict(res=a, ldr=8), dict(n=1, res=a, ldr=8), dict(n=1, res=a, ldr=4096), dict(n=1, res=a + 16, ldr=8)):
        taken(tlq, call, **fine)
    for bad in (dict(res=a, ldr=16), dict(n=1, res=a + 2, ldr=8), dict(res=a + 16, ldr=8)):
        assert call(**bad) == tlq.ERR_INVALID_ARG, bad


@pytest.mark.parametrize("dt,size", [(0, 2), (1, 4)])
def test_gradient_in_columns_beside_the_logits(tlq, addr, dt, size):
    a, far = addr, addr + (1 << 19)

    def call(z=a, n=4, v=100, ld=100, grad=None, ldg=0, loss=far + 8192):
        return tlq.lib.tlq_distill_loss(z, dt, n, v, ld, 1.0, far, far, 5, None, loss, grad, ldg, None)

    for fine in (dict(ld=200, grad=a + 100 * size, ldg=200), dict(z=a + 100 * size, ld=200, grad=a, ldg=200), dict(ld=203, grad=a + 101 * size, ldg=203),
                 dict(ld=203, grad=a + 103 * size, ldg=203), dict(z=a + 101 * size, ld=203, grad=a, ldg=203), dict(n=1, ld=200, grad=a, ldg=100)):
        taken(tlq, call, **fine)
    for bad in (dict(ld=200, grad=a + 99 * size, ldg=200), dict(ld=200, grad=a + 101 * size, ldg=200), dict(ld=203, grad=a + 104 * size, ldg=203),
                dict(ld=200, grad=a, ldg=201), dict(ld=200, loss=a + 100 * size), dict(n=1, ld=200, grad=a + size, ldg=100)):
        assert call(**bad) == tlq.ERR_INVALID_ARG, bad
