"""The 8-bit product with an activation of sums beyond the 32-bit range and of infinite biases: +infinity stays what it is, -infinity is no
number where an activation would multiply it by 0, and large finite sums go where the activation sends them."""
import math

import pytest
import torch

from test_gpu_norm_product import bf, gen, tlq  # noqa: F401

pytestmark = pytest.mark.gpu

INF = math.inf


def sums(n, co, size):
    """Codes whose products are 100 * 100 * 64 = 640000 for even, -640000 for odd channels, times steps to `size`."""
    xq = torch.full((n, 64), 100, dtype=torch.int8, device="cuda")
    wq = torch.full((co, 64), 100, dtype=torch.int8, device="cuda")
    wq[1::2] = -100
    return xq, torch.full((n,), 1e3, device="cuda"), wq, torch.full((co,), size / 640000 / 1e3, device="cuda")


@pytest.mark.parametrize("n", [1, 12, 30, 300, 2100])
@pytest.mark.parametrize("act", [0, 1, 2, 3])
def test_infinite_sums(tlq, n, act):  # noqa: F811
    co = 4096 if n > 1000 else 64
    xq, t, wq, u = sums(n, co, 1.0)
    bias = bf(torch.randn(co, generator=gen(n)))
    clean = tlq.tlq_linear_i8_act(xq, t, wq, u, bias, act).float()
    bias[3::8], bias[5::8] = INF, -INF
    y = tlq.tlq_linear_i8_act(xq, t, wq, u, bias, act).float()
    assert torch.all(y[:, 3::8] == INF)
    assert torch.all(y[:, 5::8] == -INF) if act == 0 else torch.isnan(y[:, 5::8]).all()
    keep = torch.ones(co, dtype=torch.bool, device="cuda")
    keep[3::8] = keep[5::8] = False
    assert torch.equal(y[:, keep], clean[:, keep])


@pytest.mark.parametrize("n", [1, 12, 30, 300, 2100])
@pytest.mark.parametrize("act", [1, 2, 3])
def test_sums_beyond_the_range(tlq, n, act):  # noqa: F811
    """The product of the steps and the sum is infinite: 640000 times 1e3 times 1e35; and just not, at 3e38."""
    co = 4096 if n > 1000 else 64
    xq, t, wq, u = sums(n, co, 1.0)
    y = tlq.tlq_linear_i8_act(xq, t, wq, torch.full_like(u, 1e35), act=act).float()
    assert torch.all(y[:, ::2] == INF) and torch.isnan(y[:, 1::2]).all()
    y = tlq.tlq_linear_i8_act(xq, t, wq, torch.full_like(u, 3e38 / 640000 / 1e3), act=act).float()
    assert torch.all((y[:, ::2] - 3e38).abs() <= 2.0 ** -7 * 3e38) and torch.all(y[:, 1::2] == 0)


@pytest.mark.parametrize("n", [1, 12, 30, 300, 2100])
@pytest.mark.parametrize("act", [1, 2, 3])
def test_infinite_gates(tlq, n, act):  # noqa: F811
    """Gate +infinity: the up projection's sign decides, and 0 makes no number of it; a NaN stays one."""
    co = 4096 if n > 1000 else 64
    xq, t, wq, u = sums(n, co, 1.0)
    wq[1::4], wq[3::8] = 100, 0                         # up: 1, then alternately 0 and -1
    bias = torch.zeros(co, dtype=torch.bfloat16, device="cuda")
    bias[::2] = INF
    y = tlq.tlq_linear_i8_act(xq, t, wq, u, bias, act, True).float()
    assert torch.all(y[:, ::2] == INF) and torch.isnan(y[:, 1::4]).all() and torch.all(y[:, 3::4] == -INF)
    bias[::2] = math.nan
    assert torch.isnan(tlq.tlq_linear_i8_act(xq, t, wq, u, bias, act, True).float()).all()
    assert torch.isnan(tlq.tlq_linear_i8_act(xq, t, wq, u, bias, act).float()[:, ::2]).all()
