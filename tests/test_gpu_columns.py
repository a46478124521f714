"""Inputs and outputs that are ranges of columns of one buffer: the results of calls whose buffers lie apart, and nothing else touched."""
import pytest
import torch

from test_gpu_norm_product import bf, gen as cpu_gen, tlq  # noqa: F401
from test_gpu_scoring import BF16, F32, logits_of, teacher_of, weights_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [1, 5, 700])
@pytest.mark.parametrize("c", [64, 1536, 3584, 16400])
def test_norm_of_columns_of_one_buffer(tlq, n, c):  # noqa: F811
    g = cpu_gen(n + c)
    x, r, w = bf(torch.randn(n, c, generator=g)), bf(torch.randn(n, c, generator=g)), bf(torch.randn(c, generator=g))
    want = tlq.tlq_norm_quantize(x, w, residual=r, want_values=True)
    for places in ((0, 1, 2), (2, 0, 1), (1, 2, 0)):
        for over in (None, 0, 1):                       # the sum beside both, or over one of them
            buf = torch.full((n, 3 * c + 8), 3.0, dtype=BF16, device="cuda")
            x1, r1, h1 = (buf[:, k * c:(k + 1) * c] for k in places)
            x1.copy_(x)
            r1.copy_(r)
            out = tlq.tlq_norm_quantize(x1, w, residual=r1, h=(h1, x1, r1)[0 if over is None else 1 + over], want_values=True)
            for name in ("h", "codes", "steps", "values"):
                assert torch.equal(out[name], want[name]), name
            assert torch.all(buf[:, 3 * c:] == 3)
            assert over == 0 or torch.equal(x1, x)
            assert over == 1 or torch.equal(r1, r)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,v,pitch,at,to", [(7, 1001, 2002, 0, 1001), (7, 1001, 2005, 1003, 1), (600, 20011, 40030, 3, 20015), (40, 65537, 131074, 65537, 0),
                                             (3, 262147, 524295, 0, 262148), (1, 1000, 2000, 0, 1000), (300, 50000, 100000, 0, 50000)])
def test_gradient_in_columns_beside_the_logits(tlq, n, v, pitch, at, to, dtype):  # noqa: F811
    z = torch.empty(n, pitch, dtype=dtype, device="cuda")[:, at:at + v]       # (as they lie on the memory's grid, so they are added up)
    z.copy_(logits_of(n, v, dtype))
    ids, top = teacher_of(z, 20)
    w = weights_of(n)
    loss, want = tlq.tlq_distill_loss(z, ids, top, w)
    buf = torch.full((n, pitch), 5.0, dtype=dtype, device="cuda")
    z1, g1 = buf[:, at:at + v], buf[:, to:to + v]
    z1.copy_(z)
    got, grad = tlq.tlq_distill_loss(z1, ids, top, w, grad=g1)
    assert grad is g1 and torch.equal(got, loss) and torch.equal(g1, want) and torch.equal(z1, z)
    rest = torch.ones(pitch, dtype=torch.bool, device="cuda")
    rest[at:at + v] = rest[to:to + v] = False
    assert torch.all(buf[:, rest] == 5)
