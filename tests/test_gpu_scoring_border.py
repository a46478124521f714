"""Rows whose logits lie on both sides of |scale log2(e) z| = 2^31, where the factor of a logit changes: log probabilities and distillation
against their definitions in 64 bits, with the tolerances of test_gpu_scoring (whose terms for arguments of up to 64 these rows reach)."""
import math

import pytest
import torch

from test_gpu_scoring import BF16, F32, check_distill, check_logprobs, some_ids, teacher_of, tlq  # noqa: F401

pytestmark = pytest.mark.gpu


def straddling(v, dtype, scale):
    """Rows of a below and b above the border, in all orders and both signs: side by side, far apart, batch after batch of a thread."""
    border = 2.0 ** 31 / (scale * math.log2(math.e))
    a, b = (torch.tensor(f * border, dtype=dtype).item() for f in (0.8, 1.1))
    assert a < border < b
    i = torch.arange(v, device="cuda")

    def where(mask, x, y):
        return torch.where(mask, torch.tensor(x, dtype=torch.float64, device="cuda"), torch.tensor(y, dtype=torch.float64, device="cuda"))
    rows = []
    for mask in (i == v - 1, i == v // 2, i % 7 == 3, i == 0, i // 512 % 2 == 1, i // 4096 % 2 == 1, i >= v // 2, i < v // 2):
        rows += [where(mask, b, a), where(mask, -a, -b), where(mask, b, -b), where(mask, a, -b)]
    ramp = (0.5 + i.double() / v) * border
    rows += [ramp, ramp.flip(0), -ramp, -ramp.flip(0)]
    z = torch.stack(rows).to(dtype)
    if dtype == F32:                # neighbours of 32 bits at the border itself
        low = torch.tensor(border, dtype=F32)
        low = low if low.item() * torch.tensor(scale * math.log2(math.e), dtype=F32).item() < 2.0 ** 31 else torch.nextafter(low, torch.tensor(0.0))
        high = torch.nextafter(low, torch.tensor(math.inf))
        near = torch.full((4, v), low.item(), dtype=F32, device="cuda")
        near[0, v - 1] = near[1, v // 2:] = high.item()
        near[2:] = -near[:2]
        z = torch.cat((z, near))
    return z


@pytest.mark.parametrize("scale", [1.0, 1.25, 0.5, 1000.0, 2.0 ** 16, 2.0 ** -16])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("v", [9, 1000, 16391, 131072])
def test_rows_on_both_sides_of_the_border(tlq, v, dtype, scale):  # noqa: F811
    z = straddling(v, dtype, scale)
    check_logprobs(tlq, z, some_ids(len(z), v), 5, scale)
    check_logprobs(tlq, z[:3], None, 0, scale)                       # few rows: several CTAs to one
    ids, top = teacher_of(z, 5)
    check_distill(tlq, z, ids, top, None, scale)
    check_distill(tlq, z[4:7].contiguous(), ids[4:7].contiguous(), top[4:7].contiguous(), None, scale)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_the_surest_token_beyond_the_border_is_certain(tlq, dtype):  # noqa: F811
    z = torch.full((400, 40000), 1.2e9, dtype=dtype, device="cuda")
    at = (torch.arange(400, device="cuda") * 977 % 40000).to(torch.int32)
    z[torch.arange(400, device="cuda"), at.long()] = 1.6e9
    out = tlq.tlq_token_logprobs(z, at, 1, want_entropy=True, want_lse=True)
    assert torch.all(out["logp"] == 0) and torch.all(out["entropy"] == 0) and torch.equal(out["top_ids"][:, 0], at)
    assert torch.equal(out["lse"], torch.full_like(out["lse"], torch.tensor(1.6e9, dtype=dtype).item()))
    loss, grad = tlq.tlq_distill_loss(z, at[:, None].contiguous(), torch.zeros(400, 1, device="cuda"))
    assert torch.all(loss == 0) and torch.all(grad == 0)
