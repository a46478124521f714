"""Rows whose largest logit, multiplied by scale, is the last or the first outside of the 32-bit range: the former have a distribution, the
latter are no numbers."""
import math

import pytest
import torch

from test_gpu_scoring import BF16, F32, check_distill, check_logprobs, slack, some_ids, teacher_of, tlq  # noqa: F401

pytestmark = pytest.mark.gpu


def rows_with(top, v, dtype):
    z = torch.randn(5, v, generator=torch.Generator(device="cuda").manual_seed(v), device="cuda").to(dtype)
    z[0, v // 2] = top
    z[1] = top
    z[2] = -math.inf
    z[2, v - 1] = top
    z[3, ::3] = top
    z[4] = -1
    z[4, :2] = top
    return z


def below(limit, dtype):
    """The largest number of the type that is smaller."""
    x = torch.tensor(limit, dtype=torch.float64).to(dtype)
    return (x if x.item() < limit else torch.nextafter(x, torch.zeros((), dtype=dtype))).item()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("v", [9, 1000, 50001, 131072])
@pytest.mark.parametrize("scale", [1.0, 1.25, 1.3, 1.5, 1.999, 2.0, 1000.0, 2.0 ** 16])
def test_rows_up_to_the_end_of_the_range_have_a_distribution(tlq, v, dtype, scale):  # noqa: F811
    exact = torch.tensor(scale, dtype=F32).item()
    top = below((2.0 ** 128 - 2.0 ** 103) / exact, dtype)        # from there on a product is rounded to infinity
    assert top * exact < 2.0 ** 128
    z = rows_with(top, v, dtype)
    check_logprobs(tlq, z, some_ids(5, v), 5, exact)
    ids, _ = teacher_of(z / 4, 4)
    check_distill(tlq, z, ids, torch.zeros(5, 4, device="cuda"), None, exact)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("v", [9, 1000, 50001, 131072])
@pytest.mark.parametrize("scale,top", [(1.25, 3e38), (1.3, 3e38), (1.5, 3e38), (2.0, 2e38), (1000.0, 1e36), (2.0 ** 16, 6e33)])
def test_rows_that_leave_the_range_have_none(tlq, v, dtype, scale, top):  # noqa: F811
    z = rows_with(top, v, dtype)
    clean = torch.randn(5, v, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(dtype)
    both = torch.stack((z, clean), 1).flatten(0, 1)
    out = tlq.tlq_token_logprobs(both, torch.zeros(10, dtype=torch.int32, device="cuda"), 3, scale, want_entropy=True, want_lse=True)
    want = tlq.tlq_token_logprobs(clean, torch.zeros(5, dtype=torch.int32, device="cuda"), 3, scale, want_entropy=True, want_lse=True)
    for name in ("logp", "entropy", "lse", "top_logp"):
        assert torch.isnan(out[name][::2]).all(), name
        # (another number of CTAs to a row: either within its bound)
        assert torch.all((out[name][1::2] - want[name]).abs() <= 2 * slack(v) + 2.0 ** -21 * want[name].abs()), name
    assert torch.all(out["top_ids"][::2] == -1) and torch.equal(out["top_ids"][1::2], want["top_ids"])
    ids = torch.zeros(10, 1, dtype=torch.int32, device="cuda")
    teacher = torch.zeros(10, 1, device="cuda")
    loss, grad = tlq.tlq_distill_loss(both, ids, teacher, None, scale)
    assert torch.isnan(loss[::2]).all() and torch.isnan(grad[::2].float()).all()
    assert torch.isfinite(loss[1::2]).all() and torch.isfinite(grad[1::2].float()).all()
    alone, _ = tlq.tlq_distill_loss(both, ids, teacher, None, scale, want_grad=False)
    assert torch.isnan(alone[::2]).all() and torch.isfinite(alone[1::2]).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("v", [9, 1000, 16391, 131072])
@pytest.mark.parametrize("scale", [1.0, 1.3, 2.0 ** 16])
def test_rows_in_the_last_powers_of_two_of_the_range(tlq, v, dtype, scale):  # noqa: F811
    """Logits on both sides of where a power of 2 above scale log2(e) times them leaves the range, in every order."""
    exact = torch.tensor(scale, dtype=F32).item()
    a, b, c = (torch.tensor(f * 2.0 ** 128 / exact, dtype=dtype).item() for f in (0.3, 0.6, 0.98))
    i = torch.arange(v, device="cuda")
    z = torch.empty(10, v, dtype=torch.float64, device="cuda")
    z[0], z[1], z[2], z[3], z[4] = a, a, b, b, c
    z[0, v - 1], z[1, ::5], z[2, v // 2], z[3, 1::3] = b, c, c, a
    z[5] = torch.where(i < v // 2, a, c)
    z[6] = torch.where(i < v // 2, c, a)
    z[7] = (0.1 + 0.85 * i.double() / v) * 2.0 ** 128 / exact
    z[8] = z[7].flip(0)
    z[9] = -1
    z[9, v // 3] = c
    z = z.to(dtype)
    check_logprobs(tlq, z, some_ids(10, v), 5, exact)
    ids, _ = teacher_of(z / 4, 4)
    check_distill(tlq, z, ids, torch.zeros(10, 4, device="cuda"), None, exact)
