"""Tokens so far below the surest one that the distance in powers of 2, but not the log probability, leaves the 32-bit range."""
import pytest
import torch

from test_gpu_scoring import BF16, F32, check_distill, check_logprobs, tlq  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("v", [9, 1000, 131072])
@pytest.mark.parametrize("scale,top", [(1.0, 3e38), (0.5, 3.3e38), (2.0 ** -16, 3.3e38), (1.0, 2.5e38)])
def test_log_probabilities_of_tokens_far_below_the_surest(tlq, v, dtype, scale, top):  # noqa: F811
    z = torch.randn(4, v, generator=torch.Generator(device="cuda").manual_seed(v), device="cuda").to(dtype)
    z[0, 5] = z[1, 1::2] = z[2, v - 1] = z[3] = top
    z[2, :4] = -1e30
    ids = torch.tensor([0, 0, 1, 2], dtype=torch.int32, device="cuda")
    out = check_logprobs(tlq, z, ids, 8, scale)
    assert torch.isfinite(out["logp"]).all()
    check_distill(tlq, z, ids[:, None].contiguous(), torch.zeros(4, 1, device="cuda"), None, scale)
