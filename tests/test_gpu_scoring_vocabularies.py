"""Scoring at vocabularies of about 152,000 entries, and gradients of 32 bits in more rows than the second-level cache holds."""
import pytest
import torch

from test_gpu_scoring import BF16, F32, check_distill, check_logprobs, logits_of, some_ids, teacher_of, tlq, weights_of  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("v", [151936, 152064])
@pytest.mark.parametrize("n", [1, 3, 40, 500])
def test_vocabularies_of_152_thousand_entries(tlq, n, v, dtype):  # noqa: F811
    z = logits_of(n, v, dtype)
    for k, scale in ((0, 1.0), (20, 1.25), (64, 1.0)):
        check_logprobs(tlq, z, some_ids(n, v), k, scale)
    ids, top = teacher_of(z, 64)
    check_distill(tlq, z, ids, top, weights_of(n), 0.5)


@pytest.mark.parametrize("n,v", [(700, 65537), (500, 131072), (400, 151936), (900, 20011)])
def test_gradients_of_32_bits_in_many_rows(tlq, n, v):  # noqa: F811
    z = logits_of(n, v, F32)
    ids, top = teacher_of(z, 20)
    w = weights_of(n)
    _, a = check_distill(tlq, z, ids, top, w)
    buf = torch.empty(n, v + 3, device="cuda")[:, 1:1 + v]
    _, b = tlq.tlq_distill_loss(z, ids, top, w, grad=buf)
    assert torch.equal(a, b)
    _, c = tlq.tlq_distill_loss(z, ids, top, w, grad=z)
    assert torch.equal(a, c)
