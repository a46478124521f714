"""A teacher's alternatives handed on to the distillation loss at temperatures other than 1."""
import pytest
import torch

from test_gpu_scoring import BF16, F32, distill_ref, logits_of, slack, tlq, weights_of  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("scale", [0.5, 1.25, 4.0])
@pytest.mark.parametrize("v", [1000, 50001])
def test_alternatives_at_scale_one_are_the_teacher_at_any_temperature(tlq, v, scale, dtype):  # noqa: F811
    """The teacher's log probabilities are its logits less a constant, each off by the slack of a logarithm and 2^-22 of itself: so p is off by
    twice that times scale, relative, and the loss by that of its terms, beside what the loss itself is off by."""
    from paper_2602_07899_b200 import calibrate
    n, k = 33, 20
    z, teacher, w = logits_of(n, v, dtype), logits_of(n, v, F32, seed=1), weights_of(n)
    best = tlq.tlq_token_logprobs(teacher, None, k)
    ids = best["top_ids"]
    loss, grad, size, mag = distill_ref(z, ids, teacher.gather(1, ids.long()), w, scale)
    off = 2 * scale * (slack(v) + 2.0 ** -22 * best["top_logp"].double().abs().amax(1))
    got, g = tlq.tlq_distill_loss(z, ids, best["top_logp"], w, scale)
    most = 4 * slack(v)
    weight = w.double().abs()
    assert torch.all((got.double() - loss).abs() <= (most + 2 * off) * (mag + weight) + 2.0 ** -23 * loss.abs())
    half = 2.0 ** -8 if dtype == BF16 else 2.0 ** -24
    room = (most + 2 * off)[:, None] * size
    # exponentials below the smallest normal number, 2^-126, are 0, which takes w scale / S of it from the gradient, with S >= 1: logits that are
    # 30 apart are 4 log2(e) 30 = 173 powers of 2 apart at scale 4
    least = (2.0 ** -126 * (1 + weight * scale))[:, None]
    assert torch.all((g.double() - grad).abs() <= half * (grad.abs() + room) + room + least)
    imp, _, same = calibrate.importance_from_teacher(z, ids, best["top_logp"], w, scale)
    assert torch.all((same - got).abs() <= 2 * (most * (mag + weight) + 2.0 ** -23 * loss.abs()))
    norm = g.double().norm(dim=1)
    assert torch.all((imp.double() - norm).abs() <= 1e-5 * norm)


@pytest.mark.parametrize("scale", [0.5, 2.0])
def test_alternatives_at_a_scale_are_flattened_once_more(tlq, scale):  # noqa: F811
    """What they are taken at is in them, and the loss multiplies by its own: both together are the teacher at the product."""
    n, v, k = 20, 4096, 20
    z, teacher = logits_of(n, v, F32), logits_of(n, v, F32, seed=1)
    best = tlq.tlq_token_logprobs(teacher, None, k, scale)
    ids = best["top_ids"]
    loss, _, _, mag = distill_ref(z, ids, scale * teacher.double().gather(1, ids.long()), None, scale)
    off = 2 * scale * (slack(v) + 2.0 ** -22 * best["top_logp"].double().abs().amax(1))
    got, _ = tlq.tlq_distill_loss(z, ids, best["top_logp"], None, scale, want_grad=False)
    assert torch.all((got.double() - loss).abs() <= (4 * slack(v) + 2 * off) * (mag + 1) + 2.0 ** -23 * loss.abs())
