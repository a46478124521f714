"""Importance of tokens from a teacher over vocabularies that are no multiple of a 16-byte piece, in memory that held something else."""
import pytest
import torch

from test_gpu_scoring import BF16, F32, logits_of, teacher_of, tlq, weights_of  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,v", [(1, 1), (60, 7), (60, 4093), (300, 50001)])
def test_importance_in_used_memory(tlq, n, v, dtype):  # noqa: F811
    from paper_2602_07899_b200 import calibrate
    z, w = logits_of(n, v, dtype), weights_of(n)
    ids, top = teacher_of(z, min(v, 5))
    _, grad = tlq.tlq_distill_loss(z, ids, top, w)
    for kind, norm in ((tlq.NORM_L2, grad.double().norm(dim=1)), (tlq.NORM_MEAN_ABS, grad.double().abs().mean(1))):
        used = [torch.full((n, -(-v // 8) * 8), float("nan"), dtype=dtype, device="cuda") for _ in range(4)]
        del used                    # (what is made next of this size comes to lie there)
        imp, _, _ = calibrate.importance_from_teacher(z, ids, top, w, norm_kind=kind, top_frac=1.0)
        assert torch.all((imp.double() - norm).abs() <= 1e-5 * norm)          # (an fp32 result of fp64 sums of fp32 parts)
