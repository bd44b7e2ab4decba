"""The tolerance of dW whose targets' dz has back what bf16 took from it tells such a dW from one without; on the CPU, by
emulating both."""
import pytest
import torch

from tests.loss_rest_reference import RestReference, half_step_inputs


@pytest.mark.parametrize("M,V,K,same", [(1, 50, 64, 0), (20, 300, 136, 0), (64, 257, 264, 0), (65, 90, 72, 0), (300, 700, 136, 0), (300, 90, 72, 3)])
def test_tolerance_sees_the_remainder(M, V, K, same):
    hidden, head, targets, weights = half_step_inputs(M, V, K, M + V, same, device="cpu")
    if M == 1:
        targets[:], weights[:] = 7, (1.25 + 2.0 ** -8 * 0.9) / (1 - 1.0 / V)
    ref = RestReference(hidden, head, targets, weights)
    want, tol = ref.d_head_tol()
    h = torch.where(ref.kept[:, None], ref.h, 0.0)
    dz = ref.dz.float()
    coarse = dz.to(torch.bfloat16).double()
    target = torch.zeros_like(ref.dz).scatter_(1, torch.where(ref.trained, ref.t, 0)[:, None], 1.0)
    rest = ((dz.double() - coarse) * target).to(torch.bfloat16).double()
    without = (coarse.t() @ h).to(torch.bfloat16).double()
    having = ((coarse + rest).t() @ h).to(torch.bfloat16).double()
    assert bool(((having - want).abs() <= tol).all())
    far = (without - want).abs() > tol
    assert int(far.any(1).sum()) >= 0.5 * len(set(ref.t[ref.kept].tolist()))      # (of most targets' rows)
