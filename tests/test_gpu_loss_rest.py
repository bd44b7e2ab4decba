"""dW of bf16 rows: what rounding takes from a row's dz at its target comes back, for every tile and for many rows of one
target."""
import pytest

from tests.parity import say

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
from tests.loss_rest_reference import RestReference, half_step_inputs  # noqa: E402


# up to 64 rows; then tiles of 128 x 64, 256 x 64, 256 x 128 and 256 x 256, more rows than a block lists at a time (1024 or
# 2048), and the vocabulary in pieces
@pytest.mark.parametrize("same", [0, 3], ids=["spread", "same"])
@pytest.mark.parametrize("M,V,K", [(1, 50, 64), (3, 40, 72), (20, 300, 136), (33, 1000, 520), (64, 257, 264), (65, 90, 72), (130, 700, 136), (1500, 300, 264),
                                   (66, 64, 16384), (70, 120, 16384), (100, 4096, 1032), (4500, 4200, 1024), (3000, 40001, 64)])
def test_remainders(M, V, K, same):
    from paper_2606_03113_amd import lede
    say("head loss, dW's remainders M=%d V=%d K=%d same=%d" % (M, V, K, same))
    hidden, head, targets, weights = half_step_inputs(M, V, K, M + V, same)
    if M == 1:
        targets[:], weights[:] = 7, (1.25 + 2.0 ** -8 * 0.9) / (1 - 1.0 / V)
    bad = hidden.clone()
    bad[(targets < 0) | (targets >= V) | (weights == 0)] = float("nan")     # rows left out
    lse = lede.op_head_loss(bad, head, targets).lse
    dw = lede.op_head_loss_grad(bad, head, targets, lse, weights, want_hidden=False)[1]
    want, tol = RestReference(hidden, head, targets, weights).d_head_tol()
    off = (dw.double() - want).abs()
    assert bool((off <= tol).all()), (float((off / tol).max()), (off > tol).nonzero()[:4].tolist())
    again = lede.op_head_loss_grad(bad, head, targets, lse, weights)[1]
    assert torch.equal(again, dw)
