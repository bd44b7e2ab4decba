"""The tolerances of the fp32 head loss's single products tell its six products of parts from any five; on the CPU, by
emulating them."""
import pytest
import torch

from tests.loss_parts_reference import SIX, Gradients, Scores, parts

DROPPED = [None] + SIX


@pytest.mark.parametrize("dropped", DROPPED, ids=str)
@pytest.mark.parametrize("M,V,K", [(12, 300, 72), (60, 1000, 72), (100, 200, 136)])
def test_five_products_are_seen(M, V, K, dropped):
    which = [p for p in SIX if p != dropped]
    big = Scores(M, V, K, M, True, device="cpu")
    (lse, loss), _ = big.emulated(which)
    small = Scores(M, V, K, M + 1, False, device="cpu")
    _, dw = small.emulated(which)
    grads = Gradients(M, V, K, M + 2, device="cpu")
    off = big.scores_off(lse, loss) + (small.head_gradient_off(dw),) + grads.off(*grads.emulated(which))
    if dropped is None:
        assert max(off) <= 1, off
    else:
        assert min(off) >= 3, off


def test_parts_sum_to_the_number():
    x = torch.randn(1000) * 2.0 ** torch.randint(-20, 20, (1000,))
    assert torch.equal(sum(parts(x)), x.double())
