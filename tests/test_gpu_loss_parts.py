"""The six products of parts that fp32 inputs of the head loss are multiplied by, one result at a time, in every tile."""
import pytest

from tests.parity import say

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
from tests.loss_parts_reference import Gradients, Scores  # noqa: E402

# thin tiles of 64 and 128 entries by 16, 32 and 64 rows; 64 x 128 and 128 x 128
LOGITS = [(1, 1, 8), (5, 2, 8), (12, 3000, 72), (30, 9000, 136), (60, 9000, 72), (12, 65500, 40), (30, 65500, 72), (60, 65500, 72), (100, 8200, 136), (200, 8200, 264)]


@pytest.mark.parametrize("M,V,K", LOGITS)
def test_logits(M, V, K):
    from paper_2606_03113_amd import lede
    say("head loss, parts M=%d V=%d K=%d" % (M, V, K))
    s = Scores(M, V, K, M + V, True)
    r = lede.op_head_loss(s.hidden, s.head, s.targets)
    off = s.scores_off(r.lse, r.loss)
    assert max(off) <= 1, off


@pytest.mark.parametrize("M,V,K", LOGITS)
def test_logits_in_the_gradient(M, V, K):
    from paper_2606_03113_amd import lede
    say("head loss, parts in dz M=%d V=%d K=%d" % (M, V, K))
    s = Scores(M, V, K, M + V, False)
    _, dw = lede.op_head_loss_grad(s.hidden, s.head, s.targets, s.lse.float(), s.weights, want_hidden=False)
    off = s.head_gradient_off(dw[:, s.at].t())
    assert off <= 1, off


# dW: up to 32 rows, 64 x 64, 64 x 128 and 128 x 128; dh: 256 x 16, 32 and 64, 64 x 64, 64 x 128 and 128 x 128
@pytest.mark.parametrize("M,V,K", [(1, 2, 8), (20, 700, 136), (40, 60, 264), (100, 700, 264), (200, 8200, 1032), (12, 33000, 264), (30, 33000, 264), (60, 33000, 264)])
def test_gradients(M, V, K):
    from paper_2606_03113_amd import lede
    say("head loss, parts in the gradients M=%d V=%d K=%d" % (M, V, K))
    s = Gradients(M, V, K, M + V)
    lse = lede.op_head_loss(s.hidden, s.head, s.targets).lse
    assert bool(((lse - 512).abs() <= 2.0 ** -14).all())
    dh, dw = lede.op_head_loss_grad(s.hidden, s.head, s.targets, s.lse, s.weights)
    off = s.off(dh[:, s.columns], dw[s.targets.long()])
    assert max(off) <= 1, off
    rest = torch.ones(V, dtype=torch.bool, device="cuda")
    rest[s.targets.long()], rest[V - 1] = False, False
    assert not bool(dw[rest].any())
