"""The head loss's gradient against differences of its losses, along lines where a wrong gradient shows."""
import pytest

from tests.parity import say

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
from tests.loss_differences import Line  # noqa: E402


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("which", [0, 1], ids=["hidden", "head"])
@pytest.mark.parametrize("M,V,K", [(60, 400, 128), (30, 1000, 72), (130, 700, 136)])
def test_gradient_against_differences(M, V, K, which, dtype):
    from paper_2606_03113_amd import lede
    for seed in (1, 2, 3):
        line = Line(which, dtype, seed, M, V, K)
        assert abs(line.rise) >= 20 * line.allowed, (line.rise, line.allowed)
        losses = [lede.op_head_loss(*line.at(e), line.targets).loss for e in line.ends]
        lse = lede.op_head_loss(*line.middle, line.targets).lse
        gradient = lede.op_head_loss_grad(*line.middle, line.targets, lse, line.weights)[which]
        off = line.off(losses, gradient)
        say("rise %g, off by %g of %g allowed" % (line.rise, off, line.allowed))
        assert off <= line.allowed
