"""A single row of hidden, of the head or of a gradient may lie in rows of any length: its stride leads nowhere."""
import pytest

from tests.parity import say

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
from tests.loss_reference import inputs  # noqa: E402


def single(x, stride):
    """x [1][K] with this row stride."""
    return x.contiguous().as_strided(x.shape, (stride, 1))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("stride", [75, 1 << 22, 1 << 40])
@pytest.mark.parametrize("M,V", [(1, 300), (5, 1), (1, 1), (70, 1), (1, 70000)])
def test_stride_of_one_row(M, V, stride, dtype):
    from paper_2606_03113_amd import lede
    say("head loss, M=%d V=%d, stride %d" % (M, V, stride))
    hidden, head, _, weights = inputs(M, V, 72, dtype, 5)
    targets = (torch.arange(M, device="cuda") % V).int()
    want = lede.op_head_loss(hidden, head, targets)
    grads = lede.op_head_loss_grad(hidden, head, targets, want.lse, weights)
    out = [torch.empty_like(x) for x in grads]
    h, dh = (single(hidden, stride), single(out[0], stride)) if M == 1 else (hidden, out[0])
    w, dw = (single(head, stride), single(out[1], stride)) if V == 1 else (head, out[1])
    got = lede.op_head_loss(h, w, targets)
    assert torch.equal(got.loss, want.loss) and torch.equal(got.lse, want.lse)
    lede.op_head_loss_grad(h, w, targets, got.lse, weights, out=(dh, dw))
    assert torch.equal(dh, grads[0]) and torch.equal(dw, grads[1])


def test_what_is_still_refused():
    from paper_2606_03113_amd import lede
    hidden, head, targets, _ = inputs(1, 50, 72, torch.float32, 5)
    room = torch.zeros(2, 76, device="cuda")
    for h, w in ((room[:1, 1:73], head), (hidden, torch.zeros(50, 75, device="cuda")[:, :72])):     # not 16-byte aligned; rows that are not
        with pytest.raises(lede.LedeError):
            lede.op_head_loss(h, w, targets)
