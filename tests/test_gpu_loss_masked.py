"""Vocabularies masked by infinite entries of the head: both types leave the masked entries out and keep the others."""
import pytest

from tests.parity import say

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
from tests.loss_reference import Reference, inputs  # noqa: E402
from tests.test_gpu_loss import close  # noqa: E402

INF = float("inf")
SIZES = [(1, 300, 72), (5, 1000, 64), (30, 9000, 72), (60, 9000, 72), (20, 66000, 40), (100, 8200, 72), (200, 8200, 136), (300, 1001, 200)]


def masked(V, kind):
    m = torch.zeros(V, dtype=torch.bool, device="cuda")
    if kind == "end":
        m[-(V // 5):] = True
    elif kind == "middle":
        m[V // 3:V // 3 + 77] = True
    elif kind == "spread":
        m[::7] = True
    else:
        m[:] = True
        m[V // 2] = False
    return m


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("kind", ["end", "middle", "spread", "all but one"])
@pytest.mark.parametrize("M,V,K", SIZES)
def test_masked(M, V, K, kind, dtype):
    """A column of ones in hidden and of -infinity or 0 in the head."""
    from paper_2606_03113_amd import lede
    say("head loss, masked M=%d V=%d K=%d %s" % (M, V, K, kind))
    hidden, head, targets, weights = inputs(M, V, K, dtype, M + V)
    mask = masked(V, kind)
    hidden[:, 3], head[:, 3] = 1.0, 0.0
    kept = (~mask).nonzero()[:, 0]
    place = torch.full((V,), -1, dtype=torch.long, device="cuda")
    place[kept] = torch.arange(len(kept), device="cuda")
    inside = (targets >= 0) & (targets < V)
    targets = torch.where(inside, kept[targets.clamp(0, V - 1).long() % len(kept)].int(), targets)
    ref = Reference(hidden, head[kept], torch.where(inside, place[targets.clamp(0, V - 1).long()], -1).int(), weights)
    head[mask, 3] = -INF
    r = lede.op_head_loss(hidden, head, targets)
    close(r.lse, ref.lse, ref.lse_tol, "lse")
    close(r.loss, ref.loss, ref.loss_tol, "loss")
    dh, dw = lede.op_head_loss_grad(hidden, head, targets, r.lse, weights)
    want, tol = ref.d_head()
    close(dw[kept], want, tol, "d_head")
    assert not bool(dw[mask].any())
    want, tol = ref.d_hidden()
    columns = torch.arange(K, device="cuda") != 3
    left_out = ~ref.kept
    close(dh[:, columns], want[:, columns], tol[:, columns], "d_hidden")
    assert not bool(dh[left_out].any()) and bool(torch.isnan(dh[~left_out, 3]).all())      # 0 times infinity
    # a target among the masked ones has no probability
    targets[0] = int(mask.nonzero()[0])
    again = lede.op_head_loss(hidden, head, targets)
    assert float(again.loss[0]) == INF and torch.equal(again.lse, r.lse)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("M,V,K", [(9, 700, 64), (150, 8200, 72)])
def test_what_has_a_sum(M, V, K, dtype):
    """Which rows have one is what their logits in 64 bits say, wherever infinities and NaNs stand."""
    from paper_2606_03113_amd import lede
    for seed in range(6):
        say("head loss, not finite M=%d V=%d K=%d seed %d" % (M, V, K, seed))
        hidden, head, targets, _ = inputs(M, V, K, dtype, seed)
        g = torch.Generator(device="cuda").manual_seed(seed)
        ref = Reference(hidden, head, targets)
        hidden[:, 5], head[:, 5] = hidden[:, 5].abs().clamp(min=0.1), -head[:, 5].abs().clamp(min=0.01)
        head[torch.randint(0, V, (3,), device="cuda", generator=g), 5] = -INF if seed != 5 else float("nan")
        if seed in (1, 4):
            head[V // 2, 5] = INF
        if seed in (2, 4):
            hidden[M // 2, 7] = INF
            hidden[M // 3, 8] = float("nan")
        if seed == 3:
            hidden[::2, 5] = 0.0             # (0 times infinity)
        z = (hidden.double()[:, :, None] * head.double().t()[None]).sum(1) if M * V * K < 1e6 else torch.cat([(h[None] * head.double()).sum(1)[None] for h in hidden.double()])
        lse = z.logsumexp(1)
        none = torch.isnan(z).any(1) | (z == INF).any(1) | (z == -INF).all(1)
        got = lede.op_head_loss(hidden, head, targets).lse
        assert torch.equal(torch.isnan(got), none), seed
        assert bool(((got.double() - lse).abs()[~none] <= ref.lse_tol[~none] + 2.0 ** -16).all())
