"""Refusals of the vocabulary head's loss and its gradient; no GPU needed.  A refused call touches nothing, so the pointers
here are never followed."""
import pytest
import torch

from paper_2606_03113_amd import lede
from tests.loss_reference import Reference, inputs
from tests.test_batch_ops_cpu import NULL, P, _change, lib  # noqa: F401

ARG, UNSUPPORTED = lede.LEDE_E_ARG, lede.LEDE_E_UNSUPPORTED

LOSS = ["dtype", "hidden", "ldh", "M", "head", "ldw", "V", "K", "targets", "loss", "lse", "ws", "ws_bytes", "stream"]
LOSS_GOOD = [1, P, 256, 4, P, 256, 1000, 256, P, P, P, P, 1 << 40, NULL]
GRAD = ["dtype", "hidden", "ldh", "M", "head", "ldw", "V", "K", "targets", "lse", "weights", "dh", "ld_dh", "dw", "ld_dw", "ws", "ws_bytes", "stream"]
GRAD_GOOD = [1, P, 256, 4, P, 256, 1000, 256, P, P, P, P, 256, P, 256, P, 1 << 40, NULL]

BOTH = [({k: NULL}, ARG) for k in ("hidden", "head", "targets", "lse", "ws")] + [
    (dict(dtype=2), ARG), (dict(M=-1), ARG), (dict(V=0), ARG), (dict(K=0), ARG), (dict(ldh=255), ARG), (dict(ldw=248), ARG), (dict(ldh=260), ARG),
    (dict(hidden=P + 8), ARG), (dict(head=P + 2), ARG), (dict(ws=P + 8), ARG), (dict(ws_bytes=64), ARG), (dict(K=252), UNSUPPORTED),
    (dict(K=32776, ldh=32776, ldw=32776), UNSUPPORTED), (dict(M=(1 << 18) + 1), UNSUPPORTED), (dict(V=(1 << 20) + 1), UNSUPPORTED), (dict(ldw=1 << 22), UNSUPPORTED), (dict(ldh=1 << 22), UNSUPPORTED)]


@pytest.mark.parametrize("bad,code", BOTH, ids=str)
def test_loss_refuses(lib, bad, code):  # noqa: F811
    assert lib.lede_op_head_loss(*_change(LOSS_GOOD, LOSS, **bad)) == code


@pytest.mark.parametrize("bad,code", BOTH + [(dict(ld_dh=255), ARG), (dict(ld_dw=252), ARG), (dict(dh=P + 4), ARG), (dict(dw=P + 8), ARG)], ids=str)
def test_gradient_refuses(lib, bad, code):  # noqa: F811
    assert lib.lede_op_head_loss_grad(*_change(GRAD_GOOD, GRAD, **bad)) == code


def test_no_work(lib):  # noqa: F811
    assert lib.lede_op_head_loss(*_change(LOSS_GOOD, LOSS, M=0, hidden=NULL, targets=NULL, lse=NULL, loss=NULL, ws=NULL, ws_bytes=0)) == 0
    assert lib.lede_op_head_loss_grad(*_change(GRAD_GOOD, GRAD, dh=NULL, dw=NULL)) == 0
    assert lib.lede_op_head_loss_grad(*_change(GRAD_GOOD, GRAD, M=0, dw=NULL, hidden=NULL, ws=NULL)) == 0


@pytest.mark.parametrize("sizes", [(2, 4, 100, 64), (0, -1, 100, 64), (1, 4, 0, 64), (1, 4, 100, 60), (1, (1 << 18) + 1, 100, 64), (0, 1, (1 << 20) + 1, 64)])
def test_bytes_of_what_is_refused(lib, sizes):  # noqa: F811
    assert lib.lede_op_head_loss_bytes(*sizes) == 0 and lib.lede_op_head_loss_grad_bytes(*sizes) == 0


@pytest.mark.parametrize("dtype", [0, 1])
def test_bytes_stay_far_below_the_logits(lib, dtype):  # noqa: F811
    logits = 4 * 16384 * 128256
    assert 0 < lib.lede_op_head_loss_bytes(dtype, 16384, 128256, 4096) < logits / 8
    assert 0 < lib.lede_op_head_loss_grad_bytes(dtype, 16384, 128256, 4096) < logits / 6
    # the ends of the sizes
    assert lib.lede_op_head_loss_bytes(dtype, 1 << 18, 1 << 20, 1 << 15) > 0 and lib.lede_op_head_loss_grad_bytes(dtype, 1 << 18, 1 << 20, 1 << 15) > 0
    assert lib.lede_op_head_loss_bytes(dtype, 1, 1, 8) > 0 and lib.lede_op_head_loss_grad_bytes(dtype, 1, 1, 8) > 0


def test_binding_sizes_past_32_bits():
    L = lede.load()
    assert L.lede_op_head_loss_bytes(0, 1 << 18, 1 << 20, 8) > 1 << 33
    assert L.lede_op_head_loss_grad_bytes(0, 1 << 18, 32000, 4096) > 1 << 33
    assert L.lede_op_quant_bytes(1 << 20, 1 << 14, 32) > 1 << 33


def test_binding_refuses_wrong_tensors():
    h, w, t = torch.zeros(4, 64), torch.zeros(100, 64), torch.zeros(4, dtype=torch.int32)
    for call in (lambda: lede.op_head_loss(h, w, t),              # not on the GPU
                 lambda: lede.op_head_loss(h, w[:, :32], t),
                 lambda: lede.op_head_loss(h, w.bfloat16(), t),
                 lambda: lede.op_head_loss(h.half(), w.half(), t),
                 lambda: lede.op_head_loss(h, w, t.long()),
                 lambda: lede.op_head_loss(h, w, t[:3]),
                 lambda: lede.op_head_loss(h[:, :60], w[:, :60], t),
                 lambda: lede.op_head_loss_grad(h, w, t, h[:, 0]),
                 lambda: lede.op_head_loss_grad(h, w, t, torch.zeros(4), torch.zeros(3)),
                 lambda: lede.op_head_loss_grad(h, w, t, torch.zeros(4), out=(w, h))):
        with pytest.raises(lede.LedeError):
            call()


def test_reference_gradient_is_autograd():
    hidden, head, targets, weights = inputs(12, 50, 16, torch.float32, 1, device="cpu")
    ref = Reference(hidden, head, targets, weights)
    h, w = hidden.double().requires_grad_(), head.double().requires_grad_()
    keep = ref.trained
    z = h @ w.t()
    nll = -torch.log_softmax(z, 1).gather(1, torch.where(keep, targets.long(), 0)[:, None])[:, 0]
    loss = torch.where(keep, nll, 0.0)
    (loss * weights.double()).sum().backward()
    assert torch.allclose(ref.loss, loss.detach(), atol=1e-12)
    assert torch.allclose(ref.d_hidden()[0], h.grad, atol=1e-12) and torch.allclose(ref.d_head()[0], w.grad, atol=1e-12)
