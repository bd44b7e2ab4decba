"""The head loss where every tile's ring of steps turns several times: contractions of many steps for the logits, for their
gradients' parts and for dW, in each tile of both types."""
import pytest

from tests.parity import say

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
from tests.loss_reference import inputs  # noqa: E402
from tests.test_gpu_loss import check  # noqa: E402


# logits: by M and V; steps of 64 by K (456: eight, the last short)
@pytest.mark.parametrize("M,V,K", [(200, 16500, 456), (300, 20001, 1032), (129, 16384, 192), (100, 16500, 456), (40, 16500, 456), (300, 1000, 712), (1030, 16400, 328)])
def test_bf16(M, V, K):
    say("head loss, many steps M=%d V=%d K=%d bf16" % (M, V, K))
    check(*inputs(M, V, K, torch.bfloat16, M + K))


# dW: steps of 64 by M, tiles 256 x 64, x 128 and x 256 by V and K
@pytest.mark.parametrize("M,V,K", [(400, 64, 16384), (400, 120, 16400), (520, 5000, 1024), (900, 500, 136)])
def test_bf16_head_gradient(M, V, K):
    say("head loss, many rows M=%d V=%d K=%d bf16" % (M, V, K))
    check(*inputs(M, V, K, torch.bfloat16, M + K))


# tiles of 128 x 128, 64 x 128, and thin ones of 64 and 128 by 16, 32 and 64; then dW's 128 x 128, 64 x 128 and 64 x 64, many rows
@pytest.mark.parametrize("M,V,K", [(200, 8200, 456), (130, 16390, 264), (100, 8200, 456), (60, 33000, 456), (60, 9000, 456), (30, 33000, 328), (30, 9000, 712),
                                   (12, 33000, 456), (12, 3000, 1032), (60, 1000, 456), (500, 8200, 1032), (700, 300, 520), (300, 60, 1032)])
def test_fp32(M, V, K):
    say("head loss, many steps M=%d V=%d K=%d f32" % (M, V, K))
    check(*inputs(M, V, K, torch.float32, M + K))
