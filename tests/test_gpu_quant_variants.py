"""Products with 4-bit weights in every variant that sizes choose, by groups, by how x can be read, and with more steps of the
contraction than are on their way at a time."""
import numpy as np
import pytest

from tests import quant_reference as ref
from tests.parity import say
from tests.test_gpu_quant import DT, lede, random_matrix, rounded

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

# x in LDS: 16 waves share the columns, or 8 (more than 8176 outputs); with more than 64 KiB of LDS in all
THIN = [("f32", 5, 700, 2048), ("bf16", 15, 700, 2048), ("f32", 1, 40, 10240), ("bf16", 1, 8300, 4424), ("bf16", 2, 8300, 2312), ("f32", 1, 8300, 2312),
        ("f32", 2, 8200, 4800), ("f32", 7, 8177, 520), ("f32", 16, 8200, 264)]
# blocks of 32 x 16, 64 x 16 (one and several tiles of rows), 128 x 32, 128 x 64 outputs
WIDE = [("bf16", 16, 2000, 4616), ("bf16", 40, 1300, 4616), ("bf16", 13, 9000, 2312), ("bf16", 64, 2100, 2312), ("bf16", 50, 8300, 2312), ("bf16", 250, 4200, 2312),
        ("f32", 20, 1500, 2312), ("f32", 13, 9000, 2312), ("f32", 64, 2100, 2312), ("f32", 50, 8300, 2312), ("f32", 250, 4200, 1288)]


@pytest.mark.parametrize("odd", [False, True], ids=["pieces", "elements"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype,M,N,K", THIN + WIDE)
def test_variant(dtype, M, N, K, group, odd):
    """odd: rows of x that cannot be read in 16-byte pieces."""
    K -= odd
    say("quant linear M=%d N=%d K=%d group=%d %s" % (M, N, K, group, dtype))
    r = np.random.default_rng(M + N + K + group)
    q, codes, scales, w = random_matrix(r, N, K, group)
    d, x = rounded(r.standard_normal((M, K)), dtype)
    room = torch.full((M + 2, N + 8), 7.0, device="cuda")
    y = room[1:-1, 4:-4]
    lede().op_quant_linear(q, d, out=y)
    want, tol = ref.linear(x, w, group, dtype, "f32")
    err = np.abs(y.double().cpu().numpy() - want)
    assert (err <= tol).all(), (float((err / tol).max()), np.argwhere(err > tol)[:3])
    got = lede().op_quant_linear(q, d, dtype=torch.bfloat16)
    assert torch.equal(got, y.to(torch.bfloat16))
    # rows with a single one: the weights themselves, from every part of the contraction
    at = r.permutation(K)[:M] if M > 1 else np.array([K - 1])
    at[0] = K - 1
    one = torch.zeros(M, K, device="cuda", dtype=DT[dtype])
    one[torch.arange(M), torch.from_numpy(at)] = 1.0
    lede().op_quant_linear(q, one, out=y)
    assert np.array_equal(y.double().cpu().numpy(), w[:, at].T)
    y.fill_(7.0)
    assert bool((room == 7.0).all())
