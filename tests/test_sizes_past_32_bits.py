"""Sizes that the entry points' 32-bit arguments do not hold are refused by the binding, not cut off.  The tensors are
meta ones: they have sizes and no memory."""
import pytest
import torch

from paper_2606_03113_amd import lede

BIG = (1 << 32) + 100      # cut off: 100


def meta(*shape, dtype=torch.int32):
    return torch.empty(*shape, dtype=dtype, device="meta")


def fork(n=4, width=8, pages=16):
    return lede.op_cache_fork(meta(n), meta(n), meta(n), meta(n, width), meta(pages))


def own(n=4, width=8, pages=16, free=16, moves=4):
    return lede.op_cache_own(meta(n), meta(n), meta(n), meta(free), meta(1), meta(n, width), meta(pages), moves)


def free(n=4, width=8, pages=16, free=16):
    return lede.op_cache_free(meta(n), meta(n), meta(free), meta(1), meta(n, width), meta(pages))


def compact(n=4, width=8, pages=16, free=16, moves=4):
    return lede.op_cache_compact(meta(n), meta(free), meta(1), meta(n, width), meta(pages), moves)


def copy(moves=4):
    cache = lede.Cache.__new__(lede.Cache)
    cache.region, cache.n_pages, cache.n_kv, cache.head_dim, cache.device = meta(64, dtype=torch.uint8), 1, 1, 64, torch.device("meta")
    return lede.op_cache_copy(cache, meta(moves, 2), meta(1))


def quantize(N=4, K=64):
    return lede.op_quantize(meta(N, K, dtype=torch.float32), 32)


def matrix(N=4, K=64):
    return lede.QuantMatrix(meta(N, (K + 1) // 2, dtype=torch.uint8), meta(N, -(-K // 32), dtype=torch.bfloat16), K, 32)


def linear(M=4):
    q = lede.QuantMatrix.__new__(lede.QuantMatrix)
    q.packed, q.N, q.K, q.group, q.device = meta(1152, dtype=torch.uint8), 16, 64, 32, torch.device("meta")
    return lede.op_quant_linear(q, meta(M, 64, dtype=torch.float32))


def loss(M=4, V=100, K=64):
    return lede.op_head_loss(meta(M, K, dtype=torch.float32), meta(V, K, dtype=torch.float32), meta(M))


def loss_grad(M=4, V=100, K=64):
    return lede.op_head_loss_grad(meta(M, K, dtype=torch.float32), meta(V, K, dtype=torch.float32), meta(M), meta(M, dtype=torch.float32))


CALLS = {fork: ("n", "width", "pages"), own: ("n", "width", "pages", "free", "moves"), free: ("n", "width", "pages", "free"),
         compact: ("n", "width", "pages", "free", "moves"), copy: ("moves",), quantize: ("N", "K"), matrix: ("N", "K"), linear: ("M",),
         loss: ("M", "V", "K"), loss_grad: ("M", "V", "K")}


@pytest.mark.parametrize("call,size", [(c, s) for c, sizes in CALLS.items() for s in sizes], ids=lambda x: getattr(x, "__name__", x))
def test_refused(call, size):
    with pytest.raises(lede.LedeError) as e:      # (tensors that are not on the GPU)
        call()
    assert e.value.code == lede.LEDE_E_ARG
    for n in (BIG, 1 << 31):
        with pytest.raises(lede.LedeError) as e:
            call(**{size: n})
        assert e.value.code == lede.LEDE_E_UNSUPPORTED
