"""Refusals of the calls that share, own, copy, free and compact pages, and their plain counterparts; no GPU needed.  A
refused call touches nothing, so the pointers here are never followed."""
import pytest
import torch

from paper_2606_03113_amd import lede
from tests.pages_reference import Pool
from tests.test_batch_ops_cpu import NULL, P, _change, lib  # noqa: F401

ARG, UNSUPPORTED = lede.LEDE_E_ARG, lede.LEDE_E_UNSUPPORTED

FORK = ["source", "lens", "seq", "held", "n", "tables", "ld", "shares", "n_pages", "status", "stream"]
FORK_GOOD = [P, P, P, P, 3, P, 4, P, 9, P, NULL]
OWN = ["seq", "new", "held", "n", "free", "n_free", "head", "tables", "ld", "shares", "n_pages", "pairs", "max_moves", "status", "stream"]
OWN_GOOD = [P, P, P, 3, P, 9, P, P, 4, P, 9, P, 3, P, NULL]
FREE = ["seq", "held", "n", "free", "n_free", "head", "tables", "ld", "shares", "n_pages", "status", "stream"]
FREE_GOOD = [P, P, 3, P, 9, P, P, 4, P, 9, P, NULL]
COMPACT = ["held", "n", "free", "n_free", "head", "tables", "ld", "shares", "n_pages", "pairs", "max_moves", "status", "stream"]
COMPACT_GOOD = [P, 3, P, 9, P, P, 4, P, 9, P, 4, P, NULL]
COPY = ["pairs", "count", "max_moves", "cache", "n_pages", "kv", "hd", "stream"]
COPY_GOOD = [P, P, 4, P, 9, 8, 128, NULL]

SIZES = [(dict(n=0), ARG), (dict(ld=0), ARG), (dict(n_pages=0), ARG), (dict(n=1 << 24), UNSUPPORTED), (dict(ld=1 << 29), UNSUPPORTED), (dict(n=1 << 16, ld=(1 << 14) + 1), UNSUPPORTED)]


@pytest.mark.parametrize("bad,code", [({k: NULL}, ARG) for k in ("source", "seq", "held", "tables", "shares", "status")] + SIZES, ids=str)
def test_fork_refuses(lib, bad, code):  # noqa: F811
    assert lib.lede_op_cache_fork(*_change(FORK_GOOD, FORK, **bad)) == code


@pytest.mark.parametrize("bad,code", [({k: NULL}, ARG) for k in ("seq", "new", "held", "free", "head", "tables", "shares", "pairs", "status")] + SIZES + [
    (dict(n_free=-1), ARG), (dict(max_moves=-1), ARG), (dict(max_moves=1 << 24), UNSUPPORTED)], ids=str)
def test_own_refuses(lib, bad, code):  # noqa: F811
    assert lib.lede_op_cache_own(*_change(OWN_GOOD, OWN, **bad)) == code


@pytest.mark.parametrize("bad,code", [({k: NULL}, ARG) for k in ("seq", "held", "free", "head", "tables", "shares", "status")] + SIZES + [
    (dict(n_free=-1), ARG), (dict(n_pages=(1 << 18) + 1), UNSUPPORTED)], ids=str)
def test_free_refuses(lib, bad, code):  # noqa: F811
    assert lib.lede_op_cache_free(*_change(FREE_GOOD, FREE, **bad)) == code


@pytest.mark.parametrize("bad,code", [({k: NULL}, ARG) for k in ("held", "free", "head", "tables", "shares", "pairs", "status")] + SIZES + [
    (dict(n_free=-1), ARG), (dict(max_moves=-1), ARG), (dict(n_pages=(1 << 18) + 1), UNSUPPORTED), (dict(max_moves=1 << 24), UNSUPPORTED)], ids=str)
def test_compact_refuses(lib, bad, code):  # noqa: F811
    assert lib.lede_op_cache_compact(*_change(COMPACT_GOOD, COMPACT, **bad)) == code


@pytest.mark.parametrize("bad,code", [({k: NULL}, ARG) for k in ("pairs", "count", "cache")] + [
    (dict(max_moves=-1), ARG), (dict(n_pages=0), ARG), (dict(kv=0), ARG), (dict(hd=96), UNSUPPORTED), (dict(kv=1025), UNSUPPORTED),
    (dict(cache=P + 8), ARG), (dict(max_moves=1 << 24), UNSUPPORTED)], ids=str)
def test_copy_refuses(lib, bad, code):  # noqa: F811
    assert lib.lede_op_cache_copy(*_change(COPY_GOOD, COPY, **bad)) == code


def test_no_moves_is_no_work(lib):  # noqa: F811
    assert lib.lede_op_cache_copy(*_change(COPY_GOOD, COPY, max_moves=0, pairs=NULL, count=NULL)) == 0


def test_binding_refuses_wrong_tensors():
    i = torch.zeros(4, dtype=torch.int32)
    tab, shares = torch.zeros(4, 2, dtype=torch.int32), torch.zeros(9, dtype=torch.int32)
    one = i[:1]
    for call in (lambda: lede.op_cache_fork(i, i, i, tab, shares),                        # not on the GPU
                 lambda: lede.op_cache_fork(i.long(), i, i, tab, shares),
                 lambda: lede.op_cache_fork(i, i, i[:3], tab, shares),
                 lambda: lede.op_cache_fork(i, i, i, tab[:3], shares),
                 lambda: lede.op_cache_fork(i, i, i, tab, shares, lens=i[:2]),
                 lambda: lede.op_cache_fork(i, i, i, tab, shares, status=i),
                 lambda: lede.op_cache_own(i, i, i, i, i, tab, shares, 4),
                 lambda: lede.op_cache_own(i, i, i, i, one, tab, shares, -1),
                 lambda: lede.op_cache_own(i, i, i, i, one, tab, shares, 4, out=lede.CacheMoves(i, i)),
                 lambda: lede.op_cache_free(i, i, i, one, tab, shares, status=i[:3]),
                 lambda: lede.op_cache_free(i, i, i, one, tab[:, :1], shares),
                 lambda: lede.op_cache_compact(i, i, one, tab, shares.float(), 4),
                 lambda: lede.op_cache_copy(lede.Cache(4, 2, 64, region=torch.zeros(lede.load().lede_op_cache_bytes(4, 2, 64), dtype=torch.uint8)),
                                            tab, i)):
        with pytest.raises(lede.LedeError):
            call()


# ---- the plain counterparts ------------------------------------------------------------


def _pool():
    return Pool([70, 0, 0], [2, 0, 0], [[4, 9, -1], [-1] * 3, [-1] * 3], [4, 9, 0, 1, 2, 3, 5, 6, 7, 8], 2, 10)


def test_reference_fork_own_free_compact():
    p = _pool()
    assert p.fork([-1, 0, 0], [0, 70, 64]) == [0, 3, -1]
    assert p.held.tolist() == [2, 2, 1] and p.shares()[[4, 9]].tolist() == [2, 1]
    assert p.own([1, 1, 1], 3) == ([0, 1, 3, -1], [(9, 0)])        # the first keeps page 9, the second takes page 0
    assert p.tables[0, 1] == 9 and p.tables[1, 1] == 0
    p.seq[:] = [0, 70, 0]
    assert p.release() == [0, 1, 2, -1] and p.free[2] == 9 and p.shares().sum() == 0
    assert p.compact(5) == ([0, 1, 2, 2], [(4, 1)])
    assert p.tables[1, :2].tolist() == [1, 0] and p.free[2:].tolist() == list(range(2, 10))


def test_reference_failures():
    p = _pool()
    assert p.fork([-1, 0, 1]) == [-1, 0, 2]
    assert p.fork([1, -1, -1]) == [-2, 0, 0]
    p.fork([-1, 0, 0])
    assert p.own([1, 1, 1], 1)[0] == [-1, 0, 2, 2]
    p.head = 10
    assert p.own([0, 1, 0], 3)[0] == [-3, 0, 10, 1]
