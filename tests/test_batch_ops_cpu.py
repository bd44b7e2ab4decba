"""Refusals of the batch operators' entry points, and the plain counterparts that their GPU tests compare with; no GPU
needed.  A refused call touches nothing, so the pointers here are never followed."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2606_03113_amd import lede
from tests import batch_reference as ref

P = 1 << 20          # an address of any alignment that is asked for
NULL = None


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(lede.LIB_PATH):
        from paper_2606_03113_amd import build
        build.build()
    return lede.load()


def _change(good, names, **kw):
    args = list(good)
    for k, v in kw.items():
        args[names.index(k)] = v
    return args


def test_cache_bytes(lib):
    assert lib.lede_op_cache_bytes(3, 5, 128) == 3 * 5 * (2 * 64 * 128 + 8)
    assert lib.lede_op_cache_bytes(1 << 20, 8, 128) == (1 << 20) * 8 * (2 * 64 * 128 + 8)   # past 2^32
    for bad in ((0, 1, 64), (1, 0, 64), (1, 1, 96), (1, 1, 256), (1, 1025, 64), (-1, 1, 64)):
        assert lib.lede_op_cache_bytes(*bad) == 0


PLAN = ["seq", "new", "held", "n_seqs", "free", "n_free", "head", "tables", "ld", "max_rows", "kv", "held_out", "start", "slots",
        "status", "stream"]
PLAN_GOOD = [P, P, P, 2, P, 4, P, P, 3, 8, P, P, P, P, P, NULL]


@pytest.mark.parametrize("bad", [{n: NULL} for n in PLAN if n not in ("n_seqs", "n_free", "ld", "max_rows", "stream")] +
                         [dict(n_seqs=0), dict(n_free=-1), dict(ld=0), dict(max_rows=-1)], ids=str)
def test_plan_refuses(lib, bad):
    assert lib.lede_op_cache_plan(*_change(PLAN_GOOD, PLAN, **bad)) == lede.LEDE_E_ARG


@pytest.mark.parametrize("big", [dict(n_seqs=1 << 24), dict(max_rows=1 << 24), dict(max_rows=2 ** 31 - 1)], ids=str)
def test_plan_refuses_what_32_bits_cannot_step_through(lib, big):
    assert lib.lede_op_cache_plan(*_change(PLAN_GOOD, PLAN, **big)) == lede.LEDE_E_UNSUPPORTED


APPEND = ["dtype", "k", "ldk", "v", "ldv", "slots", "n_rows", "cache", "n_pages", "n_kv", "hd", "stream"]
APPEND_GOOD = [1, P, 1024, P, 1024, P, 4, P, 2, 8, 128, NULL]
ROWS_BAD = [(dict(dtype=2), lede.LEDE_E_ARG), (dict(dtype=-1), lede.LEDE_E_ARG), (dict(k=NULL), lede.LEDE_E_ARG),
            (dict(v=NULL), lede.LEDE_E_ARG), (dict(slots=NULL), lede.LEDE_E_ARG), (dict(cache=NULL), lede.LEDE_E_ARG),
            (dict(n_rows=-1), lede.LEDE_E_ARG), (dict(n_pages=0), lede.LEDE_E_ARG), (dict(n_kv=0), lede.LEDE_E_ARG),
            (dict(hd=80), lede.LEDE_E_UNSUPPORTED), (dict(n_kv=1025), lede.LEDE_E_UNSUPPORTED), (dict(ldk=1023), lede.LEDE_E_ARG),
            (dict(ldk=1028), lede.LEDE_E_ARG), (dict(ldv=1016), lede.LEDE_E_ARG), (dict(k=P + 8), lede.LEDE_E_ARG),
            (dict(v=P + 2), lede.LEDE_E_ARG), (dict(cache=P + 8), lede.LEDE_E_ARG), (dict(n_rows=1 << 24), lede.LEDE_E_UNSUPPORTED)]


@pytest.mark.parametrize("bad,code", ROWS_BAD, ids=str)
def test_append_and_read_refuse(lib, bad, code):
    a = _change(APPEND_GOOD, APPEND, **bad)
    assert lib.lede_op_cache_append(*a) == code
    d = dict(zip(APPEND, a))
    assert lib.lede_op_cache_read(d["dtype"], d["cache"], d["n_pages"], d["n_kv"], d["hd"], d["slots"], d["n_rows"], d["k"], d["ldk"],
                                  d["v"], d["ldv"], NULL) == code


def test_no_rows_is_no_work(lib):
    assert lib.lede_op_cache_append(*_change(APPEND_GOOD, APPEND, n_rows=0, k=NULL, v=NULL, slots=NULL)) == 0
    assert lib.lede_op_cache_attention(*_change(ATTN_GOOD, ATTN, n_rows=0, q=NULL, out=NULL)) == 0
    assert lib.lede_op_logprobs(*_change(LP_GOOD, LP, n_rows=0, logits=NULL, ws=NULL)) == 0
    assert lib.lede_op_logprobs(*_change(LP_GOOD, LP, n_rows=0, logits=NULL, ws=NULL, tokens=NULL, ids=NULL, top_lp=NULL)) == 0


ATTN = ["dtype", "q", "ldq", "cache", "n_pages", "tables", "ld", "kv", "start", "n_seqs", "n_rows", "nq", "nkv", "hd", "scale", "max_new",
        "max_kv", "out", "ldo", "ws", "ws_bytes", "stream"]
ATTN_GOOD = [1, P, 4096, P, 64, P, 32, P, P, 2, 2, 32, 8, 128, 0.1, 1, 2000, P, 4096, P, 1 << 30, NULL]


@pytest.mark.parametrize("bad,code", [({n: NULL}, lede.LEDE_E_ARG) for n in ("q", "cache", "tables", "kv", "start", "out", "ws")] + [
    (dict(dtype=3), lede.LEDE_E_ARG), (dict(n_seqs=0), lede.LEDE_E_ARG), (dict(n_rows=-1), lede.LEDE_E_ARG), (dict(ld=0), lede.LEDE_E_ARG),
    (dict(nq=30), lede.LEDE_E_ARG), (dict(nq=0), lede.LEDE_E_ARG), (dict(nkv=0), lede.LEDE_E_ARG), (dict(hd=32), lede.LEDE_E_UNSUPPORTED),
    (dict(scale=float("nan")), lede.LEDE_E_ARG), (dict(scale=float("inf")), lede.LEDE_E_ARG), (dict(max_new=-1), lede.LEDE_E_ARG),
    (dict(max_kv=-1), lede.LEDE_E_ARG), (dict(ldq=4088), lede.LEDE_E_ARG), (dict(ldo=4100), lede.LEDE_E_ARG), (dict(q=P + 4), lede.LEDE_E_ARG),
    (dict(out=P + 8), lede.LEDE_E_ARG), (dict(cache=P + 4), lede.LEDE_E_ARG), (dict(ws=P + 8), lede.LEDE_E_ARG),
    (dict(ws_bytes=16), lede.LEDE_E_ARG), (dict(n_seqs=65536), lede.LEDE_E_UNSUPPORTED), (dict(nq=65544), lede.LEDE_E_UNSUPPORTED),
    (dict(n_rows=1 << 28), lede.LEDE_E_UNSUPPORTED), (dict(n_seqs=1 << 13, nq=1024, nkv=1024), lede.LEDE_E_UNSUPPORTED)], ids=str)
def test_attention_refuses(lib, bad, code):
    assert lib.lede_op_cache_attention_bytes(1, 2, 2, 32, 8, 128, 1, 2000) > 16
    assert lib.lede_op_cache_attention(*_change(ATTN_GOOD, ATTN, **bad)) == code


def test_attention_bytes(lib):
    assert lib.lede_op_cache_attention_bytes(1, 1, 1, 4, 4, 64, 1, 100) == 0            # one split
    assert lib.lede_op_cache_attention_bytes(1, 0, 1, 4, 4, 64, 1, 100) == 0
    assert lib.lede_op_cache_attention_bytes(1, 1, 1, 5, 4, 64, 1, 100) == 0
    # sizes that only spread the work may be anything
    assert lib.lede_op_cache_attention_bytes(1, 1, 1, 64, 8, 128, 1, 2 ** 31 - 1) > 0
    assert lib.lede_op_cache_attention_bytes(1, 1, 2 ** 31 - 1, 64, 8, 128, 2 ** 31 - 1, 2 ** 31 - 1) >= 0


LP = ["dtype", "logits", "ld", "n_rows", "V", "T", "tokens", "top", "lp", "ranks", "ent", "ids", "top_lp", "ws", "ws_bytes", "stream"]
LP_GOOD = [0, P, 50000, 4, 50000, 1.0, P, 5, P, P, P, P, P, P, 1 << 30, NULL]


@pytest.mark.parametrize("bad,code", [({n: NULL}, lede.LEDE_E_ARG) for n in ("logits", "tokens", "ids", "top_lp", "ws")] + [
    (dict(dtype=5), lede.LEDE_E_ARG), (dict(n_rows=-1), lede.LEDE_E_ARG), (dict(V=0), lede.LEDE_E_ARG), (dict(ld=49999), lede.LEDE_E_ARG),
    (dict(top=-1), lede.LEDE_E_ARG), (dict(top=33), lede.LEDE_E_UNSUPPORTED), (dict(V=4, top=5), lede.LEDE_E_ARG), (dict(T=0.0), lede.LEDE_E_ARG),
    (dict(T=-1.0), lede.LEDE_E_ARG), (dict(T=float("nan")), lede.LEDE_E_ARG), (dict(T=float("inf")), lede.LEDE_E_ARG),
    (dict(T=1e-45), lede.LEDE_E_ARG), (dict(logits=P + 2), lede.LEDE_E_ARG), (dict(ws=P + 8), lede.LEDE_E_ARG), (dict(ws_bytes=8), lede.LEDE_E_ARG),
    (dict(V=(1 << 20) + 1, ld=1 << 21), lede.LEDE_E_UNSUPPORTED),
    (dict(n_rows=1 << 24, ws_bytes=1 << 40), lede.LEDE_E_UNSUPPORTED)], ids=str)
def test_logprobs_refuses(lib, bad, code):
    assert lib.lede_op_logprobs(*_change(LP_GOOD, LP, **bad)) == code


def test_binding_refuses_wrong_tensors():
    f, i = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(lede.LedeError):
        lede.op_logprobs(f, i)                       # not on the GPU
    with pytest.raises(lede.LedeError):
        lede.op_logprobs(f, i.long())
    with pytest.raises(lede.LedeError):
        lede.op_logprobs(f.half(), i)
    with pytest.raises(lede.LedeError):
        lede.Cache(4, 2, 96)
    with pytest.raises(lede.LedeError):
        lede.op_cache_plan(i, i[:3], i, i, i[:1], torch.zeros(4, 2, dtype=torch.int32), 8)
    region = torch.zeros(load_bytes(4, 2, 64), dtype=torch.uint8)
    c = lede.Cache(4, 2, 64, region=region)
    with pytest.raises(lede.LedeError):
        lede.Cache(5, 2, 64, region=region)
    rows = torch.zeros(4, 2, 64)
    with pytest.raises(lede.LedeError):
        lede.op_cache_append(c, rows, rows, i)       # slots must be int64
    with pytest.raises(lede.LedeError):
        lede.op_cache_append(c, rows, rows[:, :1], i.long())
    with pytest.raises(lede.LedeError):
        lede.op_cache_attention(c, rows, i, i, i, 1, 1)


def load_bytes(*a):
    return lede.load().lede_op_cache_bytes(*a)


# ---- the plain counterparts ------------------------------------------------------------


def test_reference_codes_are_e4m3():
    """Rounding to the nearest code is torch's conversion, over every value of a fine grid and the ties."""
    x = np.concatenate([np.linspace(-448, 448, 20001), np.ldexp(np.arange(-480, 481), -14), np.ldexp(np.arange(-2048, 2049), -16),
                        np.arange(-448.0, 449.0)])
    got = ref.nearest_code(x)
    want = torch.from_numpy(x.astype(np.float32)).to(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(got.astype(np.float32), want)
    assert np.isnan(ref.nearest_code([np.nan, np.inf])).all()


@pytest.mark.parametrize("amax,e", [(0.0, -100), (448.0, 0), (449.0, 1), (224.0, -1), (1e-40, -100), (2.0 ** 127, 119), (3.4e38, 120),
                                    (448.0 * 2.0 ** -30, -30)])
def test_reference_exponent(amax, e):
    assert ref.exponent(amax) == e


def test_reference_plan():
    tables = np.array([[5, -1, -1], [6, 7, -1]], np.int32)
    free = np.array([9, 8, 1, 0], np.int32)
    kv, held, start, slots, tab, status = ref.plan([63, 64], [2, 1], [1, 2], 4, 1, 3, 5, free, tables)
    assert kv.tolist() == [65, 65] and held.tolist() == [2, 2] and start.tolist() == [0, 2, 3]
    assert slots.tolist() == [5 * 64 + 63, 8 * 64, 7 * 64, -1, -1] and tab.tolist() == [[5, 8, -1], [6, 7, -1]] and status == [0, 3, 2, -1]
    assert ref.plan([63, 64], [200, 1], [1, 2], 4, 1, 3, 500, free, tables)[-1] == [ref.E_CTX_OVERFLOW, 0, 1, 0]
    assert ref.plan([63, 64], [2, 66], [1, 2], 2, 1, 3, 500, free, tables)[-1] == [ref.E_KV_FULL, 0, 1, 1]
