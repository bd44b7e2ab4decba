"""Refusals of the 4-bit matrices' entry points, and their plain counterparts; no GPU needed.  A refused call touches
nothing, so the pointers here are never followed."""
import numpy as np
import pytest
import torch

from paper_2606_03113_amd import lede
from tests import quant_reference as ref
from tests.test_batch_ops_cpu import NULL, P, _change, lib  # noqa: F401

ARG, UNSUPPORTED = lede.LEDE_E_ARG, lede.LEDE_E_UNSUPPORTED
SHAPE = [(dict(N=0), ARG), (dict(K=0), ARG), (dict(group=16), UNSUPPORTED), (dict(group=0), UNSUPPORTED), (dict(group=256), UNSUPPORTED),
         (dict(N=1 << 24), UNSUPPORTED)]

QUANTIZE = ["dtype", "w", "ldw", "N", "K", "group", "codes", "scales", "stream"]
QUANTIZE_GOOD = [1, P, 300, 20, 300, 32, P, P, NULL]
PACK = ["codes", "scales", "N", "K", "group", "packed", "stream"]
PACK_GOOD = [P, P, 20, 300, 32, P, NULL]
LINEAR = ["dtype", "packed", "N", "K", "group", "x", "ldx", "M", "y_dtype", "y", "ldy", "stream"]
LINEAR_GOOD = [1, P, 20, 300, 32, P, 300, 4, 0, P, 20, NULL]


def test_bytes(lib):  # noqa: F811
    assert lib.lede_op_quant_bytes(16, 128, 32) == 1024 + 128
    assert lib.lede_op_quant_bytes(17, 129, 128) == 4 * (1024 + 32)
    assert lib.lede_op_quant_bytes(128256, 16384, 64) == 8016 * 128 * (1024 + 64)
    for bad in ((0, 1, 32), (1, 0, 32), (1, 1, 48), (-4, 8, 32), (1 << 24, 8, 32), ((1 << 24) - 1, (1 << 24) - 1, 32)):
        assert lib.lede_op_quant_bytes(*bad) == 0


@pytest.mark.parametrize("bad,code", [({k: NULL}, ARG) for k in ("w", "codes", "scales")] + SHAPE + [
    (dict(K=1 << 24, ldw=1 << 24), UNSUPPORTED), (dict(dtype=2), ARG), (dict(ldw=299), ARG), (dict(w=P + 1), ARG), (dict(scales=P + 1), ARG)], ids=str)
def test_quantize_refuses(lib, bad, code):  # noqa: F811
    assert lib.lede_op_quantize(*_change(QUANTIZE_GOOD, QUANTIZE, **bad)) == code


@pytest.mark.parametrize("bad,code", [({k: NULL}, ARG) for k in ("codes", "scales", "packed")] + SHAPE + [(dict(packed=P + 8), ARG)], ids=str)
def test_pack_refuses(lib, bad, code):  # noqa: F811
    assert lib.lede_op_quant_pack(*_change(PACK_GOOD, PACK, **bad)) == code


@pytest.mark.parametrize("bad,code", [({k: NULL}, ARG) for k in ("packed", "x", "y")] + SHAPE + [
    (dict(dtype=-1), ARG), (dict(y_dtype=2), ARG), (dict(M=-1), ARG), (dict(M=1 << 20), UNSUPPORTED), (dict(N=1 << 15, ldy=1 << 15, M=(1 << 19) + 1), UNSUPPORTED), (dict(ldx=299), ARG), (dict(ldy=19), ARG),
    (dict(packed=P + 4), ARG), (dict(x=P + 1), ARG), (dict(y=P + 2), ARG), (dict(dtype=0, x=P + 2), ARG)], ids=str)
def test_linear_refuses(lib, bad, code):  # noqa: F811
    assert lib.lede_op_quant_linear(*_change(LINEAR_GOOD, LINEAR, **bad)) == code


def test_no_rows_is_no_work(lib):  # noqa: F811
    assert lib.lede_op_quant_linear(*_change(LINEAR_GOOD, LINEAR, M=0, x=NULL, y=NULL)) == 0


def test_binding_refuses_wrong_tensors():
    w = torch.zeros(4, 64)
    codes, scales = torch.zeros(4, 32, dtype=torch.uint8), torch.zeros(4, 2, dtype=torch.bfloat16)
    for call in (lambda: lede.op_quantize(w, 32),                  # not on the GPU
                 lambda: lede.op_quantize(w, 33),
                 lambda: lede.op_quantize(w[0], 32),
                 lambda: lede.op_quantize(w.t(), 32),
                 lambda: lede.op_quantize(w.half(), 32),
                 lambda: lede.QuantMatrix(codes, scales, 64, 32),
                 lambda: lede.QuantMatrix(codes, scales, 66, 32),
                 lambda: lede.QuantMatrix(codes, scales[:, :1], 64, 32),
                 lambda: lede.QuantMatrix(codes, scales.float(), 64, 32),
                 lambda: lede.QuantMatrix(codes, scales, 64, 65)):
        with pytest.raises(lede.LedeError):
            call()


def test_reference_codes():
    w = np.array([[0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, -0.2, -5.01, 0.0, 0.26]], np.float32)
    codes, scales = ref.quantize(w, 32)
    assert scales.tolist() == [[1.0]]
    assert codes.tolist() == [[0, 2, 2, 4, 4, 6, 6, 7, 8, 15, 0, 1]]
    assert ref.pack_rows(codes)[0].tolist() == [0x20, 0x42, 0x64, 0x76, 0xF8, 0x10]
    assert ref.values(codes, scales, 32)[0, 7] == 6.0
    assert np.isnan(ref.bf16(np.float32(np.nan))) and ref.bf16(np.float32(1.00390625)) == 1.0 and ref.bf16(np.float32(1.01171875)) == 1.015625
