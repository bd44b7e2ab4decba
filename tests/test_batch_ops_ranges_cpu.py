"""Refusals of the batch operators at the ends of their ranges; no GPU needed.  A refused call touches nothing, so the
pointers here are never followed."""
import os
import subprocess

import pytest

from paper_2606_03113_amd import lede
from tests.sanitize.build import CLANG
from tests.test_batch_ops_cpu import ATTN, ATTN_GOOD, _change, lib  # noqa: F401


@pytest.mark.parametrize("scale", [1.1e38, -1.1e38, 3.4e38, -3.4e38], ids=str)
def test_attention_refuses_scales_beyond_its_range(lib, scale):  # noqa: F811
    """In the exponent's base the scale is 2 log2(e) times as large: from 1.2e38 on it would be infinite there."""
    assert lib.lede_op_cache_attention(*_change(ATTN_GOOD, ATTN, scale=scale)) == lede.LEDE_E_ARG
    assert lib.lede_op_cache_attention(*_change(ATTN_GOOD, ATTN, scale=scale / 4, n_rows=0)) == 0


@pytest.mark.skipif(not os.path.exists(CLANG), reason="ROCm compilers not installed")
def test_attention_workspace_over_the_ends_of_its_sizes(tmp_path):
    """No overflow in the rules that spread the work, nothing for sizes that the call refuses, and less than a GiB."""
    exe = str(tmp_path / "cache_sizes")
    subprocess.check_call([CLANG, "-O1", "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-D__HIP_PLATFORM_AMD__",
                           "-I/opt/rocm/include", os.path.join(os.path.dirname(os.path.abspath(__file__)), "cache_sizes.cpp"), "-o", exe])
    p = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert p.returncode == 0, p.stdout + p.stderr
