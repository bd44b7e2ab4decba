"""The ring in LDS of the head loss's bf16 products: what orders its reads and copies stands in the source and in the code
that the compiler makes of it (no GPU needed)."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2606_03113_amd import build as b


def functions(text):
    """(header, body) of every function definition: from a line that opens a brace at no indentation to the one that closes it."""
    out, lines, at = [], text.split("\n"), 0
    for i, line in enumerate(lines):
        if line == "}" or line.startswith("};"):
            head = [x for x in lines[at:i] if not x.startswith("//")]
            out.append("\n".join(head))
            at = i + 1
    return out


def test_no_barrier_among_pointers_said_to_be_apart():
    """A `__restrict__` pointer holds for a function's whole body, so memory that another pointer writes there must not be the
    same on the two sides of a barrier."""
    seen = 0
    for src in sorted(os.listdir(b.CSRC)):
        if not src.endswith((".hip", ".h")):
            continue
        for f in functions(open(os.path.join(b.CSRC, src)).read()):
            if "lds8* __restrict__" in f:
                seen += 1
                assert not re.search(r"barrier<|s_barrier|lds_barrier\(|__syncthreads", f), (src, f[:200])
    assert seen


@pytest.mark.skipif(not os.path.exists(b.HIPCC) or not shutil.which("c++filt"), reason="hipcc not installed")
def test_a_step_lies_between_its_barriers(tmp_path):
    """In the loop that copies, from one barrier to the next: one step's copies and one step's reads, so none has moved over a
    barrier (products, which touch registers alone, may)."""
    out = str(tmp_path / "loss.s")
    p = subprocess.run([b.HIPCC, "-x", "hip", *b.FLAGS, "--cuda-device-only", "-S", os.path.join(b.CSRC, "loss.hip"), "-o", out], capture_output=True,
                       text=True, timeout=600)
    assert p.returncode == 0, p.stderr[-2000:]
    text, kernels = open(out).read(), 0
    for m in re.finditer(r"^(_ZN4lede6k_headILb\S+):(.*?)\.size\s+\1", text, re.S | re.M):
        name = subprocess.run(["c++filt", m.group(1)], capture_output=True, text=True).stdout
        args = re.search(r"k_head<(.*?)>", name).group(1).split(", ")
        ca, cb = (x == "true" for x in args[:2])
        ti, tj, wi, wj = (int(x) for x in args[2:6])
        ni, nj = ti // wi // 16, tj // wj // 16
        copies = (ti + tj) // (8 * wi * wj)
        body = "\n".join(x.split(";")[0] for x in m.group(2).split("\n"))
        parts = [x for x in re.split(r"s_barrier\b", body) if "buffer_load_dwordx4" in x and re.search(r"buffer_load_dwordx4[^\n]*\blds\b", x)]
        loops = [x for x in parts if "ds_read" in x]
        assert len(parts) == 2 and len(loops) == 1, (name, len(parts), len(loops))      # (the first copies, then the loop's)
        loop = loops[0]
        got = [len(re.findall(r, loop)) for r in (r"buffer_load_dwordx4[^\n]*\blds\b", r"\bds_read_b64_tr_b16\b", r"\bds_read_b128\b")]
        want = [copies, 4 * (ni * ca + nj * cb), 2 * (ni * (not ca) + nj * (not cb))]
        assert got == want, (name, got, want)
        kernels += 1
    assert kernels == 16
