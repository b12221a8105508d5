"""What the compiler says of the fp32 attention kernels without a window: they are
kernels of their own, and hold what they need in registers."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_fp32_kernels_without_a_window_do_not_spill(tmp_path):
    from paper_2609_36692_gb300 import build
    try:
        nvcc = build._nvcc()
    except RuntimeError:
        pytest.skip("needs nvcc")
    filt = shutil.which("c++filt")
    if not filt:
        pytest.skip("needs c++filt")
    r = subprocess.run([nvcc, *build.ARCH, *build.CFLAGS, "-Xptxas", "-v", "-c", os.path.join(build.CSRC, "attn_simt.cu"), "-o",
                        str(tmp_path / "x.o")], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    text = subprocess.run([filt], input=r.stderr, capture_output=True, text=True).stdout
    spills = re.findall(r"Compiling entry function '(.*?)'.*?(\d+) bytes spill stores, (\d+) bytes spill loads", text, re.S)
    whole = [s for s in spills if re.search(r"k_attn_(fwd|bwd)<float, \d+, false>", s[0])]
    assert len(whole) == 4
    assert all(s[1] == s[2] == "0" for s in whole), whole
