"""Compiled code of the append and sampling kernels (CPU, hipcc only): no spills, no private arrays, and no access whose
memory is only known at run time. (An array in LDS reached through such an access may lie outside the LDS' window of the
address space.)"""
import os
import re
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)


@pytest.mark.skipif(not os.path.exists("/opt/rocm/bin/hipcc") and shutil.which("hipcc") is None, reason="no hipcc")
@pytest.mark.parametrize("src", ["k_append.hip", "k_sample.hip"])
def test_no_spills_and_no_generic_accesses(src, tmp_path):
    from paper_2503_22562_amd import build as B
    out = tmp_path / "k.s"
    cmd = [B.HIPCC, *B.COMMON, *B.HIP_FLAGS, *B.EXTRA_FLAGS.get(src, []), "--cuda-device-only", "-S",
           "-Rpass-analysis=kernel-resource-usage", os.path.join(B.CSRC, src), "-o", str(out)]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-2000:]
    names = re.findall(r"Function Name: (\S+)", r.stderr)
    for what in (r"VGPRs Spill: (\d+)", r"ScratchSize \[bytes/lane\]: (\d+)"):
        found = [int(v) for v in re.findall(what, r.stderr)]
        assert names and len(found) == len(names)
        assert not any(found), (what, list(zip(names, found)))
    lds = [int(v) for v in re.findall(r"LDS Size \[bytes/block\]: (\d+)", r.stderr)]
    assert len(lds) == len(names) and max(lds) <= 64 << 10, lds
    assert not re.findall(r"^\s+(?:flat_|scratch_)\w+", out.read_text(), re.M)
