"""Compiled code of the attention kernels (CPU, hipcc only): no instantiation spills registers or uses scratch memory."""
import os
import re
import shutil
import subprocess

import pytest


@pytest.mark.skipif(not os.path.exists("/opt/rocm/bin/hipcc") and shutil.which("hipcc") is None, reason="no hipcc")
def test_attention_kernels_do_not_spill(tmp_path):
    from paper_2503_22562_amd import build as B
    cmd = [B.HIPCC, *B.COMMON, *B.HIP_FLAGS, *B.EXTRA_FLAGS.get("k_attention.hip", []), "--cuda-device-only",
           "-Rpass-analysis=kernel-resource-usage", "-c", os.path.join(B.CSRC, "k_attention.hip"), "-o", str(tmp_path / "k.o")]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-2000:]
    blocks = re.split(r"Function Name: ", r.stderr)[1:]
    names = [b.split()[0] for b in blocks]
    assert any("attn_kernel" in n for n in names) and any("attn_merge_kernel" in n for n in names)
    for what in ("VGPRs Spill", "SGPRs Spill", r"ScratchSize \[bytes/lane\]"):
        used = [int(re.search(what + r": (\d+)", b).group(1)) for b in blocks]
        assert not any(used), (what, [(n, u) for n, u in zip(names, used) if u])
