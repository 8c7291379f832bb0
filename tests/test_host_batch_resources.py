"""Registers and scratch of the batched bf16 attention's kernels, from the compiler's own report
(CPU: the file is compiled as the library's build does, for its remarks)."""

import os
import re
import subprocess

import pytest

from paper_2609_33503_amd import build


def _report(name, out):
    """{kernel: {resource: number}}"""
    src = os.path.join(build.CSRC, name)
    cmd = [build._hipcc(), *build.COMMON, *build.PER_FILE.get(name, []), "-Rpass-analysis=kernel-resource-usage",
           "-x", "hip", "-c", src, "-o", out]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    kernels, cur = {}, None
    for line in r.stderr.splitlines():
        m = re.search(r"remark:\s+(.+?): (\S+) \[-Rpass", line)
        if not m:
            continue
        if m.group(1) == "Function Name":
            cur = kernels.setdefault(m.group(2), {})
        elif cur is not None and m.group(2).isdigit():
            cur[m.group(1)] = int(m.group(2))
    return kernels


def test_no_scratch_in_the_bf16_attention(tmp_path):
    """Neither the attention nor its merge goes through scratch memory, and three workgroups of the
    shared attention's four waves fit a CU's registers."""
    if not os.path.exists(build._hipcc()):
        pytest.skip("needs hipcc")
    kernels = _report("batch_attn.hip", str(tmp_path / "x.o"))
    bf16 = {k: v for k, v in kernels.items() if "battn_bf16" in k or "batch_mergeI" in k}
    assert len(bf16) == 8, sorted(kernels)
    for k, v in bf16.items():
        assert v["ScratchSize [bytes/lane]"] == 0, k
        assert "battn" not in k or v["Occupancy [waves/SIMD]"] >= 3, k
