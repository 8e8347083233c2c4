"""The kernel of few rows counts the loads behind the one that it waits for, so it must have no others in its loop: no spilled registers."""
import os
import re
import shutil
import subprocess

import pytest

import paper_2602_11543_amd as S

TOOLS = "/opt/rocm/llvm/bin:/opt/rocm/lib/llvm/bin:" + os.environ.get("PATH", "")
OBJDUMP, READELF = shutil.which("llvm-objdump", path=TOOLS), shutil.which("llvm-readelf", path=TOOLS)


@pytest.mark.skipif(OBJDUMP is None or READELF is None, reason="no llvm-objdump or llvm-readelf")
def test_kernels_that_count_loads_spill_nothing(tmp_path):
    shutil.copy(S.library_path(), tmp_path / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=tmp_path, check=True, capture_output=True)
    seen = 0
    for name in sorted(os.listdir(tmp_path)):
        if "gfx950" not in name:
            continue
        notes = subprocess.run([READELF, "--notes", name], cwd=tmp_path, check=True, capture_output=True, text=True).stdout
        for kernel in re.split(r"\n  - \.agpr_count", notes)[1:]:
            fields = dict(re.findall(r"^    \.(\w+):\s+(\S+)$", kernel, re.M))
            if "attn_few_kernel" in fields["name"]:
                seen += 1
                assert fields["private_segment_fixed_size"] == "0" == fields["vgpr_spill_count"], fields["name"]
    assert seen == 11             # four widths in bf16, seven in fp32
