"""Every load into LDS of the built library finds its resource settled.

The loads stand in assembly, so the compiler does not know that they read their four scalar registers.  A vector instruction (a readfirstlane, a
readlane, a compare) that writes a scalar register must be five wait states ahead of a vector-memory instruction that reads it; an
instruction is one, s_nop n is n + 1."""
import os
import re
import shutil
import subprocess

import pytest

import paper_2602_11543_amd as S

OBJDUMP = shutil.which("llvm-objdump", path="/opt/rocm/llvm/bin:/opt/rocm/lib/llvm/bin:" + os.environ.get("PATH", ""))
STATES = 5


def scalars(text):
    """Numbers of the scalar registers in an operand."""
    m = re.match(r"s\[(\d+):(\d+)\]$", text)
    if m:
        return set(range(int(m[1]), int(m[2]) + 1))
    m = re.match(r"s(\d+)$", text)
    return {int(m[1])} if m else set()


def check(lines):
    """Number of loads into LDS in a disassembly, and those that come too soon."""
    loads, bad, written, last_label = 0, [], {}, 0          # written: scalar register -> wait states since a vector instruction wrote it
    for n, line in enumerate(lines):
        text = line.split("//")[0].strip()
        if not re.match(r"[a-z]\w+(\s|$)", text):
            continue                                          # (labels: what was written ahead of them still counts)
        op, _, rest = text.partition(" ")
        operands = [o.strip() for o in rest.split(",")]
        if op.startswith("buffer_load") and text.endswith(" lds"):
            loads += 1
            if any(r in written for r in scalars(operands[1])):
                bad.append((n, text))
        passed = 1 + (int(operands[0], 0) if op == "s_nop" else 0)
        written = {r: a + passed for r, a in written.items() if a + passed < STATES}
        if op.startswith("v_"):
            for o in operands[:2]:                             # a destination, or a vector one and a carry
                for r in scalars(o) if op.startswith(("v_readfirstlane", "v_readlane", "v_cmp")) or o is operands[1] and "_co_" in op or o is operands[1] and op.startswith(("v_mad_u64", "v_mad_i64", "v_div_scale")) else ():
                    written[r] = 0
                if op.startswith(("v_readfirstlane", "v_readlane", "v_cmp")):
                    break
        elif op.startswith("s_") and operands and not op.startswith(("s_nop", "s_waitcnt", "s_cmp", "s_cbranch", "s_branch", "s_barrier")):
            for r in scalars(operands[0]):
                written.pop(r, None)                           # a scalar instruction's result is there
    return loads, bad


@pytest.mark.skipif(OBJDUMP is None, reason="no llvm-objdump")
def test_resource_of_every_load(tmp_path):
    shutil.copy(S.library_path(), tmp_path / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=tmp_path, check=True, capture_output=True)
    total = 0
    for name in sorted(os.listdir(tmp_path)):
        if "gfx950" in name:
            text = subprocess.run([OBJDUMP, "-d", "--symbolize-operands", name], cwd=tmp_path, check=True, capture_output=True, text=True).stdout
            loads, bad = check(text.splitlines())
            assert not bad, (name, len(bad), bad[:3])
            total += loads
    assert total > 1000


def test_the_rule_itself():
    load, read = "\tbuffer_load_dwordx4 v1, s[4:7], 0 offen lds", "\tv_readfirstlane_b32 s5, v2   // 0: x"
    other = "\tv_add_u32_e32 v0, v1, v2"
    assert len(check([read, load])[1]) == 1 and len(check([read, other, other, load])[1]) == 1 and len(check([read] + 4 * [other] + [load])[1]) == 1
    assert check([read] + 5 * [other] + [load])[1] == [] and check([read, "\ts_nop 4", load])[1] == []
    assert len(check([read, "\ts_nop 3", load])[1]) == 1
    assert check([read, "\ts_mov_b32 s5, s9", load])[1] == []
    assert len(check(["\tv_cmp_lt_i32_e64 s[6:7], v0, v1", "<L1>:", load])[1]) == 1
    assert check([read.replace("s5", "s8"), load])[1] == [] and check([load])[0] == 1
