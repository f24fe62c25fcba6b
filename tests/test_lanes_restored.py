"""CPU check of the compiled kernels: no lane is missed by what the compiler adds where branches meet.

Lanes that skip a region come back where it ends: there the execution mask is widened first, and then the registers are moved on.  In a kernel that
uses all its registers the compiler has been seen to put copies of registers into others in front of that (a register of scalars
being spilled at the same place), for the lanes of the region only; the others read stale addresses later.  Such code may fault, so it is looked
for in the built library, whose kernels are disassembled."""
import os
import re
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

import paper_2602_16249_amd as aff

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
LINE = re.compile(r"^\t(\S+)(.*?)\s*// 0*([0-9A-F]+):.*?(?:<(\S+?)(?:\+0x([0-9a-f]+))?>)?$")
WIDENS = re.compile(r"s_(or|mov)_b64 exec,|s_(or|andn2|xor)_saveexec_b64 ")
LEAVES = re.compile(r"s_c?branch|s_endpgm|s_setpc|s_and_saveexec_b64 |s_and(n2)?_b64 exec,")
WRITES = re.compile(r"v_(?!cmp|readlane|readfirstlane|writelane)|scratch_|ds_|global_|buffer_|flat_")


def _missed(text):
    """(kernel, instructions) that stand between the target of a branch around a region, or the end of a loop that lanes leave one by one, and the
    instruction that widens the mask there."""
    found = []
    kernel, code, targets = "", [], set()

    def finish():
        for at in targets:
            block = []
            for op in code[places[at]:places[at] + 500] if at in places else ():
                if WIDENS.match(op):
                    if block:
                        found.append((kernel, block))
                    break
                if LEAVES.match(op):
                    break
                if WRITES.match(op):
                    block.append(op)

    places, start, loop_ends = {}, 0, False
    for line in text.splitlines():
        head = re.match(r"^0*([0-9a-f]+) <(\S+)>:", line)
        if head:
            finish()
            kernel, start, code, targets, places, loop_ends = head[2], int(head[1], 16), [], set(), {}, False
            continue
        m = LINE.match(line)
        if not m:
            continue
        op = m[1] + " " + m[2].strip()
        places[int(m[3], 16)] = len(code)
        code.append(op)
        if m[1] == "s_cbranch_execz" and m[4]:
            targets.add(start + int(m[5] or "0", 16))
        if loop_ends:
            targets.add(int(m[3], 16))
        loop_ends = m[1] == "s_cbranch_execnz" and int(m[2]) >= 0x8000  # (backwards)
    finish()
    return found


GOOD = """0000000000000100 <kernel>:
\ts_and_saveexec_b64 s[2:3], vcc                             // 000000000100: BE82206A
\ts_cbranch_execz 2                                          // 000000000104: BF880002 <kernel+0xc>
\tv_mov_b32_e32 v1, 0                                        // 000000000108: 7E020280
\ts_or_b64 exec, exec, s[2:3]                                // 00000000010C: 87FE027E
\tv_accvgpr_write_b32 a1, v7                                 // 000000000110: D3D94001 18000107
"""
BAD = GOOD.replace("00000000010C: 87FE027E", "000000000114: 87FE027E").replace("000000000110: D3D94001", "00000000010C: D3D94001")


def test_the_check_itself():
    lines = BAD.splitlines()
    lines[-2:] = lines[:-3:-1]
    assert _missed(GOOD) == []
    assert _missed("\n".join(lines)) == [("kernel", ["v_accvgpr_write_b32 a1, v7"])]


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no disassembler")
@pytest.mark.parametrize("library", ["libaffmae.so", "libaffmae_timed.so"])
def test_no_lane_is_missed_where_branches_meet(tmp_path, library):
    aff.load_library()  # (builds both where nothing is built)
    shutil.copy(os.path.join(os.path.dirname(aff.library_path()), library), tmp_path / "library.so")
    subprocess.run([OBJDUMP, "--offloading", "library.so"], cwd=tmp_path, check=True, capture_output=True)
    parts = sorted(p for p in os.listdir(tmp_path) if p.endswith("gfx950"))
    assert len(parts) > 10, parts

    def check(part):
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", part], cwd=tmp_path, check=True, capture_output=True, text=True).stdout
        assert "s_endpgm" in text or os.path.getsize(tmp_path / part) < 4096, part
        return _missed(text)

    with ThreadPoolExecutor(max_workers=8) as pool:
        found = [x for some in pool.map(check, parts) for x in some]
    assert not found, found[:5]
