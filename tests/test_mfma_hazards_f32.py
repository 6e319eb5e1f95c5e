"""The fp32 multiplications of the attention kernels take twice the passes of the bf16 ones (8 on gfx950), so their results have to be left
alone for longer: 10 wait states, where tests/test_mfma_hazards.py looks 8 behind every MFMA.  Along every path that branches leave open, in
the built library's code."""
import os
import shutil
import subprocess

import pytest

from paper_2602_19362_amd import oapl
from tests.test_mfma_hazards import OBJDUMP, VECTOR, _functions, _registers

SHAPE, STATES = "v_mfma_f32_16x16x4_f32", 10


def hazards(listing):
    found, multiplications = [], 0
    for code, labels in _functions(listing):
        regs = [[_registers(x) for x in operands] for _, _, operands, _ in code]
        for i, (_, op, _, _) in enumerate(code):
            if op != SHAPE:
                continue
            multiplications += 1
            result, seen, todo = regs[i][0], set(), [(i, 0)]
            while todo:
                at, passed = todo.pop()
                follow = [] if code[at][1] in ("s_branch", "s_endpgm") else [at + 1]
                if code[at][1].startswith(("s_branch", "s_cbranch")):
                    follow.append(labels[code[at][2][0]])
                for n in follow:
                    if n >= len(code) or passed >= STATES or (n, passed) in seen:
                        continue
                    seen.add((n, passed))
                    text, name, _, states = code[n]
                    if name.startswith("v_mfma"):
                        dst, a, b, c = regs[n][:4]
                        bad = result & (a | b) or (result & (c | dst) and not result == c == dst)
                    else:
                        bad = name.startswith(VECTOR) and result & frozenset().union(*regs[n])
                    if bad:
                        found.append(text)
                    todo.append((n, passed + states))
    return found, multiplications


MFMA = "v_mfma_f32_16x16x4_f32 v[20:23], v0, v4, v[20:23]"


@pytest.mark.parametrize("listing, bad", [
    ([MFMA, "s_nop 7", "v_mov_b32_e32 v9, v23"], 1),
    ([MFMA, "s_nop 7", "s_nop 0", "v_mov_b32_e32 v9, v23"], 1),
    ([MFMA, "s_nop 7", "s_nop 1", "v_mov_b32_e32 v9, v23"], 0),
    ([MFMA, "s_nop 7", "v_mov_b32_e32 v20, v9"], 1),
    ([MFMA, MFMA], 0),
    ([MFMA, "s_nop 7", "v_mfma_f32_16x16x4_f32 v[30:33], v20, v4, v[30:33]"], 1),
    ([MFMA, "s_nop 7", "v_mfma_f32_16x16x32_bf16 v[20:23], v[0:3], v[4:7], v[20:23]"], 0),
    (["<L1>:", "v_add_f32_e32 v9, v23, v9", MFMA, "s_nop 7", "s_cbranch_scc0 L1", "s_endpgm"], 1),
    (["v_mfma_f32_16x16x32_bf16 v[20:23], v[0:3], v[4:7], v[20:23]", "s_nop 7", "v_mov_b32_e32 v9, v23"], 0),
])
def test_the_reader_sees_hazards(listing, bad):
    assert len(hazards(listing)[0]) == bad


def test_no_hazards_in_the_built_library(tmp_path):
    assert os.path.exists(OBJDUMP), "the distances cannot be checked without the compiler's llvm-objdump"
    lib = tmp_path / "lib.so"
    shutil.copy(oapl.lib_path(), lib)
    subprocess.run([OBJDUMP, "--offloading", lib.name], cwd=tmp_path, check=True, stdout=subprocess.DEVNULL)
    code = [f for f in os.listdir(tmp_path) if f.endswith("gfx950")]
    assert len(code) == 1
    out = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", "--no-leading-addr", "--symbolize-operands", code[0]], cwd=tmp_path, check=True,
                         stdout=subprocess.PIPE, text=True).stdout
    found, multiplications = hazards(out.splitlines())
    assert multiplications > 1000
    assert not found, found[:10]
