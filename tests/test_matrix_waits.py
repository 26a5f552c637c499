"""Wait states behind the matrix instructions of the built kernels (CPU only: a listing of
the code objects in libspot.so).

An instruction that uses the result of a 16x16 matrix instruction of four passes has to
come 8 wait states after it, on every path.  The compiler (ROCm 7.2) counts them along one
path only where a branch lies between: behind an `if` that can be skipped, results have
been read 1 to 3 states after the last product, without it.
"""
import os
import re
import subprocess

import pytest

from paper_2606_22874_amd import build
from test_kernel_resources import MARK

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
STATES = 8
REG = re.compile(r"\b([va])(?:\[(\d+):(\d+)\]|(\d+)\b)")


def regs(operand):
    out = set()
    for kind, lo, hi, one in REG.findall(operand):
        out |= {(kind, i) for i in (range(int(lo), int(hi) + 1) if lo else [int(one)])}
    return out


def functions(listing):
    """(name, [(op, operands)], {label: index}) of each function with matrix instructions."""
    for part in re.split(r"\n(?=[0-9a-f]* ?<_Z)", listing):
        if "v_mfma" not in part:
            continue
        code, labels = [], {}
        for line in part.split("\n")[1:]:
            line = line.split("//")[0].strip()
            if line.startswith("<L"):
                labels[line[1:-2]] = len(code)
            elif line and not line.endswith(":"):
                op, _, rest = line.partition(" ")
                code.append((op, rest.strip()))
        yield part.split("\n")[0], code, labels


def early(code, labels):
    """(matrix instruction, the one that uses its result too early, states between)."""
    found = []
    for i, (op, rest) in enumerate(code):
        if not op.startswith("v_mfma"):
            continue
        todo = [(i + 1, 0, regs(rest.split(",")[0]))]
        while todo:
            at, age, live = todo.pop()
            while age < STATES and live and at < len(code):
                op, rest = code[at]
                if op.startswith("v_mfma"):
                    d, a, b = (regs(x) for x in rest.split(",")[:3])
                    if live & (a | b):
                        found.append((i, at, age))
                        break
                    live = live - d              # later ones count from there
                elif op[:2] in ("v_", "ds") or op.split("_")[0] in ("global", "flat", "buffer",
                                                                    "scratch"):
                    if live & regs(rest):
                        found.append((i, at, age))
                        break
                elif op in ("s_endpgm", "s_setpc_b64"):
                    break
                elif op == "s_branch":
                    at, age = labels[rest], age + 1
                    continue
                elif op.startswith("s_cbranch"):
                    todo.append((labels[rest], age + 1, live))
                age += int(rest, 0) + 1 if op == "s_nop" else 1
                at += 1
    return found


SKIPPED = """
0000 <_Zsample>:
\tv_mfma_f32_16x16x32_bf16 v[8:11], v[0:3], v[4:7], v[8:11]
\ts_and_saveexec_b64 s[20:21], s[14:15]
\ts_cbranch_execz L0
\tv_readfirstlane_b32 s2, v30
\ts_nop %d
<L0>:
\ts_or_b64 exec, exec, s[20:21]
%s\tv_mul_f32_e32 v20, v21, v%d
\ts_endpgm
"""


def test_a_path_around_the_states_is_found():
    """The states that the compiler counted lie in a block that is skipped."""
    def look(text):
        (_, code, labels), = functions(text)
        return early(code, labels)
    assert look(SKIPPED % (7, "", 9)) == [(0, 6, 3)]
    assert look(SKIPPED % (7, "\ts_nop 3\n", 9)) == [(0, 7, 7)]
    assert look(SKIPPED % (7, "\ts_nop 4\n", 9)) == []       # eight on the short path too
    assert look(SKIPPED % (0, "\ts_nop 7\n", 9)) == []
    assert look(SKIPPED % (0, "", 12)) == []                 # another register


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="needs llvm-objdump")
def test_results_are_not_used_too_early(tmp_path):
    if not os.path.exists(build.SO):
        build.build()
    with open(build.SO, "rb") as f:
        data = f.read()
    count = 0
    for m in re.finditer(re.escape(MARK), data):
        at, nxt = data.find(b"\x7fELF", m.start()), data.find(MARK, m.start() + 1)
        if at < 0:
            continue
        obj = tmp_path / "code.o"
        obj.write_bytes(data[at:nxt if nxt > 0 else len(data)])
        listing = subprocess.run([OBJDUMP, "-d", "--symbolize-operands", "--no-show-raw-insn",
                                  "--no-leading-addr", str(obj)], capture_output=True, text=True,
                                 check=True).stdout
        for name, code, labels in functions(listing):
            count += sum(op.startswith("v_mfma") for op, _ in code)
            for i, j, age in early(code, labels):
                raise AssertionError((name, code[i], code[j], age))
    assert count > 10000
