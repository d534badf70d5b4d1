"""The compiler waits for a matrix instruction's result before a vector instruction that
it knows reads it, and for nothing before inline asm.  In the attention over the cache no
vector instruction of inline asm reads a register that a matrix instruction may have
written last, on any way through a kernel.  Compiled here from the sources: heads of up to
64 channels, whose code is every width's."""
import os
import re
import subprocess

import pytest

from paper_2111_13824_amd import build


def registers(operand):
    found = set()
    for m in re.finditer(r"\bv\[(\d+):(\d+)\]|\bv(\d+)\b", operand):
        found |= {int(m.group(3))} if m.group(3) else set(range(int(m.group(1)), int(m.group(2)) + 1))
    return found


class Block:
    def __init__(self):
        self.code, self.next, self.falls = [], [], True     # code: (op, written, read, whether it is asm)


def blocks(text):
    """The basic blocks of a kernel's listing, by label."""
    found, now, inside = {"": Block()}, "", False
    for line in text.split("\n"):
        line = line.strip()
        label = re.match(r"^(\.LBB\w+):", line)
        if label or (found[now].code and not found[now].falls):
            new = label.group(1) if label else f"behind {len(found)}"
            if found[now].falls:
                found[now].next.append(new)
            now = new
            found[now] = Block()
        if label:
            continue
        if "#ASMSTART" in line or "#ASMEND" in line:
            inside = "#ASMSTART" in line
            continue
        m = re.match(r"^([a-z]\w+)\s*([^;]*)", line)
        if not m:
            continue
        op, operands = m.group(1), [x.strip() for x in m.group(2).split(",")]
        stores = re.match(r"(global|flat|buffer)_(store|atomic)|ds_(write|store|add|max)|v_cmp|v_readlane|v_readfirst", op)
        written = set() if stores else registers(operands[0])
        read = set().union(*map(registers, operands if stores else operands[1:]), set())
        found[now].code.append((op, written, read, inside))
        if op.startswith("s_cbranch"):
            found[now].next.append(operands[0])
            behind = f"behind {len(found)}"
            found[now].next.append(behind)
            now = behind
            found[now] = Block()
        elif op == "s_branch":
            found[now].next.append(operands[0])
            found[now].falls = False
        elif op == "s_endpgm":
            found[now].falls = False
    return found


def through(block, state, bad=None):
    """Registers whose last writer may be a matrix instruction, behind the block."""
    state = set(state)
    for op, written, read, inside in block.code:
        if bad is not None and inside and op.startswith("v_") and read & state:
            bad.append((op, sorted(read & state)))
        if op.startswith("v_mfma"):
            state |= written
        else:
            state -= written
    return state


def unwaited(text):
    found = blocks(text)
    before = {name: set() for name in found}
    work = list(found)
    while work:
        name = work.pop()
        after = through(found[name], before[name])
        for n in found[name].next:
            if n in before and not after <= before[n]:
                before[n] |= after
                work.append(n)
    bad = []
    for name, block in found.items():
        through(block, before[name], bad)
    return bad


def test_the_analysis_sees_a_way_around():
    """An accumulator that one way rewrites and the other does not; waits in asm are none."""
    start = "v_mfma_i32_16x16x64_i8 v[0:3], v[8:11], v[12:15], v[0:3]\ns_cbranch_scc1 .LBB0_2\n"
    middle = "v_cndmask_b32_e32 v2, v4, v2, vcc\n"
    end = ".LBB0_2:\n;;#ASMSTART\nv_med3_i32 v5, v2, s3, 0\n;;#ASMEND\ns_endpgm"
    assert unwaited(start + middle + end) == [("v_med3_i32", [2])]
    assert not unwaited(start.replace("s_cbranch_scc1 .LBB0_2\n", "") + middle + end)
    assert not unwaited((start + middle + end).replace(";;#", ";"))
    assert not unwaited(start + middle + end.replace("v_med3_i32 v5, v2, s3, 0", "s_waitcnt lgkmcnt(0)"))


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("asm") / "paged.s")
    flags = [f for f in build.FLAGS if f not in ("-shared", "-fPIC")]
    subprocess.run([build.HIPCC, *flags, "-DFQ_PAGED_64", "-I", os.path.join(build.ROOT, "include"), "-I",
                    build.CSRC, "--offload-device-only", "-S", os.path.join(build.CSRC, "lis_paged.hip"), "-o", out],
                   check=True, capture_output=True)
    with open(out) as f:
        text = f.read()
    return dict(re.findall(r"^(_Z\w*lis_paged_kernel\w*):[^\n]*\n(.*?)^\.Lfunc_end", text, re.M | re.S))


def test_no_inline_asm_reads_a_matrix_result(kernels):
    assert len(kernels) > 20
    asm = 0
    for name, text in kernels.items():
        bad = unwaited(text)
        assert not bad, (name, len(bad), bad[:3])
        asm += sum(inside and op.startswith("v_") for b in blocks(text).values() for op, _, _, inside in b.code)
    assert asm > 0
