"""The linear layers' tile kernel turns blocks through LDS between the lanes of
one wavefront.  LDS serves a wavefront in order, but nothing else keeps the
compiler from reading before other lanes' writes: in the kernel's intermediate
code no LDS read follows an LDS write of the epilogue without a fence of the
wavefront between them, and none is overwritten unfenced.  Compiled here from
the sources, the smallest tile; its epilogue is every tile's."""
import os
import re
import subprocess

import pytest

from paper_2111_13824_amd import build


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """The lines of each kernel's intermediate code, by its mangled name."""
    out = str(tmp_path_factory.mktemp("ir") / "tile.ll")
    flags = [f for f in build.FLAGS if f not in ("-shared", "-fPIC")]
    subprocess.run([build.HIPCC, *flags, "-DFQ_TILE_64", "-I", os.path.join(build.ROOT, "include"), "-I",
                    build.CSRC, "--offload-device-only", "-emit-llvm", "-S",
                    os.path.join(build.CSRC, "linear_tile.hip"), "-o", out], check=True, capture_output=True)
    with open(out) as f:
        text = f.read()
    found = re.findall(r"^define [^\n]*@(\w*linear_tile_kernel\w*)\([^\n]*\{\n(.*?)^\}", text, re.M | re.S)
    # the form whose loads go straight into LDS: its loop has no LDS writes of its own
    return {name: body.split("\n") for name, body in found if "ELb1ELi3EE" in name}


def test_reads_after_other_lanes_writes_are_fenced(kernels):
    assert len(kernels) == 7
    for name, lines in kernels.items():
        last = max(i for i, x in enumerate(lines) if "s_barrier" in x or 'syncscope("workgroup")' in x)
        # acc, residual: the last two of the kernel's template arguments
        residual, acc = (x == "1" for x in re.search(r"Lb(\d)ELb(\d)EEEv", name).groups())
        written = read = False
        fences = reads = 0
        for x in lines[last + 1:]:                     # 16 bytes a lane; the table's values are single ones
            if 'fence syncscope("wavefront") acquire' in x:
                written = read = False
                fences += 1
            elif re.search(r"\bstore <4 x i32> .*addrspace\(3\)", x):
                assert not read or residual, (name, x)       # a residual's lane overwrites what it alone read
                written = True
            elif re.search(r"\bload <4 x i32>, ptr addrspace\(3\)", x):
                assert not written, (name, x)
                read = True
                reads += 1
        assert reads > 0
        assert fences == (4 if acc else 3 if residual else 2), name
