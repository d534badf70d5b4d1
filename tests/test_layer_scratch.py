"""No kernel of the linear layers, the rotation and the heads' way back to rows
keeps registers in scratch memory, by the metadata of the code objects in
libfqvit.so.  (With 16 bytes a lane in the widest tile a product of 9232 x 1024 x
4096 with a table wrote 53 MB instead of 50.5 and read 84 instead of 82.)"""
import os
import re
import subprocess

import pytest

from test_kernel_scratch import READELF, _code_objects


@pytest.fixture(scope="module")
def scratch(tmp_path_factory):
    """Bytes of scratch a lane of every kernel, by mangled name."""
    from paper_2111_13824_amd import binding
    assert os.path.exists(binding.LIB_PATH), "libfqvit.so is not built"
    with open(binding.LIB_PATH, "rb") as f:
        data = f.read()
    sizes, path = {}, tmp_path_factory.mktemp("code") / "object.elf"
    for elf in _code_objects(data):
        path.write_bytes(elf)
        notes = subprocess.run([READELF, "--notes", str(path)], capture_output=True, text=True,
                               check=True).stdout
        for block in re.split(r"\n  - (?=\.)", notes)[1:]:
            name = re.search(r"^\s*\.name:\s+(_Z\S+)$", block, re.M)
            if name:
                sizes[name.group(1)] = int(re.search(r"\.private_segment_fixed_size:\s+(\d+)", block).group(1))
    return sizes


@pytest.mark.parametrize("kernel,instances", [("linear_tile_kernel", 63), ("linear_rows_kernel", 14),
                                              ("linear_fold_kernel", 1), ("rope_qkv_kernel", 9),
                                              ("rope_qkv_bytes_kernel", 1), ("requant_heads_kernel", 2)])
def test_kernels_hold_their_state(scratch, kernel, instances):
    found = {n: s for n, s in scratch.items() if re.search(rf"\d{kernel}[IE]", n)}
    assert len(found) == instances, sorted(found)
    bad = {n: s for n, s in found.items() if s}
    assert not bad, bad
