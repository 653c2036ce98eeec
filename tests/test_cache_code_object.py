"""The device code of the operators on paged caches, a code object of its own in
the library: kernels without calls (see test_build_code_object.py), and no
spilled registers in the kernels that take rows of the 4-bit cache from memory."""
import os
import re
import subprocess

import pytest

from paper_2606_12688_amd import attn
from tests.test_build_code_object import LLVM, TOOLS

TOOLS = (*TOOLS, "llvm-readelf")


def _tool(name, *args):
    return subprocess.run([os.path.join(LLVM, name), *args], check=True, capture_output=True, text=True).stdout


@pytest.mark.skipif(not all(os.path.exists(os.path.join(LLVM, t)) for t in TOOLS), reason="ROCm LLVM tools missing")
def test_cache_kernels(tmp_path):
    if not os.path.exists(attn.LIB_PATH):
        pytest.skip("library not built")
    fat = tmp_path / "fatbin"
    _tool("llvm-objcopy", f"--dump-section=.hip_fatbin={fat}", attn.LIB_PATH, str(tmp_path / "stripped.so"))
    data = fat.read_bytes()
    starts = [m.start() for m in re.finditer(b"__CLANG_OFFLOAD_BUNDLE__", data)] + [len(data)]
    found = []
    for i, (a, b) in enumerate(zip(starts[:-1], starts[1:])):
        part, co = tmp_path / f"part{i}", tmp_path / f"part{i}.co"
        part.write_bytes(data[a:b])
        _tool("clang-offload-bundler", "--unbundle", "--type=o", f"--input={part}",
              "--targets=hipv4-amdgcn-amd-amdhsa--gfx950", f"--output={co}")
        notes = _tool("llvm-readelf", "--notes", str(co))
        if "few4_kernel" not in notes:
            continue
        found += re.findall(r"\.name:\s+(\S*_kernel\S*)", notes)
        assert "s_swappc" not in _tool("llvm-objdump", "-d", "--no-show-raw-insn", str(co))
        for block in notes.split(".agpr_count")[1:]:
            name = re.search(r"\.name:\s+(\S+)", block).group(1)
            if "tile_kernel" not in name:
                assert re.search(r"\.vgpr_spill_count:\s+0\b", block), name
    for kernel in ("append4_kernel", "unpack4_kernel", "few4_kernel", "tile_kernel", "tables_kernel"):
        assert any(kernel in n for n in found), kernel
