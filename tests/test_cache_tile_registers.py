"""Spilled registers of the 4-bit tile kernel, instance by instance, in the built
code object: none with key groups and at D = 128 but for one instance, a few at
D = 64 where four waves share a SIMD's registers.  The counts may fall; one that
grows puts reloads into the tile loop."""
import os
import re

import pytest

from paper_2606_12688_amd import attn
from tests.test_build_code_object import LLVM
from tests.test_cache_code_object import TOOLS, _tool

ROWS, PACKED, CASCADE = 0, 1, 2


def _limit(d, mode, keys, groups, few):
    """Spilled VGPRs of tile_kernel<d, 2, 4-bit pool, mode, keys, groups, few>."""
    if groups > 1:
        return 0
    if d == 128:
        return 4 if keys == 32 and mode == ROWS and few else 0
    return {ROWS: 12, PACKED: 9, CASCADE: 4}[mode] if few else {ROWS: 4, PACKED: 4, CASCADE: 2}[mode]


@pytest.mark.skipif(not all(os.path.exists(os.path.join(LLVM, t)) for t in TOOLS), reason="ROCm LLVM tools missing")
def test_spills_of_every_instance(tmp_path):
    if not os.path.exists(attn.LIB_PATH):
        pytest.skip("library not built")
    fat = tmp_path / "fatbin"
    _tool("llvm-objcopy", f"--dump-section=.hip_fatbin={fat}", attn.LIB_PATH, str(tmp_path / "stripped.so"))
    data = fat.read_bytes()
    starts = [m.start() for m in re.finditer(b"__CLANG_OFFLOAD_BUNDLE__", data)] + [len(data)]
    seen = set()
    for i, (a, b) in enumerate(zip(starts[:-1], starts[1:])):
        part, co = tmp_path / f"part{i}", tmp_path / f"part{i}.co"
        part.write_bytes(data[a:b])
        _tool("clang-offload-bundler", "--unbundle", "--type=o", f"--input={part}",
              "--targets=hipv4-amdgcn-amd-amdhsa--gfx950", f"--output={co}")
        for block in _tool("llvm-readelf", "--notes", str(co)).split(".agpr_count")[1:]:
            # tile_kernel<d, rows, cache, mode, keys, groups, few>, cache 2 being the 4-bit pool
            name = re.search(r"\.name:\s+\S*tile_kernelILi(\d+)ELi2ELi2ELi(\d)ELi(\d+)ELi(\d)ELi(\d)E", block)
            if name:
                inst = tuple(int(x) for x in name.groups())
                seen.add(inst)
                spilled = int(re.search(r"\.vgpr_spill_count:\s+(\d+)", block).group(1))
                assert spilled <= _limit(*inst), (inst, spilled)
    assert {i[0] for i in seen} == {64, 128} and {i[1] for i in seen} == {ROWS, PACKED, CASCADE}
    assert {i[4] for i in seen} == {0, 1, 2} and len(seen) == 30, sorted(seen)
