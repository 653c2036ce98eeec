"""The benchmark's hash of the attention kernels' device code, under which counters
are recorded: it changes with that code and with nothing else in the library."""
import os
import re

import pytest

import bench
from paper_2606_12688_amd import attn
from tests.test_build_code_object import LLVM
from tests.test_cache_code_object import TOOLS, _tool


@pytest.mark.skipif(not all(os.path.exists(os.path.join(LLVM, t)) for t in TOOLS), reason="ROCm LLVM tools missing")
def test_hash_follows_the_kernels_code_only(tmp_path, monkeypatch):
    if not os.path.exists(attn.LIB_PATH):
        pytest.skip("library not built")
    with open(attn.LIB_PATH, "rb") as f:
        lib = f.read()
    fat = tmp_path / "fatbin"
    _tool("llvm-objcopy", f"--dump-section=.hip_fatbin={fat}", attn.LIB_PATH, str(tmp_path / "stripped.so"))
    data = fat.read_bytes()
    starts = [m.start() for m in re.finditer(b"__CLANG_OFFLOAD_BUNDLE__", data)] + [len(data)]
    text = {}  # offset in the library of the code of the object with the kernels, and of the 4-bit cache's
    for i, (a, b) in enumerate(zip(starts[:-1], starts[1:])):
        part, co = tmp_path / f"part{i}", tmp_path / f"part{i}.co"
        part.write_bytes(data[a:b])
        _tool("clang-offload-bundler", "--unbundle", "--type=o", f"--input={part}",
              "--targets=hipv4-amdgcn-amd-amdhsa--gfx950", f"--output={co}")
        sections = _tool("llvm-readelf", "-S", "--wide", str(co))
        offset = int(re.search(r"\]\s+\.text\s+\S+\s+\S+\s+(\S+)", sections).group(1), 16)
        elf = co.read_bytes()
        kind = "4bit" if b"few4_kernel" in elf else "kernels" if b"merge_kernel" in elf else None
        if kind:
            assert lib.count(elf) == 1
            text[kind] = lib.index(elf) + offset
    want = bench.kernel_code_sha()
    assert re.fullmatch("[0-9a-f]{16}", want) and want == bench.kernel_code_sha()
    for kind, same in (("4bit", True), ("kernels", False)):
        other = bytearray(lib)
        other[text[kind] + 64] ^= 1
        path = tmp_path / f"{kind}.so"
        path.write_bytes(other)
        monkeypatch.setattr(attn, "LIB_PATH", str(path))
        assert (bench.kernel_code_sha() == want) == same, kind
        monkeypatch.undo()
    path = tmp_path / "empty.so"
    path.write_bytes(b"\x7fELF")
    monkeypatch.setattr(attn, "LIB_PATH", str(path))
    with pytest.raises(RuntimeError):
        bench.kernel_code_sha()
