"""Kernels of several rows per sequence keep nothing in scratch memory, read from the notes of the built library."""
import re
import subprocess

from paper_2601_16986_amd import ckv
from tests.test_kernel_resources_cpu import _tool


def test_nothing_is_kept_in_scratch(tmp_path):
    fat, part, co = (str(tmp_path / x) for x in ("fat", "part", "co"))
    subprocess.run([_tool("llvm-objcopy"), f"--dump-section=.hip_fatbin={fat}", ckv.LIB_PATH, str(tmp_path / "copy.so")], check=True)
    with open(fat, "rb") as f:
        bundles = f.read().split(b"__CLANG_OFFLOAD_BUNDLE__")[1:]         # one of each source
    got = {}
    for bundle in bundles:
        with open(part, "wb") as f:
            f.write(b"__CLANG_OFFLOAD_BUNDLE__" + bundle)
        subprocess.run([_tool("clang-offload-bundler"), "--type=o", "--unbundle", f"--input={part}", "--targets=hipv4-amdgcn-amd-amdhsa--gfx950", f"--output={co}"], check=True)
        notes = subprocess.run([_tool("llvm-readelf"), "--notes", co], check=True, capture_output=True, text=True).stdout
        for block in re.split(r"\n  - ", notes):
            name = re.search(r"\.name:\s+(_Z\S+)", block)
            if name and re.search(r"paged_(rows|attend|append_rotated|join)", name.group(1)):
                got[name.group(1)] = {k: int(v) for k, v in re.findall(r"\.(\w+):\s+(\d+)$", block, re.M)}
    assert len(got) >= 24
    for n, k in got.items():
        assert k["vgpr_spill_count"] == 0 and k["private_segment_fixed_size"] == 0, f"{n}: {k['vgpr_spill_count']} vector registers spilled"
