"""Rules of the chunk attention's inline assembly, checked on the ISA the build produces.  CPU only."""
import os
import re
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_13327_amd", "csrc")

pytestmark = pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc not available")


@pytest.fixture(scope="module")
def blocks(tmp_path_factory):
    """The inline assembly of the kernels, block by block, as lists of instructions."""
    asm = tmp_path_factory.mktemp("isa") / "chunk_attn.s"
    subprocess.check_call(["hipcc", "--offload-arch=gfx950", "-O3", "-std=c++17", "-S", "--cuda-device-only", "-Xclang", "-target-feature",
                           "-Xclang", "-packed-fp32-ops", os.path.join(CSRC, "chunk_attn.hip"), "-o", str(asm)], stderr=subprocess.DEVNULL)
    found = re.findall(r";;#ASMSTART\n(.*?);;#ASMEND", asm.read_text(), re.S) or re.findall(r";APP\n(.*?);NO_APP", asm.read_text(), re.S)
    return [[line.split(";")[0].strip() for line in block.splitlines() if line.split(";")[0].strip()] for block in found]


def test_fetches_leave_m0_as_it_was(blocks):
    """m0 cannot be named among what an asm statement overwrites, so the fetches put back what they found there."""
    fetches = [b for b in blocks if any(i.startswith("global_load_lds") for i in b)]
    assert len(fetches) > 20
    for b in fetches:
        keep = re.fullmatch(r"s_mov_b32 (s\d+), m0", b[0])
        assert keep and b[-1] == f"s_mov_b32 m0, {keep[1]}", b
        assert re.fullmatch(r"s_mov_b32 m0, s\d+", b[1]) and b[1].split()[-1] != keep[1] and b[2] == "s_nop 0" and len(b) == 5, b
