"""Rules of the chunk attention's inline assembly, checked on the ISA the build produces.  CPU only."""
import os
import re
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_13327_amd", "csrc")

pytestmark = pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc not available")


@pytest.fixture(scope="module")
def text(tmp_path_factory):
    asm = tmp_path_factory.mktemp("isa") / "chunk_attn.s"
    subprocess.check_call(["hipcc", "--offload-arch=gfx950", "-O3", "-std=c++17", "-S", "--cuda-device-only", "-Xclang", "-target-feature",
                           "-Xclang", "-packed-fp32-ops", os.path.join(CSRC, "chunk_attn.hip"), "-o", str(asm)], stderr=subprocess.DEVNULL)
    return asm.read_text()


INLINE = re.compile(r";;#ASMSTART\n(.*?);;#ASMEND", re.S)


def _instructions(s):
    return [line.split(";")[0].strip() for line in s.splitlines() if line.split(";")[0].strip()]


def test_fetches_leave_m0_as_it_was(text):
    """m0 cannot be named among what an asm statement overwrites, so the fetches put back what they found there."""
    fetches = [b for b in map(_instructions, INLINE.findall(text)) if any(i.startswith("global_load_lds") for i in b)]
    assert len(fetches) > 20
    for b in fetches:
        keep = re.fullmatch(r"s_mov_b32 (s\d+), m0", b[0])
        assert keep and b[-1] == f"s_mov_b32 m0, {keep[1]}", b
        assert re.fullmatch(r"s_mov_b32 m0, s\d+", b[1]) and b[1].split()[-1] != keep[1] and b[2] == "s_nop 0" and len(b) == 5, b


def test_rows_on_their_way_are_waited_for_by_their_count(text):
    """A wavefront has 4 loads of a tile and 8 of a step on their way with heads of 128, 2 and 4 with heads of 64: the next one's may stay
    there, or none.  The compiler's own waits count everything, so where rows are fetched or multiplied there are none."""
    kernels = re.split(r"(?m)^_ZN3etc22chunk_attention_kernelILi(\d+)E\w+:", text)[1:]
    assert kernels[0::2] == ["128", "64"]
    for head, body in zip(kernels[0::2], kernels[1::2]):
        body = body.split(".Lfunc_end")[0]
        waits = [int(n) for b in INLINE.findall(body) for n in re.findall(r"s_waitcnt vmcnt\((\d+)\)", b)]
        assert set(waits) == {"128": {0, 4, 8}, "64": {0, 2, 4}}[head]
        busy = [b for b in re.split(r"(?m)^(?:\.LBB\w+:|; %bb\.\d+:)", body) if "global_load_lds" in b or "v_mfma" in b]
        assert len(busy) > 10
        for b in busy:
            assert "vmcnt" not in INLINE.sub("", b)
