"""The loops of the chunk attention wait for rows on their way to LDS by counting the wavefront's vector memory operations
(s_waitcnt vmcnt(n)): a reload of a spilled register is one more of them, waits for all rows in front of it and cost a quarter of the
time where the compiler put one there.  Checked on the ISA the build produces: no scratch memory at all.  CPU only."""
import os
import re
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_13327_amd", "csrc")

pytestmark = pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc not available")


def test_no_scratch_memory(tmp_path):
    asm = tmp_path / "chunk_attn.s"
    subprocess.check_call(["hipcc", "--offload-arch=gfx950", "-O3", "-std=c++17", "-S", "--cuda-device-only", "-Xclang", "-target-feature",
                           "-Xclang", "-packed-fp32-ops", os.path.join(CSRC, "chunk_attn.hip"), "-o", str(asm)], stderr=subprocess.DEVNULL)
    text = asm.read_text()
    kernels = re.findall(r"^(_ZN3etc22chunk_attention_kernel\w+):", text, re.M)
    assert len(kernels) == 2 and text.count("v_mfma_f32_32x32x16_bf16") > 100
    assert not re.findall(r"^\s+scratch_\w+", text, re.M)
    # what waits for rows also counts them: every fetch is followed by its counted wait, none by a compiler's
    assert text.count("global_load_lds_dwordx4") > 20
