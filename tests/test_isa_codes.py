"""The attention over a cache of codes waits for rows on their way to LDS by counting the wavefront's vector memory operations, and its second
product has its accumulators in registers beside two steps of codes: a reload of a spilled register inside a loop would wait for all rows in front of
it.  Checked on the ISA the build produces: scratch memory only beside the count of values that are no numbers, which runs where a tile holds some.
The append and the scores use none at all.  CPU only."""
import os
import re
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_13327_amd", "csrc")

pytestmark = pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc not available")


def _asm(tmp_path, source):
    out = tmp_path / (source + ".s")
    subprocess.check_call(["hipcc", "--offload-arch=gfx950", "-O3", "-std=c++17", "-S", "--cuda-device-only", "-Xclang", "-target-feature",
                           "-Xclang", "-packed-fp32-ops", os.path.join(CSRC, source), "-o", str(out)], stderr=subprocess.DEVNULL)
    return out.read_text()


def test_attention_loops_have_no_scratch_memory(tmp_path):
    text = _asm(tmp_path, "chunk_attn_codes.hip")
    assert len(re.findall(r"^(_ZN3etc28chunk_attention_codes_kernel\w+):", text, re.M)) == 2
    assert text.count("v_mfma_scale_f32_32x32x64_f8f6f4") > 20 and text.count("ds_read_b64_tr_b8") > 20
    # rows and scales come to LDS without registers
    assert text.count("global_load_lds_dwordx4") > 20 and text.count("global_load_lds_ubyte") >= 4
    for block in re.split(r"(?m)^(?=\.LBB\w+:)", text):
        if "v_mfma_scale" in block or "v_exp_f32" in block:
            assert "scratch_" not in block, block.split(":")[0]
    # no form of packed fp32 arithmetic
    assert not re.findall(r"^\s+v_pk_(?:add|mul|fma)_f32", text, re.M)


@pytest.mark.parametrize("source, kernel, n", [("append_codes.hip", "serving_append_codes_kernel", 8), ("score.hip", "serving_score_kernel", 2)])
def test_no_scratch_memory(tmp_path, source, kernel, n):
    text = _asm(tmp_path, source)
    assert len(re.findall(rf"^(_ZN3etc\d+{kernel}\w+):", text, re.M)) == n
    assert not re.findall(r"^\s+scratch_\w+", text, re.M)
    assert not re.findall(r"^\s+v_pk_(?:add|mul|fma)_f32", text, re.M)
