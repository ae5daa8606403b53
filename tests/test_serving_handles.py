"""Handles of the serving operators, on the CPU over a stub runtime (tests/serving_handles.cpp)."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "..", "paper_2604_13327_amd", "csrc")
HIP = "/opt/rocm/include"

pytestmark = pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir(HIP), reason="no compiler or HIP headers")


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    exe = tmp_path_factory.mktemp("serving") / "serving_handles"
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                           "-I", CSRC, "-I", HIP, "-o", str(exe), os.path.join(HERE, "serving_handles.cpp")])
    return str(exe)


@pytest.mark.parametrize("which", ["read_error", "memory"])
def test_handles(program, which):
    out = subprocess.run([program, which], capture_output=True, text=True, timeout=60)
    assert out.returncode == 0, out.stdout + out.stderr


def test_library_without_serving_operators_loads(tmp_path):
    """One that the front end generated for a graph before the serving operators were there."""
    from paper_2604_13327_amd import binding
    src, so = tmp_path / "old.c", tmp_path / "old.so"
    src.write_text("".join(f"int {name}(void) {{ return 0; }}\n" for name in binding.EXPORTS if not name.startswith("etc_serving_")))
    subprocess.check_call(["gcc", "-shared", "-fPIC", "-o", str(so), str(src)])
    L = binding.load_library(str(so))
    assert L.etc_graph_user_fn_count.argtypes and not hasattr(L, "etc_serving_create")


def test_page_arrays_go_together():
    """One without the other: refused by the call (on the device it is a status of -1 for every step that holds a page)."""
    import torch
    from paper_2604_13327_amd.binding import Serving
    sv = object.__new__(Serving)                          # the check comes in front of any use of the handle
    sv._h, sv._device, sv._i32 = None, 0, (torch.int32,)
    t = torch.zeros(2, dtype=torch.int32)
    for kw in ({"page_indptr": t}, {"page_ids": t}):
        with pytest.raises(ValueError, match="page_indptr and page_ids"):
            sv.tables(t, t, t.view(2, 1), t, t[:1], q_indptr=t, slots=t, positions=t, status=t[:1], **kw)
